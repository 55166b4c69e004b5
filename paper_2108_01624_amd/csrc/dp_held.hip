// Gradients that the caller holds, many tensors X_l [B, n_l]: the squared norm of every unit over all of them, the clip-weighted sums
// and the scaled gradients.
//
// Roofline: HBM.  The norm reads every element once (one multiply-add each); the sums read it again and read and write 4 bytes per
// entry of the sums; the scaled form reads and writes it.  Rows start wherever n_l puts them: wide accesses are declared with the
// alignment of an element, which the hardware serves at any address.
//
// 334 M bf16 elements of 388 tensors, one unit: norms 112 us in three launches and their join (6.0 TB/s), sums 558 us (6.0 TB/s of reading and writing);
// 128 units of 96 tensors of 8,192 bf16 elements: norms 34 us (6.0 TB/s), sums 41; 41 M fp32 elements scaled: 56 us (5.9 TB/s).
#include "dp_common.h"

namespace {

constexpr int HELD_TABLE = 160;          // tensors per launch: their table is a kernel argument, of less than 4 KiB
constexpr int HELD_FEW = 32;             // a small table where it is enough (16 tensors: a call of the sums 4.7 -> 3.8 us of host time)
constexpr uint64_t HELD_ENTRY = 1ull << 31;  // most elements of an entry (32-bit counters have room behind them); one unit's longer tensors are several entries
constexpr uint64_t HELD_PIECE = 16384;   // elements of a workgroup of the norms (334 M bf16 in 388 tensors: 112 us; 4,096: 144, 65,536: 114)
constexpr int WAVE_ROW = 4096;           // rows up to this length are one wave's (256 units of 96 rows of 2,048 bf16: 45 us norms and sums; up to 1,024: 59)
constexpr unsigned ADD_GRID = 256;       // most workgroups, and units, of a launch of norms whose last workgroup adds them up (16 tensors of a small
                                         // block: a launch behind them costs a pass 5 us more)
constexpr int ADD_UNITS = 16;
constexpr int ADD_COLS = 256 * 4;        // columns of a workgroup of the sums, one unit
constexpr int SUM_COLS = 64 * 8;         // ... several units
constexpr uint64_t LAST_LEVEL = 192ull << 20;  // bytes of the 256 MiB behind the L2s that a gradient may count on
constexpr int FACTORS = 1024;            // clip factors in LDS at a time

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));
typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));

// Elements from any address of an element.  STREAM: with the non-temporal hint.  The second pass and the sums carry it; the norms do where the
// gradients are more than the last-level cache keeps for the second pass (164 MB fp32, norms and scaling: 87 us with cached norms, 97 with
// streamed ones; 668 MB bf16 streamed, norms alone: 112 us, cached 124).
template <bool BF16, bool STREAM = true>
struct Held {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    // (a template over the pointer's type would lose its alignment)
#define HELD_LD(type, p) (STREAM ? __builtin_nontemporal_load(reinterpret_cast<const type*>(p)) : *reinterpret_cast<const type*>(p))
    static __device__ __forceinline__ void load4(const elem* p, float v[4]) {
        if constexpr (BF16) {
            const u32x2_t w = HELD_LD(u32x2_a2, p);
            v[0] = dp_bf16_lo(w[0]);
            v[1] = dp_bf16_hi(w[0]);
            v[2] = dp_bf16_lo(w[1]);
            v[3] = dp_bf16_hi(w[1]);
        } else {
            const f32x4_t w = HELD_LD(f32x4_a4, p);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = w[k];
        }
    }
    static __device__ __forceinline__ void load8(const elem* p, float v[8]) {
        if constexpr (BF16) {
            const u32x4_t w = HELD_LD(u32x4_a2, p);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = dp_bf16_lo(w[k]);
                v[2 * k + 1] = dp_bf16_hi(w[k]);
            }
        } else {
            load4(p, v);
            load4(p + 4, v + 4);
        }
    }
    static __device__ __forceinline__ float load1(const elem* p) {
        if constexpr (BF16) return dp_bf16_bits_to_f32(*p);
        else return *p;
    }
    static __device__ __forceinline__ void store4(elem* p, const float v[4]) {
        if constexpr (BF16) {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            const bf16x4_t w = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            __builtin_nontemporal_store(__builtin_bit_cast(u32x2_t, w), reinterpret_cast<u32x2_a2*>(p));
        } else {
            __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_a4*>(p));
        }
    }
    static __device__ __forceinline__ void store1(elem* p, float v) {
        if constexpr (BF16) *reinterpret_cast<__bf16*>(p) = (__bf16)v;
        else *p = v;
    }
};

// The tensors of a launch.  Workgroups first[l] .. first[l + 1] - 1 are tensor l's.
template <int N>
struct HeldTable {
    const void* x[N];   // (pointers, not numbers: the compiler takes those of an argument for global memory)
    void* y[N];         // sums or scaled gradients; norms: the first of the tensor's partial norms, as a number
    uint32_t count[N];  // elements of a unit
    uint32_t first[N];
    int n;
};
typedef HeldTable<HELD_TABLE> HeldFull;

// launch(table): the full one, or a small copy of it.
template <typename Launch>
void with_table(const HeldFull& t, Launch launch) {
    if (t.n > HELD_FEW) return launch(t);
    HeldTable<HELD_FEW> few;
    for (int l = 0; l < t.n; ++l) {
        few.x[l] = t.x[l];
        few.y[l] = t.y[l];
        few.count[l] = t.count[l];
        few.first[l] = t.first[l];
    }
    few.n = t.n;
    launch(few);
}

// The tensor of workgroup b: a search by halves over scalar loads.  (Three entries a lane and ballots, one round of vector loads: 334 M bf16 elements
// added to their sums 555 us, 558 this way.)
template <int N>
__device__ __forceinline__ int held_tensor(const HeldTable<N>& t, uint32_t b) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= b) lo = mid;
        else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// workgroups of a row that is not one wave's (0: it is)
__host__ __device__ __forceinline__ uint32_t held_pieces(uint64_t count, uint32_t per) { return count <= WAVE_ROW ? 0 : (uint32_t)((count + per - 1) / per); }

// What of a tensor a workgroup (a wave, for short rows) does: elements [from, to) of a unit's `count`.
struct HeldPiece {
    int unit;
    uint32_t piece, from, to;
    int lane, lanes;
};
__device__ __forceinline__ HeldPiece held_piece(uint32_t count, uint32_t k, int B, uint32_t per) {
    HeldPiece p;
    const uint32_t pieces = held_pieces(count, per);
    if (pieces == 0) {
        p.unit = 4 * k + (threadIdx.x >> 6);
        p.piece = 0;
        p.from = 0;
        p.to = p.unit < B ? count : 0;
        p.lane = threadIdx.x & 63;
        p.lanes = 64;
    } else {
        p.unit = k / pieces;
        p.piece = k - p.unit * pieces;
        p.from = p.piece * per;
        p.to = count - p.from < per ? count : p.from + per;
        p.lane = threadIdx.x;
        p.lanes = 256;
    }
    return p;
}

// part[unit * J + y[l] + piece] = sum of squares.  Four independent chains a thread, four loads in flight.
// ADD: a launch of few workgroups, the only one; the last of them adds the parts to the norms (a launch behind it would cost as much again).
template <bool BF16, bool STREAM, bool ADD, int N>
__global__ __launch_bounds__(256) void held_sqnorms_kernel(HeldTable<N> t, int B, uint32_t per, uint32_t J, float* __restrict__ part, float* __restrict__ sqnorms,
                                                           uint32_t* __restrict__ ticket) {
    typedef Held<BF16, STREAM> IO;
    __shared__ float red[4];
    __shared__ bool last;
    const int l = held_tensor(t, blockIdx.x);
    const uint32_t count = t.count[l];
    const HeldPiece p = held_piece(count, blockIdx.x - t.first[l], B, per);
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + (uint64_t)p.unit * count + p.from;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const uint32_t len = p.to > p.from ? p.to - p.from : 0, whole = len / 8 * 8, step = p.lanes * 8;
    uint32_t k = p.lane * 8;
    for (; k + 3 * step < whole; k += 4 * step) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) IO::load8(x + k + u * step, v[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e & 3] += v[u][e] * v[u][e];
    }
    for (; k < whole; k += step) {
        float v[8];
        IO::load8(x + k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e & 3] += v[e] * v[e];
    }
    if (whole + p.lane < len) {
        const float v = IO::load1(x + whole + p.lane);
        s[0] += v * v;
    }
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
    float* out = part + (size_t)p.unit * J + (uintptr_t)t.y[l] + p.piece;
    if (p.lanes == 64) {
        sum = dp_wave_sum(sum);
        if (p.lane == 0 && p.unit < B) *out = sum;
    } else {
        sum = dp_block_sum<256>(sum, red);
        if (threadIdx.x == 0) *out = sum;
    }
    if constexpr (ADD) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");  // every thread's own part
        __syncthreads();
        if (threadIdx.x == 0) last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        for (int i = threadIdx.x >> 6; i < B; i += 4) {
            float s = 0.f;
            for (uint32_t j = threadIdx.x & 63; j < J; j += 64) s += __hip_atomic_load(part + (size_t)i * J + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s = dp_wave_sum(s);
            if ((threadIdx.x & 63) == 0) sqnorms[i] += s;
        }
        if (threadIdx.x == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// sqnorms[i] += the J partial sums of unit i, one workgroup a unit.
__global__ __launch_bounds__(1024) void held_finish_kernel(const float* __restrict__ part, uint32_t J, float* __restrict__ sqnorms) {
    __shared__ float red[16];
    const float* p = part + (size_t)blockIdx.x * J;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t k = threadIdx.x;
    for (; (uint64_t)k + 3 * 1024 < J; k += 4 * 1024) {
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += p[k + u * 1024];
    }
    for (; k < J; k += 1024) s[0] += p[k];
    const float sum = dp_block_sum<1024>((s[0] + s[1]) + (s[2] + s[3]), red);
    if (threadIdx.x == 0) sqnorms[blockIdx.x] += sum;
}

// The clip factor of unit i; `tell`: a norm that has none is reported (by one workgroup of a launch: all units', or its own unit's).
__device__ __forceinline__ float held_factor(const float* sqnorms, int i, float C, int* err, bool tell) {
    const float c = dp_clip_factor(sqnorms[i], C);
    if (tell && c != c) atomicOr(err, DP_ERRBIT_NORM);
    return c;
}

// sums[k] += c x[k], one unit.  Four elements a thread, the sums' access the wide one, neighbouring workgroups on neighbouring
// memory: 334 M bf16 elements 558 us (6.0 TB/s); eight neighbouring elements a thread 608; two and four groups of four, 1,024 apart, 535 and 546.
template <bool BF16, int N>
__global__ __launch_bounds__(256) void held_add_kernel(HeldTable<N> t, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    const int l = held_tensor(t, blockIdx.x);
    const uint32_t count = t.count[l], k = (blockIdx.x - t.first[l]) * ADD_COLS + threadIdx.x * 4;
    if (k >= count) return;
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + k;
    float* y = (float*)t.y[l] + k;
    const bool tell = blockIdx.x == 0 && threadIdx.x == 0;
    if (count - k >= 4) {
        float v[4], s[4];
        IO::load4(x, v);
        Held<false>::load4(y, s);
        const float c = held_factor(sqnorms, 0, C, err, tell);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += c * v[e];
        Held<false>::store4(y, s);
    } else {
        const float c = held_factor(sqnorms, 0, C, err, tell);
        for (uint32_t e = 0; e < count - k; ++e) y[e] += c * IO::load1(x + e);
    }
}

// sums[k] += sum_i c_i x[i][k]: RG waves share the units of 512 columns, eight a lane, and are added in a fixed order.
template <bool BF16, int RG, int N>
__global__ __launch_bounds__(64 * RG) void held_sums_kernel(HeldTable<N> t, int B, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    __shared__ float fac[FACTORS];
    __shared__ float red[RG][SUM_COLS];
    const int l = held_tensor(t, blockIdx.x), lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t count = t.count[l], k0 = (blockIdx.x - t.first[l]) * SUM_COLS, k = k0 + 8 * lane;
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + k;
    const int have = k >= count ? 0 : count - k < 8 ? (int)(count - k) : 8;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int b0 = 0; b0 < B; b0 += FACTORS) {
        const int nb = B - b0 < FACTORS ? B - b0 : FACTORS;
        __syncthreads();
        for (int i = threadIdx.x; i < nb; i += 64 * RG) fac[i] = held_factor(sqnorms, b0 + i, C, err, blockIdx.x == 0);
        __syncthreads();
        if (have == 8) {
            int i = w;
            for (; i + 3 * RG < nb; i += 4 * RG) {
                float v[4][8];
#pragma unroll
                for (int u = 0; u < 4; ++u) IO::load8(x + (uint64_t)(b0 + i + u * RG) * count, v[u]);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float c = fac[i + u * RG];
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += c * v[u][e];
                }
            }
            for (; i < nb; i += RG) {
                float v[8];
                IO::load8(x + (uint64_t)(b0 + i) * count, v);
                const float c = fac[i];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += c * v[e];
            }
        } else if (have) {
            for (int i = w; i < nb; i += RG) {
                const float c = fac[i];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < have) s[e] += c * IO::load1(x + (uint64_t)(b0 + i) * count + e);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[w][8 * lane + e] = s[e];
    __syncthreads();
    float* y = (float*)t.y[l] + k0;
    for (uint32_t j = threadIdx.x; j < SUM_COLS && j < count - k0; j += 64 * RG) {
        float a = red[0][j];
#pragma unroll
        for (int g = 1; g < RG; ++g) a += red[g][j];
        y[j] += a;
    }
}

// y[i][k] = c_i x[i][k], rounded once; nothing to do in place where c_i is one.
template <bool BF16, int N>
__global__ __launch_bounds__(256) void held_scale_kernel(HeldTable<N> t, int B, uint32_t per, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    const int l = held_tensor(t, blockIdx.x);
    const uint32_t count = t.count[l];
    const HeldPiece p = held_piece(count, blockIdx.x - t.first[l], B, per);
    if (p.from >= p.to) return;
    const float c = held_factor(sqnorms, p.unit, C, err, p.piece == 0 && p.lane == 0);
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + (uint64_t)p.unit * count;
    typename IO::elem* y = (typename IO::elem*)t.y[l] + (uint64_t)p.unit * count;
    if (c == 1.f && x == y) return;
    for (uint32_t k = p.from + p.lane * 4; k < p.to; k += p.lanes * 4) {
        if (p.to - k >= 4) {
            float v[4];
            IO::load4(x + k, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= c;
            IO::store4(y + k, v);
        } else {
            for (uint32_t e = k; e < p.to; ++e) IO::store1(y + e, c * IO::load1(x + e));
        }
    }
}

bool held_overlap(uintptr_t a, uint64_t na, uintptr_t b, uint64_t nb) { return a < b + nb * sizeof(float) && b < a + na * sizeof(float); }

// The tensors that have elements, one after the other (those of one unit in entries of at most 2^31), into launches of as many as a
// table holds and a grid can number, sums that share a buffer in launches of their own.
// blocks(count): workgroups of an entry; columns(count): its partial norms (0: none are wanted); go(table, grid).
template <typename Blocks, typename Columns, typename Go>
dp_status held_launches(dp_ctx* ctx, int n, const void* const* X, void* const* Y, const uint64_t* count, int B, int xsize, int ysize, bool sums, Blocks blocks, Columns columns,
                        Go go) {
    HeldFull t;
    t.n = 0;
    uint64_t grid = 0, col = 0;
    uintptr_t lo = UINTPTR_MAX, hi = 0;  // hull of the sums of a launch: in a flat buffer's order every tensor lies outside it
    auto flush = [&]() -> dp_status {
        const dp_status st = t.n ? go(t, (unsigned)grid) : DP_OK;
        t.n = 0;
        grid = 0;
        lo = UINTPTR_MAX;
        hi = 0;
        return st;
    };
    for (int l = 0; l < n; ++l) {
        for (uint64_t done = 0; done < count[l];) {
            const uint64_t c = B > 1 || count[l] - done <= HELD_ENTRY ? count[l] - done : HELD_ENTRY;
            const uintptr_t x = (uintptr_t)X[l] + done * xsize, y = Y ? (uintptr_t)Y[l] + done * ysize : 0;
            const uint64_t nb = blocks(c);
            if (nb > 0x7FFFFFFFull) {
                DP_SET_ERR(ctx, "tensor %d: too many elements for one launch", l);
                return DP_ERR_SHAPE;
            }
            bool apart = t.n == HELD_TABLE || grid + nb > 0x7FFFFFFFull;
            if (sums && !apart && y < hi && y + c * ysize > lo)
                for (int k = 0; k < t.n && !apart; ++k) apart = held_overlap((uintptr_t)t.y[k], t.count[k], y, c);
            if (apart) {
                const dp_status st = flush();
                if (st != DP_OK) return st;
            }
            t.x[t.n] = (const void*)x;
            t.y[t.n] = (void*)(Y ? y : (uintptr_t)col);
            t.count[t.n] = (uint32_t)c;
            t.first[t.n] = (uint32_t)grid;
            t.n++;
            grid += nb;
            col += columns(c);
            lo = y < lo ? y : lo;
            hi = y + c * ysize > hi ? y + c * ysize : hi;
            done += c;
        }
    }
    return flush();
}

// workgroups of an entry, and partial norms of a tensor in entries
uint64_t held_blocks(uint64_t c, uint32_t per, int B) {
    const uint32_t p = held_pieces(c, per);
    return p ? (uint64_t)p * B : ((uint64_t)B + 3) / 4;
}
uint64_t held_columns(uint64_t c, uint32_t per, int B) {
    uint64_t j = 0;
    for (; B == 1 && c > HELD_ENTRY; c -= HELD_ENTRY) j += held_pieces(HELD_ENTRY, per);
    return c ? j + (held_pieces(c, per) ? held_pieces(c, per) : 1) : j;
}

}  // namespace

dp_status dpk_held_sqnorms(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float* sqnorms) {
    const uint64_t room = ctx->ws_bytes / sizeof(float) / B;
    const int size = dt == DP_BF16 ? 2 : 4;
    uint64_t total = 0;
    for (int l = 0; l < n; ++l) total += count[l];
    const bool stream = total * B * size > LAST_LEVEL;
    if (room == 0) {
        DP_SET_ERR(ctx, "the workspace does not hold a partial norm of %d units", B);
        return DP_ERR_WORKSPACE;
    }
    // Tensors in groups whose partial norms fit the workspace: as a rule one, and one sum at the end.  A tensor that alone has too many
    // is cut into longer pieces.
    float* part = (float*)ctx->ws;
    for (int l0 = 0; l0 < n;) {
        uint32_t per = HELD_PIECE;
        uint64_t J = 0;
        int m = 0;
        for (; l0 + m < n; ++m) {
            const uint64_t j = held_columns(count[l0 + m], per, B);
            if (J + j > room) break;
            J += j;
        }
        if (m == 0) {
            const uint64_t c = count[l0], entry = B == 1 && c > HELD_ENTRY ? HELD_ENTRY : c, pieces = room / ((c + entry - 1) / entry);
            if (pieces == 0) {
                DP_SET_ERR(ctx, "the workspace holds %llu partial norms of a unit, tensor %d needs more", (unsigned long long)room, l0);
                return DP_ERR_WORKSPACE;
            }
            per = (uint32_t)(((entry + pieces - 1) / pieces + 7) / 8 * 8);
            J = held_columns(c, per, B);
            m = 1;
        }
        const uint32_t width = (uint32_t)J;
        auto blocks = [&](uint64_t c) { return held_blocks(c, per, B); };
        auto columns = [&](uint64_t c) { return held_columns(c, per, B); };
        bool added = false;
        const dp_status st = held_launches(ctx, m, X + l0, nullptr, count + l0, B, size, 4, false, blocks, columns, [&](const HeldFull& full, unsigned grid) {
            uint64_t cols = 0;
            for (int l = 0; l < full.n; ++l) cols += held_columns(full.count[l], per, B);
            added = cols == width && grid <= ADD_GRID && B <= ADD_UNITS;
            with_table(full, [&](const auto& t) {
                constexpr int N = sizeof(t.count) / sizeof(t.count[0]);
                auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, ctx->stream, t, B, per, width, part, sqnorms, ctx->ticket); };
                if (dt == DP_BF16 && added) launch(held_sqnorms_kernel<true, false, true, N>);
                else if (added) launch(held_sqnorms_kernel<false, false, true, N>);
                else if (dt == DP_BF16 && stream) launch(held_sqnorms_kernel<true, true, false, N>);
                else if (dt == DP_BF16) launch(held_sqnorms_kernel<true, false, false, N>);
                else if (stream) launch(held_sqnorms_kernel<false, true, false, N>);
                else launch(held_sqnorms_kernel<false, false, false, N>);
            });
            DP_LAUNCH_CHECK(ctx, "held_sqnorms");
            return DP_OK;
        });
        if (st != DP_OK) return st;
        if (width > 512 && !added) {
            hipLaunchKernelGGL(held_finish_kernel, dim3(B), dim3(1024), 0, ctx->stream, part, width, sqnorms);
            DP_LAUNCH_CHECK(ctx, "held_finish");
        } else if (width > 0 && !added) {
            const dp_status fin = dpk_finish_partials(ctx, part, B, (int)width, sqnorms);
            if (fin != DP_OK) return fin;
        }
        l0 += m;
    }
    return DP_OK;
}

dp_status dpk_held_sums(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float C, const float* sqnorms,
                        float* const* sums) {
    const uint64_t cols = B == 1 ? ADD_COLS : SUM_COLS;
    uint64_t tiles = 0;
    for (int l = 0; l < n; ++l) tiles += (count[l] + cols - 1) / cols;
    // 16 waves share the units where there is no tile for every CU: 192 tiles of 512 units 27.7 -> 19.4 us, 8 tiles 12.6 -> 9.1; 384 tiles of 256
    // units would take 21.8 instead of 18.8.
    const bool tall = tiles < 256 && B >= 64;
    auto blocks = [&](uint64_t c) { return (c + cols - 1) / cols; };
    return held_launches(ctx, n, X, (void* const*)sums, count, B, dt == DP_BF16 ? 2 : 4, 4, true, blocks, [](uint64_t) { return (uint64_t)0; }, [&](const HeldFull& full, unsigned grid) {
        with_table(full, [&](const auto& t) {
            constexpr int N = sizeof(t.count) / sizeof(t.count[0]);
            auto launch = [&](auto kernel, int threads, auto... args) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, ctx->stream, t, args..., C, sqnorms, ctx->err_word); };
            if (B == 1 && dt == DP_BF16) launch(held_add_kernel<true, N>, 256);
            else if (B == 1) launch(held_add_kernel<false, N>, 256);
            else if (dt == DP_BF16 && tall) launch(held_sums_kernel<true, 16, N>, 1024, B);
            else if (dt == DP_BF16) launch(held_sums_kernel<true, 4, N>, 256, B);
            else if (tall) launch(held_sums_kernel<false, 16, N>, 1024, B);
            else launch(held_sums_kernel<false, 4, N>, 256, B);
        });
        DP_LAUNCH_CHECK(ctx, "held_sums");
        return DP_OK;
    });
}

dp_status dpk_held_scale(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float C, const float* sqnorms, void* const* Y) {
    const uint32_t per = ADD_COLS;
    const int size = dt == DP_BF16 ? 2 : 4;
    auto blocks = [&](uint64_t c) { return held_blocks(c, per, B); };
    return held_launches(ctx, n, X, Y, count, B, size, size, false, blocks, [](uint64_t) { return (uint64_t)0; }, [&](const HeldFull& full, unsigned grid) {
        with_table(full, [&](const auto& t) {
            constexpr int N = sizeof(t.count) / sizeof(t.count[0]);
            auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, ctx->stream, t, B, per, C, sqnorms, ctx->err_word); };
            if (dt == DP_BF16) launch(held_scale_kernel<true, N>);
            else launch(held_scale_kernel<false, N>);
        });
        DP_LAUNCH_CHECK(ctx, "held_scale");
        return DP_OK;
    });
}
