// Gradients that the caller holds, many tensors X_l [B, n_l]: the squared norm of every unit over all of them, the clip-weighted sums
// and the scaled gradients.
//
// Roofline: HBM.  The norm reads every element once (one multiply-add each); the sums read it again and read and write 4 bytes per
// entry of the sums; the scaled form reads and writes it.  Rows start wherever n_l puts them: 16-byte accesses are declared with the
// alignment of an element, which the hardware serves at any address.
#include "dp_common.h"

namespace {

constexpr int HELD_TABLE = 120;     // tensors per launch: their table is a kernel argument, of less than 4 KiB
constexpr int WAVE_ROW = 4096;      // rows up to this length are one wave's, longer ones one or several workgroups'
constexpr int SUM_COLS = 64 * 8;    // columns of a workgroup of the sums over several units
constexpr int FACTORS = 1024;       // clip factors in LDS at a time

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));
typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));

template <bool BF16>
struct Held {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    // eight elements from any address of an element
    static __device__ __forceinline__ void load8(const elem* p, float v[8]) {
        if constexpr (BF16) {
            const u32x4_t w = *reinterpret_cast<const u32x4_a2*>(p);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = dp_bf16_lo(w[k]);
                v[2 * k + 1] = dp_bf16_hi(w[k]);
            }
        } else {
            const f32x4_t a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = a[k];
                v[4 + k] = b[k];
            }
        }
    }
    static __device__ __forceinline__ float load1(const elem* p) {
        if constexpr (BF16) return dp_bf16_bits_to_f32(*p);
        else return *p;
    }
    static __device__ __forceinline__ void store8(elem* p, const float v[8]) {
        if constexpr (BF16) {
            typedef __bf16 bf16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));
            bf16x8_t w;
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = (__bf16)v[k];
            *reinterpret_cast<bf16x8_a2*>(p) = w;
        } else {
            *reinterpret_cast<f32x4_a4*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_a4*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
        }
    }
    static __device__ __forceinline__ void store1(elem* p, float v) {
        if constexpr (BF16) *reinterpret_cast<__bf16*>(p) = (__bf16)v;
        else *p = v;
    }
};

// The tensors of a launch.  Workgroups first[l] .. first[l + 1] - 1 are tensor l's.
struct HeldTable {
    const void* x[HELD_TABLE];
    void* y[HELD_TABLE];            // sums or scaled gradients (not used by the norms)
    uint64_t count[HELD_TABLE];     // elements of a unit
    int first[HELD_TABLE];
    int n;
};

// The tensor of workgroup b: two entries a lane and two ballots (a search by halves would be seven dependent loads).
__device__ __forceinline__ int held_tensor(const HeldTable& t, int b) {
    const int lane = threadIdx.x & 63;
    const bool lo = lane < t.n && t.first[lane] <= b, hi = lane + 64 < t.n && t.first[lane + 64] <= b;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lo)) + __popcll(__ballot(hi)) - 1);
}

// What of a tensor a workgroup (a wave, for short rows) does: elements [from, to) of unit `unit`, in whole groups of eight but for the last.
struct HeldPiece {
    int unit, piece;
    uint64_t from, to;
    int lane, lanes;
};
__device__ __forceinline__ HeldPiece held_piece(const HeldTable& t, int l, int b, int B, int pieces) {
    HeldPiece p;
    const uint64_t count = t.count[l];
    const int k = b - t.first[l];
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
        const uint64_t per = ((count + 7) / 8 + pieces - 1) / pieces * 8;
        p.from = per * p.piece < count ? per * p.piece : count;
        p.to = p.from + per < count ? p.from + per : count;
        p.lane = threadIdx.x;
        p.lanes = 256;
    }
    return p;
}
// pieces of a row for `per` elements each (0: a wave takes it whole)
__host__ __device__ __forceinline__ int held_pieces(uint64_t count, uint64_t per) { return count <= WAVE_ROW ? 0 : (int)((count + per - 1) / per); }

// part[unit * J + col[l] + piece] = sum of squares.  Four independent chains a thread.
struct HeldCols {
    int col[HELD_TABLE];
};
template <bool BF16>
__global__ __launch_bounds__(256) void held_sqnorms_kernel(HeldTable t, HeldCols cols, int B, uint64_t per, int J, float* __restrict__ part) {
    typedef Held<BF16> IO;
    __shared__ float red[4];
    const int l = held_tensor(t, blockIdx.x), pieces = held_pieces(t.count[l], per);
    const HeldPiece p = held_piece(t, l, blockIdx.x, B, pieces);
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + (p.to ? (uint64_t)p.unit * t.count[l] : 0);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const uint64_t whole = p.from + (p.to - p.from) / 8 * 8, step = (uint64_t)p.lanes * 8;
    uint64_t k = p.from + (uint64_t)p.lane * 8;
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
    if (whole + p.lane < p.to) {
        const float v = IO::load1(x + whole + p.lane);
        s[0] += v * v;
    }
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (pieces == 0) {
        sum = dp_wave_sum(sum);
        if (p.lane == 0 && p.unit < B) part[(size_t)p.unit * J + cols.col[l]] = sum;
    } else {
        sum = dp_block_sum<256>(sum, red);
        if (threadIdx.x == 0) part[(size_t)p.unit * J + cols.col[l] + p.piece] = sum;
    }
}

// sqnorms[i] += the J partial sums of unit i, one workgroup a unit.
__global__ __launch_bounds__(256) void held_finish_kernel(const float* __restrict__ part, int J, float* __restrict__ sqnorms) {
    __shared__ float red[4];
    const float* p = part + (size_t)blockIdx.x * J;
    float s = 0.f;
    for (int k = threadIdx.x; k < J; k += 256) s += p[k];
    s = dp_block_sum<256>(s, red);
    if (threadIdx.x == 0) sqnorms[blockIdx.x] += s;
}

// The clip factor of unit i; `tell`: a norm that has none is reported (by one workgroup of a launch: all units', or its own unit's).
__device__ __forceinline__ float held_factor(const float* sqnorms, int i, float C, int* err, bool tell) {
    const float c = dp_clip_factor(sqnorms[i], C);
    if (tell && c != c) atomicOr(err, DP_ERRBIT_NORM);
    return c;
}

// sums[k] += c x[k], one unit: a thread's eight elements.
template <bool BF16>
__global__ __launch_bounds__(256) void held_add_kernel(HeldTable t, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    const int l = held_tensor(t, blockIdx.x);
    const uint64_t count = t.count[l], k = ((uint64_t)(blockIdx.x - t.first[l]) * 256 + threadIdx.x) * 8;
    if (k >= count) return;
    const typename IO::elem* x = (const typename IO::elem*)t.x[l];
    float* y = (float*)t.y[l];
    const float c = held_factor(sqnorms, 0, C, err, blockIdx.x == 0 && threadIdx.x == 0);
    if (k + 8 <= count) {
        float v[8], s[8];
        IO::load8(x + k, v);
        Held<false>::load8(y + k, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += c * v[e];
        Held<false>::store8(y + k, s);
    } else {
        for (uint64_t e = k; e < count; ++e) y[e] += c * IO::load1(x + e);
    }
}

// sums[k] += sum_i c_i x[i][k]: RG waves share the units of 512 columns, eight a lane, and are added in a fixed order.
template <bool BF16, int RG>
__global__ __launch_bounds__(64 * RG) void held_sums_kernel(HeldTable t, int B, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    __shared__ float fac[FACTORS];
    __shared__ float red[RG][SUM_COLS];
    const int l = held_tensor(t, blockIdx.x), lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t count = t.count[l], k0 = (uint64_t)(blockIdx.x - t.first[l]) * SUM_COLS, k = k0 + 8 * lane;
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + k;
    const int have = k + 8 <= count ? 8 : k < count ? (int)(count - k) : 0;
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
    float* y = (float*)t.y[l];
    for (int j = threadIdx.x; j < SUM_COLS; j += 64 * RG) {
        if (k0 + j >= count) break;
        float a = red[0][j];
#pragma unroll
        for (int g = 1; g < RG; ++g) a += red[g][j];
        y[k0 + j] += a;
    }
}

// y[i][k] = c_i x[i][k], rounded once; nothing to do in place where c_i is one.
template <bool BF16>
__global__ __launch_bounds__(256) void held_scale_kernel(HeldTable t, int B, uint64_t per, float C, const float* __restrict__ sqnorms, int* __restrict__ err) {
    typedef Held<BF16> IO;
    const int l = held_tensor(t, blockIdx.x);
    const HeldPiece p = held_piece(t, l, blockIdx.x, B, held_pieces(t.count[l], per));
    if (p.from >= p.to) return;
    const float c = held_factor(sqnorms, p.unit, C, err, p.piece == 0 && p.lane == 0);
    const typename IO::elem* x = (const typename IO::elem*)t.x[l] + (uint64_t)p.unit * t.count[l];
    typename IO::elem* y = (typename IO::elem*)t.y[l] + (uint64_t)p.unit * t.count[l];
    if (c == 1.f && x == y) return;
    const uint64_t whole = p.from + (p.to - p.from) / 8 * 8, step = (uint64_t)p.lanes * 8;
    for (uint64_t k = p.from + (uint64_t)p.lane * 8; k < whole; k += step) {
        float v[8];
        IO::load8(x + k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= c;
        IO::store8(y + k, v);
    }
    if (whole + p.lane < p.to) IO::store1(y + whole + p.lane, c * IO::load1(x + whole + p.lane));
}

// Elements a workgroup of the norms and of the scaled gradients takes: 8,192, more where that would be many more workgroups than the chip
// holds at a time.
uint64_t held_per(int n, const uint64_t* count, int B) {
    uint64_t total = 0;
    for (int l = 0; l < n; ++l) total += count[l];
    const uint64_t even = total / 4096 * B;
    return even < 8192 ? 8192 : (even + 7) / 8 * 8;
}

bool held_overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    return na && nb && (uintptr_t)a < (uintptr_t)b + nb * sizeof(float) && (uintptr_t)b < (uintptr_t)a + na * sizeof(float);
}

// Launches over the tensors that have elements, as many at a time as a table holds, fit `room` columns of partial norms and a grid, and
// (sums) do not share a buffer.  blocks(l): workgroups of tensor l; columns(l): its partial norms; go(table, columns' places, grid, columns).
template <typename Blocks, typename Columns, typename Go>
dp_status held_launches(dp_ctx* ctx, int n, const void* const* X, void* const* Y, const uint64_t* count, bool sums, long room, Blocks blocks, Columns columns, Go go) {
    HeldTable t{};
    HeldCols cols{};
    long grid = 0, used = 0;
    auto flush = [&]() -> dp_status {
        if (!t.n) return DP_OK;
        const dp_status st = go(t, cols, (unsigned)grid, (int)used);
        t.n = 0;
        grid = used = 0;
        return st;
    };
    for (int l = 0; l < n; ++l) {
        if (!count[l]) continue;
        const long nb = blocks(count[l]), nc = columns(count[l]);
        if (nb > 0x7FFFFFFFl) {
            DP_SET_ERR(ctx, "tensor %d: too many elements for one launch", l);
            return DP_ERR_SHAPE;
        }
        if (nc > room) {
            DP_SET_ERR(ctx, "the workspace holds %ld partial norms of a unit, %ld are needed", room, nc);
            return DP_ERR_WORKSPACE;
        }
        bool shared = false;
        for (int k = 0; sums && k < t.n && !shared; ++k) shared = held_overlap(t.y[k], t.count[k], Y[l], count[l]);
        if (t.n == HELD_TABLE || grid + nb > 0x7FFFFFFFl || used + nc > room || shared) {
            const dp_status st = flush();
            if (st != DP_OK) return st;
        }
        t.x[t.n] = X[l];
        t.y[t.n] = Y ? Y[l] : nullptr;
        t.count[t.n] = count[l];
        t.first[t.n] = (int)grid;
        cols.col[t.n] = (int)used;
        t.n++;
        grid += nb;
        used += nc;
    }
    return flush();
}

}  // namespace

dp_status dpk_held_sqnorms(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float* sqnorms) {
    uint64_t per = held_per(n, count, B);
    const long room = (long)(ctx->ws_bytes / sizeof(float) / B);
    for (int l = 0; l < n; ++l)  // a small workspace: longer pieces
        if (room > 0 && (count[l] + per - 1) / per > (uint64_t)room) per = ((count[l] + room - 1) / room + 7) / 8 * 8;
    float* part = (float*)ctx->ws;
    auto blocks = [&](uint64_t c) { const int p = held_pieces(c, per); return p ? (long)p * B : ((long)B + 3) / 4; };
    auto columns = [&](uint64_t c) { const int p = held_pieces(c, per); return p ? (long)p : 1l; };
    return held_launches(ctx, n, X, nullptr, count, false, room, blocks, columns, [&](const HeldTable& t, const HeldCols& cols, unsigned grid, int J) {
        if (dt == DP_BF16) hipLaunchKernelGGL(held_sqnorms_kernel<true>, dim3(grid), dim3(256), 0, ctx->stream, t, cols, B, per, J, part);
        else hipLaunchKernelGGL(held_sqnorms_kernel<false>, dim3(grid), dim3(256), 0, ctx->stream, t, cols, B, per, J, part);
        DP_LAUNCH_CHECK(ctx, "held_sqnorms");
        if (J <= 512) return dpk_finish_partials(ctx, part, B, J, sqnorms);
        hipLaunchKernelGGL(held_finish_kernel, dim3(B), dim3(256), 0, ctx->stream, part, J, sqnorms);
        DP_LAUNCH_CHECK(ctx, "held_finish");
        return DP_OK;
    });
}

dp_status dpk_held_sums(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float C, const float* sqnorms,
                        float* const* sums) {
    const uint64_t cols = B == 1 ? 256 * 8 : SUM_COLS;
    uint64_t tiles = 0;
    for (int l = 0; l < n; ++l) tiles += (count[l] + cols - 1) / cols;
    const bool tall = tiles < 512 && B >= 64;
    auto blocks = [&](uint64_t c) { return (long)((c + cols - 1) / cols); };
    return held_launches(ctx, n, X, (void* const*)sums, count, true, 1l << 40, blocks, [](uint64_t) { return 0l; }, [&](const HeldTable& t, const HeldCols&, unsigned grid, int) {
        auto launch = [&](auto kernel, int threads, auto... args) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, ctx->stream, t, args..., C, sqnorms, ctx->err_word); };
        if (B == 1 && dt == DP_BF16) launch(held_add_kernel<true>, 256);
        else if (B == 1) launch(held_add_kernel<false>, 256);
        else if (dt == DP_BF16 && tall) launch(held_sums_kernel<true, 16>, 1024, B);
        else if (dt == DP_BF16) launch(held_sums_kernel<true, 4>, 256, B);
        else if (tall) launch(held_sums_kernel<false, 16>, 1024, B);
        else launch(held_sums_kernel<false, 4>, 256, B);
        DP_LAUNCH_CHECK(ctx, "held_sums");
        return DP_OK;
    });
}

dp_status dpk_held_scale(dp_ctx* ctx, int n, const void* const* X, const uint64_t* count, dp_dtype dt, int B, float C, const float* sqnorms, void* const* Y) {
    const uint64_t per = held_per(n, count, B);
    auto blocks = [&](uint64_t c) { const int p = held_pieces(c, per); return p ? (long)p * B : ((long)B + 3) / 4; };
    return held_launches(ctx, n, X, Y, count, false, 1l << 40, blocks, [](uint64_t) { return 0l; }, [&](const HeldTable& t, const HeldCols&, unsigned grid, int) {
        if (dt == DP_BF16) hipLaunchKernelGGL(held_scale_kernel<true>, dim3(grid), dim3(256), 0, ctx->stream, t, B, per, C, sqnorms, ctx->err_word);
        else hipLaunchKernelGGL(held_scale_kernel<false>, dim3(grid), dim3(256), 0, ctx->stream, t, B, per, C, sqnorms, ctx->err_word);
        DP_LAUNCH_CHECK(ctx, "held_scale");
        return DP_OK;
    });
}
