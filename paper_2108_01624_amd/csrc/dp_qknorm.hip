// Root-mean-square norm of every head of queries and keys with a gain, the rotation by position in the same pass, and its backward with every
// example's gradients of the two gains.
//
//   r = 1 / sqrt(mean_j x_j^2 + eps)     y = Rot_p (g * x r)
//   u = Rot_p^T dy     dg += u * x r     dx = r (g * u - x r * mean_j (g_j u_j x_j r))
//
// Roofline: HBM.  The forward reads x and writes y, the backward reads x and dy and writes dx; a cosine and a sine per pair of numbers come
// out of the caches, whose rows all heads of a token share.  32 x 512 tokens of 16 + 16 heads of 64 bf16 numbers: forward 22 us (6.1 TB/s),
// 512 x 128 tokens backward 157 us (5.1 TB/s).  A wave's instruction takes four cycles here, so that a budget of 25 instructions a number is all
// that the forward has at that rate: addresses are scalars, sums over lanes are operands of the additions, the layouts are template arguments.
// (The same with addresses and choices per lane, and sums by exchanges through LDS: 39 and 200 us.)
//
// A head is shared by the fewest lanes, a power of two from four on, that hold eight of its numbers each.  Numbers that are rotated together lie
// in one lane, so that a rotation needs no exchange: with halves rotated against each other lane c holds [4 c, 4 c + 4) of both halves,
// otherwise, and behind the rotated part, [8 c, 8 c + 8).  Either way its pairs have the angles 4 c .. 4 c + 3.
#include "dp_common.h"

namespace {

constexpr int U = 2;                // rounds of a wave at a time (1, 2, 4: 512 x 128 tokens backward 174, 172, 221 us)
constexpr int GRADS_BLOCKS = 8192;  // workgroups of the backward that are aimed at: what is in flight lies close together (1,024: 175 us, 4,096: 170, 8,192: 161)

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));

// Queries or keys: their tensors and what is theirs of a launch.
struct Side {
    const void *x, *dy;     // [B][T][H][D], tokens ld numbers apart; dy dense
    void* y;                // forward: dense; backward: laid out as x, or NULL
    const float* gain;      // [D]
    float* part;            // backward: [B][chunks][D], examples `apart` numbers apart
    long ld, apart;
    int H, rpt, tpw;        // heads; rounds of a token, tokens of a round
    int chunks, per;        // backward: workgroups of an example, tokens of each
    unsigned blocks;        // workgroups
};
struct QkArgs {
    Side s[2];
    const float *cos, *sin; // [n_pos][R / 2]
    const int32_t* pos;     // [B][T], or NULL: a token's place in its example
    int* err;
    long tokens;            // B * T
    int n_pos, T, D, R;
    float eps;
};

template <bool BF16>
struct Num {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    typedef typename std::conditional<BF16, u32x2_t, f32x4_t>::type four;  // four numbers as they are stored
    static __device__ __forceinline__ four raw4(const elem* p) {
        if constexpr (BF16) return *reinterpret_cast<const u32x2_a2*>(p);
        else return *reinterpret_cast<const f32x4_a4*>(p);
    }
    static __device__ __forceinline__ void wide4(four w, float v[4]) {
        if constexpr (BF16) {
            v[0] = dp_bf16_lo(w[0]);
            v[1] = dp_bf16_hi(w[0]);
            v[2] = dp_bf16_lo(w[1]);
            v[3] = dp_bf16_hi(w[1]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = w[k];
        }
    }
    // Results are not read again here: streamed (forward 25 us, cached 31); loads are not, what made the numbers may have left them in a cache.
    static __device__ __forceinline__ void store4(elem* p, const float v[4]) {
        if constexpr (BF16) {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            const bf16x4_t w = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            __builtin_nontemporal_store(__builtin_bit_cast(u32x2_t, w), reinterpret_cast<u32x2_a2*>(p));
        } else {
            __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_a4*>(p));
        }
    }
};

// What of a head lane c holds: numbers a .. a + 3 and b .. b + 3.  ALL: heads fill their lanes and are rotated as a whole.
struct Part {
    int a, b, angle;   // angle: the first of its pairs'
    bool on, turned;   // a lane that holds nothing reads what lane 0 reads
};
template <bool INTER, bool ALL>
__device__ __forceinline__ Part part_of(const QkArgs& A, int c) {
    Part p;
    p.on = ALL || 8 * c < A.D;
    p.turned = ALL || 8 * c < A.R;
    if (!p.on) c = 0;
    const bool halves = !INTER && (ALL || 8 * c < A.R);
    p.a = halves ? 4 * c : 8 * c;
    p.b = halves ? A.R / 2 + 4 * c : 8 * c + 4;
    p.angle = ALL || 8 * c < A.R ? 4 * c : 0;
    return p;
}

// v[0..3] and v[4..7] are the two parts; (x, y) -> (x cos - y sin, y cos + x sin), the other way round with -sin.
template <bool INTER>
__device__ __forceinline__ void turn(float v[8], f32x4_t c, f32x4_t s) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = INTER ? 2 * k : k, j = INTER ? 2 * k + 1 : 4 + k;
        const float x = v[i], y = v[j];
        v[i] = x * c[k] - y * s[k];
        v[j] = y * c[k] + x * s[k];
    }
}

__device__ __forceinline__ void load4(const float* p, float v[4]) {
    const f32x4_t w = *reinterpret_cast<const f32x4_a4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = w[k];
}

// A wave works on N = 64 / LPH heads at a time, a round: of one token, whose H heads take `rpt` rounds, or of `tpw` whole tokens.
void set_rounds(Side& S, int lph) {
    const int N = 64 / lph, H = S.H ? S.H : 1;
    S.rpt = H < N ? 1 : (H + N - 1) / N;
    S.tpw = H < N ? N / H : 1;
}
// A lane's token and head within a round.
template <int LPH>
struct Place {
    static constexpr int N = 64 / LPH;
    int token, head;
    bool on;
    __device__ __forceinline__ Place(const Side& S, int lane) {
        const int s = lane / LPH;
        token = 0;
        head = s;
        if (S.tpw > 1 && S.H) {
            token = s / S.H;
            head = s - token * S.H;
        }
        on = token < S.tpw && head < S.H;
    }
};

// Where a round lies.  Its first head is the same for all lanes, and a lane's place behind it the same in every round: an address is a scalar
// and a register.  Lanes without a head (at the end of a token's heads or of the tokens) read what the round's first one reads.
struct Spot {
    long at, out;  // the round's first head in x (and its gradient), and in dense tensors
    int p;         // position of this lane's token
    bool there;

    // Heads hr N .. of the tokens group tpw .. of the n that begin at token0.
    // GIVEN: positions are.  EXAMPLE: all tokens are of one example, the first of them its token `place`.
    template <bool GIVEN, bool EXAMPLE, int LPH>
    __device__ __forceinline__ void find(const QkArgs& A, const Side& S, const Place<LPH>& L, long token0, int place, int n, int group, int hr, bool within) {
        constexpr int N = Place<LPH>::N;
        there = within && L.on && group * S.tpw + L.token < n && hr * N + L.head < S.H;
        const long token = token0 + (long)group * S.tpw;
        at = token * S.ld + (long)hr * N * A.D;
        out = (token * S.H + (long)hr * N) * A.D;
        const int mine = there ? L.token : 0;
        if constexpr (GIVEN) p = A.pos[token + mine];
        else if constexpr (EXAMPLE) p = place + group * S.tpw + mine;
        else p = (int)((uint32_t)(token + mine) % (uint32_t)A.T);
    }
};

// A round, loaded.
template <bool BF16, bool ALL, bool BACK>
struct Round {
    typedef Num<BF16> IO;
    typedef typename IO::elem elem;
    typename IO::four x[2], dy[BACK ? 2 : 1];
    f32x4_t cs, sn;
    bool good;

    __device__ __forceinline__ void numbers(const Side& S, const Part& P, const Spot& at, long x_off, long y_off) {
        const elem* px = (const elem*)S.x + at.at + (at.there ? x_off : 0);
        x[0] = IO::raw4(px + P.a);
        x[1] = IO::raw4(px + P.b);
        if constexpr (BACK) {
            const elem* pd = (const elem*)S.dy + at.out + (at.there ? y_off : 0);
            dy[0] = IO::raw4(pd + P.a);
            dy[1] = IO::raw4(pd + P.b);
        }
    }
    __device__ __forceinline__ void angles(const QkArgs& A, const Part& P, const Spot& at) {
        good = true;
        if (ALL || A.R) {
            good = (unsigned)at.p < (unsigned)A.n_pos;
            const long row = (long)(good ? at.p : 0) * (A.R / 2) + P.angle;
            cs = *reinterpret_cast<const f32x4_a4*>(A.cos + row);
            sn = *reinterpret_cast<const f32x4_a4*>(A.sin + row);
        }
    }
};

// A wave does U rounds one behind the other, all their loads first: positions, which the angles wait for, then numbers, then angles.
template <bool BF16, int LPH, bool INTER, bool ALL, bool GIVEN>
__global__ __launch_bounds__(256) void qk_norm_kernel(QkArgs A) {
    typedef Num<BF16> IO;
    typedef typename IO::elem elem;
    const bool second = blockIdx.x >= A.s[0].blocks;
    const Side S = second ? A.s[1] : A.s[0];
    const int lane = threadIdx.x & 63, c = lane % LPH;
    const Place<LPH> L(S, lane);
    const uint32_t item = __builtin_amdgcn_readfirstlane(((blockIdx.x - (second ? A.s[0].blocks : 0)) * 4 + (threadIdx.x >> 6)) * U);
    int group = (int)(item / (uint32_t)S.rpt), hr = (int)(item - (uint32_t)group * S.rpt);
    const int tokens = (int)A.tokens;
    if ((long)group * S.tpw >= tokens) return;
    const Part P = part_of<INTER, ALL>(A, c);
    const long x_off = L.token * S.ld + (long)L.head * A.D, y_off = (long)(L.token * S.H + L.head) * A.D;
    Spot at[U];
    Round<BF16, ALL, false> in[U];
    bool within = true;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u].template find<GIVEN, false>(A, S, L, 0, 0, tokens, group, hr, within);
        if (hr + 1 < S.rpt) ++hr;
        else if ((long)(group + 1) * S.tpw < tokens) {
            hr = 0;
            ++group;
        } else within = false;  // (the last round once more, for nobody)
    }
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].numbers(S, P, at[u], x_off, 0);
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].angles(A, P, at[u]);
    float g[8];
    load4(S.gain + P.a, g);
    load4(S.gain + P.b, g + 4);
    const float inv = 1.f / (float)A.D;
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float v[8];
        IO::wide4(in[u].x[0], v);
        IO::wide4(in[u].x[1], v + 4);
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e] * v[e];
        if (!ALL && !P.on) s = 0.f;
        const float r = __builtin_amdgcn_rsqf(dp_lanes_sum<LPH>(s) * inv + A.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= r * g[e];
        if (P.turned) turn<INTER>(v, in[u].cs, in[u].sn);
        if (!in[u].good) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
            bad = bad || at[u].there;
        }
        if (at[u].there && P.on) {
            elem* y = (elem*)S.y + at[u].out + y_off;
            IO::store4(y + P.a, v);
            IO::store4(y + P.b, v + 4);
        }
    }
    if (bad) atomicOr(A.err, DP_ERRBIT_INDEX);
}

// part[example][chunk][D] = gradient of a gain over a chunk's tokens; y, if there is one, the gradient of x.
template <bool BF16, int LPH, bool INTER, bool ALL, bool GIVEN>
__global__ __launch_bounds__(256) void qk_norm_grads_kernel(QkArgs A) {
    typedef Num<BF16> IO;
    typedef typename IO::elem elem;
    extern __shared__ float red[];  // [4 waves][D]
    const bool second = blockIdx.x >= A.s[0].blocks;
    const Side S = second ? A.s[1] : A.s[0];
    const unsigned block = blockIdx.x - (second ? A.s[0].blocks : 0);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % LPH;
    const Place<LPH> L(S, lane);
    const int ex = block / (unsigned)S.chunks, ch = block - ex * S.chunks;
    const int t0 = ch * S.per, n = !S.H ? 0 : A.T - t0 < S.per ? A.T - t0 : S.per;  // tokens t0 .. t0 + n - 1
    const Part P = part_of<INTER, ALL>(A, c);
    const long x_off = L.token * S.ld + (long)L.head * A.D, y_off = (long)(L.token * S.H + L.head) * A.D;
    const float inv = 1.f / (float)A.D;
    float acc[8] = {}, g[8] = {};
    if (S.H) {
        load4(S.gain + P.a, g);
        load4(S.gain + P.b, g + 4);
    }
    const int rounds = (n + S.tpw - 1) / S.tpw * S.rpt;
    bool bad = false;
    Spot next[U];
    auto find = [&](int first) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int rd = first + u < rounds ? first + u : rounds - 1, group = (unsigned)rd / (unsigned)S.rpt, hr = rd - group * S.rpt;
            next[u].template find<GIVEN, true>(A, S, L, (long)ex * A.T + t0, t0, n, group, hr, first + u < rounds);
        }
    };
    if (rounds > 0) find(w * U);  // positions are asked for a step ahead: the angles need them
    for (int first = w * U; first < rounds; first += 4 * U) {
        Spot at[U];
        Round<BF16, ALL, true> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = next[u];
            in[u].numbers(S, P, at[u], x_off, y_off);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) in[u].angles(A, P, at[u]);
        find(first + 4 * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8], d[8], gd[8];
            IO::wide4(in[u].x[0], v);
            IO::wide4(in[u].x[1], v + 4);
            IO::wide4(in[u].dy[0], d);
            IO::wide4(in[u].dy[1], d + 4);
            if (P.turned) turn<INTER>(d, in[u].cs, -in[u].sn);
            float s = 0.f, m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s += v[e] * v[e];
                gd[e] = g[e] * d[e];
                m += gd[e] * v[e];
            }
            if (!ALL && !P.on) s = m = 0.f;
            const float r = __builtin_amdgcn_rsqf(dp_lanes_sum<LPH>(s) * inv + A.eps);
            m = dp_lanes_sum<LPH>(m) * inv * r;
            if (!at[u].there) continue;
            if (in[u].good) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float xh = v[e] * r;
                    acc[e] += d[e] * xh;
                    d[e] = r * (gd[e] - xh * m);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = 0.f;
                bad = true;
            }
            if (P.on && S.y) {
                elem* o = (elem*)S.y + at[u].at + x_off;
                IO::store4(o + P.a, d);
                IO::store4(o + P.b, d + 4);
            }
        }
    }
    if (bad) atomicOr(A.err, DP_ERRBIT_INDEX);
    // over the heads of a wave, then over the waves
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int o = LPH; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o, 64);
    if (lane < LPH && P.on) {
#pragma unroll
        for (int e = 0; e < 8; ++e) red[w * A.D + (e < 4 ? P.a + e : P.b + e - 4)] = acc[e];
    }
    __syncthreads();
    float* out = S.part + (long)ex * S.apart + (long)ch * A.D;
    for (int j = threadIdx.x; j < A.D; j += 256) out[j] = (red[j] + red[A.D + j]) + (red[2 * A.D + j] + red[3 * A.D + j]);
}

// grads[example][side][D] = sum over the side's chunks: a workgroup an example and side, its threads the columns in as many groups of
// chunks as there are threads for.
__global__ __launch_bounds__(512) void qk_join_kernel(QkArgs A, float* __restrict__ grads) {
    __shared__ float red[512];
    const Side S = A.s[blockIdx.x & 1];
    const int ex = blockIdx.x >> 1, groups = 512 / A.D, g = threadIdx.x / A.D, j = threadIdx.x - g * A.D;
    const float* p = S.part + (long)ex * S.apart + j;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (g < groups) {
        int k = g;
        for (; k + 3 * groups < S.chunks; k += 4 * groups)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += p[(long)(k + u * groups) * A.D];
        for (; k < S.chunks; k += groups) s[0] += p[(long)k * A.D];
    }
    red[threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if ((int)threadIdx.x < A.D) {
        float sum = red[threadIdx.x];
        for (int k = 1; k < groups; ++k) sum += red[k * A.D + threadIdx.x];
        grads[(long)blockIdx.x * A.D + threadIdx.x] = sum;
    }
}

int head_lanes(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64; }

template <typename F>
void by_lanes(int D, F f) {
    switch (head_lanes(D)) {
        case 4: return f(std::integral_constant<int, 4>());
        case 8: return f(std::integral_constant<int, 8>());
        case 16: return f(std::integral_constant<int, 16>());
        case 32: return f(std::integral_constant<int, 32>());
        default: return f(std::integral_constant<int, 64>());
    }
}

// f(BF16, INTER, ALL)
template <int LPH, typename F>
void by_layout(const dp_qk_args& a, F f) {
    auto all = [&](auto bf16, auto inter) {
        if (a.D == 8 * LPH && a.R == a.D) f(bf16, inter, std::true_type());
        else f(bf16, inter, std::false_type());
    };
    if (a.dtype == DP_BF16 && a.interleaved) all(std::true_type(), std::true_type());
    else if (a.dtype == DP_BF16) all(std::true_type(), std::false_type());
    else if (a.interleaved) all(std::false_type(), std::true_type());
    else all(std::false_type(), std::false_type());
}

QkArgs make_args(dp_ctx* ctx, const dp_qk_args& a) {
    QkArgs A{};
    A.s[0].x = a.q;
    A.s[1].x = a.k;
    A.s[0].gain = a.gain_q;
    A.s[1].gain = a.gain_k;
    A.s[0].ld = a.ldq;
    A.s[1].ld = a.ldk;
    A.s[0].H = a.Hq;
    A.s[1].H = a.Hk;
    A.cos = a.cos;
    A.sin = a.sin;
    A.pos = a.R ? a.positions : nullptr;
    A.err = ctx->err_word;
    A.tokens = (long)a.B * a.T;
    A.n_pos = a.n_pos;
    A.T = a.T;
    A.D = a.D;
    A.R = a.R;
    A.eps = a.eps;
    return A;
}

}  // namespace

dp_status dpk_qk_norm(dp_ctx* ctx, const dp_qk_args& a, void* yq, void* yk) {
    QkArgs A = make_args(ctx, a);
    A.s[0].y = yq;
    A.s[1].y = yk;
    dp_status st = DP_OK;
    by_lanes(a.D, [&](auto lph) {
        constexpr int L = decltype(lph)::value;
        uint64_t rounds[2];
        for (int s = 0; s < 2; ++s) {
            Side& S = A.s[s];
            set_rounds(S, L);
            rounds[s] = S.H ? ((uint64_t)A.tokens + S.tpw - 1) / S.tpw * S.rpt : 0;
        }
        uint64_t grid = 0;
        for (int s = 0; s < 2; ++s) {
            const uint64_t blocks = (rounds[s] + 4 * U - 1) / (4 * U);
            A.s[s].blocks = (unsigned)blocks;
            grid += blocks;
        }
        if (grid > 0x7FFFFFFFull || rounds[0] + 4 * U > 0xFFFFFFFFull || rounds[1] + 4 * U > 0xFFFFFFFFull) {
            DP_SET_ERR(ctx, "too many heads for one launch");
            st = DP_ERR_SHAPE;
            return;
        }
        by_layout<L>(a, [&](auto bf16, auto inter, auto all) {
            constexpr bool BF16 = decltype(bf16)::value, INTER = decltype(inter)::value, ALL = decltype(all)::value;
            if (A.pos) hipLaunchKernelGGL((qk_norm_kernel<BF16, L, INTER, ALL, true>), dim3((unsigned)grid), dim3(256), 0, ctx->stream, A);
            else hipLaunchKernelGGL((qk_norm_kernel<BF16, L, INTER, ALL, false>), dim3((unsigned)grid), dim3(256), 0, ctx->stream, A);
        });
    });
    if (st != DP_OK) return st;
    DP_LAUNCH_CHECK(ctx, "qk_norm");
    return DP_OK;
}

dp_status dpk_qk_norm_grads(dp_ctx* ctx, const dp_qk_args& a, const void* dyq, const void* dyk, float* grads, void* dq, void* dk, bool wanted) {
    QkArgs A = make_args(ctx, a);
    A.s[0].dy = dyq;
    A.s[1].dy = dyk;
    if (wanted) {
        A.s[0].y = dq;
        A.s[1].y = dk;
    }
    // Workgroups of an example: a side's share of GRADS_BLOCKS, each of at least two steps of its waves' rounds, as long as their parts fit the
    // workspace (otherwise one a side, straight into the gradients).  A side without heads has one, which writes zeros.
    const size_t room = ctx->ws_bytes / sizeof(float) / a.B / a.D;
    float* ws = (float*)ctx->ws;
    const long share = (GRADS_BLOCKS + a.B - 1) / a.B;
    size_t used = 0;
    for (int s = 0; s < 2; ++s) {
        Side& S = A.s[s];
        set_rounds(S, head_lanes(a.D));
        const long rounds = S.H ? (long)((a.T + S.tpw - 1) / S.tpw) * S.rpt : 1;
        long chunks = (share * S.H + a.Hq + a.Hk - 1) / (a.Hq + a.Hk);
        if (chunks > rounds / (8 * U)) chunks = rounds / (8 * U);
        S.chunks = chunks > 1 ? (int)chunks : 1;
        used += S.chunks;
    }
    const bool direct = (A.s[0].chunks == 1 && A.s[1].chunks == 1) || used > room;
    uint64_t grid = 0;
    for (Side& S : A.s) {
        if (direct) S.chunks = 1;
        S.per = (int)(((long)a.T + S.chunks - 1) / S.chunks);
        S.chunks = (int)(((long)a.T + S.per - 1) / S.per);
        S.blocks = (unsigned)S.chunks * (unsigned)a.B;
        grid += (uint64_t)S.chunks * a.B;
        if ((long)S.per * S.rpt > 0x7FFFFFFFl - 8 * U) {  // (a wave counts two steps ahead)
            DP_SET_ERR(ctx, "too many heads of one example");
            return DP_ERR_SHAPE;
        }
    }
    if (grid > 0x7FFFFFFFull) {
        DP_SET_ERR(ctx, "too many examples for one launch");
        return DP_ERR_SHAPE;
    }
    for (int s = 0; s < 2; ++s) {
        A.s[s].part = direct ? grads + (size_t)s * a.D : ws + (s ? (size_t)a.B * A.s[0].chunks * a.D : 0);
        A.s[s].apart = direct ? 2 * a.D : (long)A.s[s].chunks * a.D;
    }
    by_lanes(a.D, [&](auto lph) {
        constexpr int L = decltype(lph)::value;
        const size_t lds = 4 * (size_t)a.D * sizeof(float);
        by_layout<L>(a, [&](auto bf16, auto inter, auto all) {
            constexpr bool BF16 = decltype(bf16)::value, INTER = decltype(inter)::value, ALL = decltype(all)::value;
            if (A.pos) hipLaunchKernelGGL((qk_norm_grads_kernel<BF16, L, INTER, ALL, true>), dim3((unsigned)grid), dim3(256), lds, ctx->stream, A);
            else hipLaunchKernelGGL((qk_norm_grads_kernel<BF16, L, INTER, ALL, false>), dim3((unsigned)grid), dim3(256), lds, ctx->stream, A);
        });
    });
    DP_LAUNCH_CHECK(ctx, "qk_norm_grads");
    if (direct) return DP_OK;
    hipLaunchKernelGGL(qk_join_kernel, dim3(2 * (unsigned)a.B), dim3(512), 0, ctx->stream, A, grads);
    DP_LAUNCH_CHECK(ctx, "qk_join");
    return DP_OK;
}
