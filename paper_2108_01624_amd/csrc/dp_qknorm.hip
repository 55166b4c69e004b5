// Root-mean-square norm of every head of queries and keys with a gain, the rotation by position in the same pass, and its backward with every
// example's gradients of the two gains.
//
//   r = 1 / sqrt(mean_j x_j^2 + eps)     y = Rot_p (g * x r)
//   u = Rot_p^T dy     dg += u * x r     dx = r (g * u - x r * mean_j (g_j u_j x_j r))
//
// Roofline: HBM.  The forward reads x and writes y, the backward reads x and dy and writes dx; a cosine and a sine per pair of numbers are
// loaded once per token and used by all its heads.
//
// A head is shared by the fewest lanes, a power of two of them, that hold eight of its numbers each.  Numbers that are rotated together lie
// in one lane, so that a rotation needs no exchange: with halves rotated against each other lane c holds [4 c, 4 c + 4) of both halves,
// otherwise, and behind the rotated part, [8 c, 8 c + 8).  Either way its pairs have the angles 4 c .. 4 c + 3.
#include "dp_common.h"

namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t u32x2_a2 __attribute__((aligned(2)));
typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));

struct QkArgs {
    const void *q, *k;      // [B][T][heads][D], tokens ldq / ldk numbers apart
    const float *gq, *gk;   // [D]
    const float *cos, *sin; // [n_pos][R / 2]
    const int32_t* pos;     // [B][T], or NULL: a token's place in its example
    int* err;
    long ldq, ldk;
    int n_pos, inter, T, Hq, Hk, D, R;
    float eps;
    long tokens;            // B * T
};

template <bool BF16>
struct Num {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    static __device__ __forceinline__ void load4(const elem* p, float v[4]) {
        if constexpr (BF16) {
            const u32x2_t w = *reinterpret_cast<const u32x2_a2*>(p);
            v[0] = dp_bf16_lo(w[0]);
            v[1] = dp_bf16_hi(w[0]);
            v[2] = dp_bf16_lo(w[1]);
            v[3] = dp_bf16_hi(w[1]);
        } else {
            const f32x4_t w = *reinterpret_cast<const f32x4_a4*>(p);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = w[k];
        }
    }
    static __device__ __forceinline__ void store4(elem* p, const float v[4]) {
        if constexpr (BF16) {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            typedef bf16x4_t bf16x4_a2 __attribute__((aligned(2)));
            *reinterpret_cast<bf16x4_a2*>(p) = bf16x4_t{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        } else {
            *reinterpret_cast<f32x4_a4*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
        }
    }
};

// What of a head lane c holds: numbers a .. a + 3 and b .. b + 3.
struct Part {
    int a, b;
    bool on, turned;
};
__device__ __forceinline__ Part part_of(const QkArgs& A, int c) {
    Part p;
    p.on = 8 * c < A.D;
    p.turned = 8 * c < A.R;
    const bool halves = p.turned && !A.inter;
    p.a = halves ? 4 * c : 8 * c;
    p.b = halves ? A.R / 2 + 4 * c : 8 * c + 4;
    return p;
}

// v[0..3] and v[4..7] are the two parts; (x, y) -> (x cos - y sin, y cos + x sin), the other way round with -sin.
__device__ __forceinline__ void turn(float v[8], const float c[4], const float s[4], bool inter) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = inter ? 2 * k : k, j = inter ? 2 * k + 1 : 4 + k;
        const float x = v[i], y = v[j];
        v[i] = x * c[k] - y * s[k];
        v[j] = y * c[k] + x * s[k];
    }
}

// Cosines and sines of a token for lane c; false (and the error reported) for a position outside the table.
__device__ __forceinline__ bool angles(const QkArgs& A, long token, int c, bool turned, float cs[4], float sn[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        cs[k] = 1.f;
        sn[k] = 0.f;
    }
    if (A.R == 0) return true;
    const int p = A.pos ? A.pos[token] : (int)(token % A.T);
    if (p < 0 || p >= A.n_pos) {
        if (c == 0) atomicOr(A.err, DP_ERRBIT_INDEX);
        return false;
    }
    if (turned) {
        Num<false>::load4(A.cos + (size_t)p * (A.R / 2) + 4 * c, cs);
        Num<false>::load4(A.sin + (size_t)p * (A.R / 2) + 4 * c, sn);
    }
    return true;
}

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// How the SLOTS = 64 / LPH heads that a wave works on at a time lie: all of one token, `round` rounds of them, or of `tpw` whole tokens.
template <int LPH>
struct Slots {
    static constexpr int N = 64 / LPH;
    int heads, tpw, token, first;
    bool on;
    __device__ __forceinline__ Slots(int heads_, int lane) : heads(heads_) {
        const int s = lane / LPH;
        tpw = heads < N ? N / heads : 1;
        token = heads < N ? s / heads : 0;
        first = heads < N ? s - token * heads : s;
        on = token < tpw;
    }
};

template <bool BF16, int LPH>
__global__ __launch_bounds__(256) void qk_norm_kernel(QkArgs A, void* __restrict__ yq, void* __restrict__ yk) {
    typedef Num<BF16> IO;
    typedef typename IO::elem elem;
    const int lane = threadIdx.x & 63, c = lane % LPH;
    const Slots<LPH> sl(A.Hq + A.Hk, lane);
    const long token = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * sl.tpw + sl.token;
    if (!sl.on || token >= A.tokens) return;
    const Part P = part_of(A, c);
    float cs[4], sn[4];
    const bool good = angles(A, token, c, P.turned, cs, sn);
    const float inv = 1.f / (float)A.D;
    for (int h = sl.first; h < sl.heads; h += Slots<LPH>::N) {
        const bool isq = h < A.Hq;
        const elem* x = isq ? (const elem*)A.q + token * A.ldq + (long)h * A.D : (const elem*)A.k + token * A.ldk + (long)(h - A.Hq) * A.D;
        elem* y = isq ? (elem*)yq + (token * A.Hq + h) * A.D : (elem*)yk + (token * A.Hk + h - A.Hq) * A.D;
        const float* g = isq ? A.gq : A.gk;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, gv[8];
        if (P.on) {
            IO::load4(x + P.a, v);
            IO::load4(x + P.b, v + 4);
        }
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e] * v[e];
        const float r = 1.f / sqrtf(head_sum<LPH>(s) * inv + A.eps);
        if (!P.on) continue;
        Num<false>::load4(g + P.a, gv);
        Num<false>::load4(g + P.b, gv + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = good ? v[e] * r * gv[e] : 0.f;
        if (P.turned) turn(v, cs, sn, A.inter);
        IO::store4(y + P.a, v);
        IO::store4(y + P.b, v + 4);
    }
}

// out[example][chunk][2][D] = gradients of the gains over a chunk's tokens; dq, dk, if wanted, laid out as q, k.
template <bool BF16, int LPH>
__global__ __launch_bounds__(256) void qk_norm_grads_kernel(QkArgs A, const void* __restrict__ dyq, const void* __restrict__ dyk, void* __restrict__ dq, void* __restrict__ dk,
                                                            int wanted, int chunks, int per, float* __restrict__ out) {
    typedef Num<BF16> IO;
    typedef typename IO::elem elem;
    extern __shared__ float red[];  // [4 waves][2][D]
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = lane % LPH;
    const Slots<LPH> sl(A.Hq + A.Hk, lane);
    const int ex = blockIdx.x / chunks, ch = blockIdx.x - ex * chunks;
    const int t0 = ch * per, t1 = t0 + per < A.T ? t0 + per : A.T;
    const Part P = part_of(A, c);
    const float inv = 1.f / (float)A.D;
    float accq[8] = {}, acck[8] = {}, gq[8] = {}, gk[8] = {};
    if (P.on) {
        if (A.Hq) {
            Num<false>::load4(A.gq + P.a, gq);
            Num<false>::load4(A.gq + P.b, gq + 4);
        }
        if (A.Hk) {
            Num<false>::load4(A.gk + P.a, gk);
            Num<false>::load4(A.gk + P.b, gk + 4);
        }
    }
    for (int t = t0 + w * sl.tpw + sl.token; t < t1 && sl.on; t += 4 * sl.tpw) {
        const long token = (long)ex * A.T + t;
        float cs[4], sn[4];
        const bool good = angles(A, token, c, P.turned, cs, sn);
#pragma unroll
        for (int k = 0; k < 4; ++k) sn[k] = -sn[k];
        for (int h = sl.first; h < sl.heads; h += Slots<LPH>::N) {
            const bool isq = h < A.Hq;
            const long at = isq ? token * A.ldq + (long)h * A.D : token * A.ldk + (long)(h - A.Hq) * A.D;
            const elem* x = (isq ? (const elem*)A.q : (const elem*)A.k) + at;
            const elem* dy = isq ? (const elem*)dyq + (token * A.Hq + h) * A.D : (const elem*)dyk + (token * A.Hk + h - A.Hq) * A.D;
            float v[8] = {}, u[8] = {};
            if (P.on) {
                IO::load4(x + P.a, v);
                IO::load4(x + P.b, v + 4);
                IO::load4(dy + P.a, u);
                IO::load4(dy + P.b, u + 4);
            }
            if (P.turned) turn(u, cs, sn, A.inter);
            float s = 0.f, m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s += v[e] * v[e];
                m += (isq ? gq[e] : gk[e]) * u[e] * v[e];
            }
            const float r = 1.f / sqrtf(head_sum<LPH>(s) * inv + A.eps);
            m = head_sum<LPH>(m) * inv * r;
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = v[e] * r, ux = good ? u[e] * xh : 0.f;
                if (isq) accq[e] += ux;
                else acck[e] += ux;
                d[e] = good ? r * ((isq ? gq[e] : gk[e]) * u[e] - xh * m) : 0.f;
            }
            if (P.on && wanted) {
                elem* o = (isq ? (elem*)dq : (elem*)dk) + at;
                IO::store4(o + P.a, d);
                IO::store4(o + P.b, d + 4);
            }
        }
    }
    // over the heads of a wave, then over the waves
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = LPH; o < 64; o <<= 1) {
            accq[e] += __shfl_xor(accq[e], o, 64);
            acck[e] += __shfl_xor(acck[e], o, 64);
        }
    }
    if (lane < LPH && P.on) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = e < 4 ? P.a + e : P.b + e - 4;
            red[(2 * w) * A.D + j] = accq[e];
            red[(2 * w + 1) * A.D + j] = acck[e];
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * A.D; j += 256)
        out[(size_t)blockIdx.x * 2 * A.D + j] = (red[j] + red[2 * A.D + j]) + (red[4 * A.D + j] + red[6 * A.D + j]);
}

// grads[example][n] = sum over its chunks
__global__ __launch_bounds__(256) void qk_join_kernel(const float* __restrict__ part, int chunks, int n, float* __restrict__ grads) {
    const float* p = part + (size_t)blockIdx.x * chunks * n;
    for (int j = threadIdx.x; j < n; j += 256) {
        float s = p[j];
        for (int k = 1; k < chunks; ++k) s += p[(size_t)k * n + j];
        grads[(size_t)blockIdx.x * n + j] = s;
    }
}

template <typename F>
void by_lanes(int D, F f) {
    if (D <= 8) f(std::integral_constant<int, 1>());
    else if (D <= 16) f(std::integral_constant<int, 2>());
    else if (D <= 32) f(std::integral_constant<int, 4>());
    else if (D <= 64) f(std::integral_constant<int, 8>());
    else if (D <= 128) f(std::integral_constant<int, 16>());
    else if (D <= 256) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
}

QkArgs make_args(dp_ctx* ctx, const dp_qk_args& a) {
    return {a.q, a.k, a.gain_q, a.gain_k, a.cos, a.sin, a.positions, ctx->err_word, (long)a.ldq, (long)a.ldk, a.n_pos, a.interleaved, a.T, a.Hq, a.Hk, a.D, a.R, a.eps, (long)a.B * a.T};
}

}  // namespace

dp_status dpk_qk_norm(dp_ctx* ctx, const dp_qk_args& a, void* yq, void* yk) {
    const QkArgs A = make_args(ctx, a);
    by_lanes(a.D, [&](auto lph) {
        constexpr int L = decltype(lph)::value;
        const int heads = a.Hq + a.Hk, tpw = heads < 64 / L ? 64 / L / heads : 1;
        const dim3 grid((unsigned)((A.tokens + 4 * tpw - 1) / (4 * tpw)));
        if (a.dtype == DP_BF16) hipLaunchKernelGGL((qk_norm_kernel<true, L>), grid, dim3(256), 0, ctx->stream, A, yq, yk);
        else hipLaunchKernelGGL((qk_norm_kernel<false, L>), grid, dim3(256), 0, ctx->stream, A, yq, yk);
    });
    DP_LAUNCH_CHECK(ctx, "qk_norm");
    return DP_OK;
}

dp_status dpk_qk_norm_grads(dp_ctx* ctx, const dp_qk_args& a, const void* dyq, const void* dyk, float* grads, void* dq, void* dk, bool wanted) {
    const QkArgs A = make_args(ctx, a);
    // workgroups of an example: as many as fill the chip, of at least four tokens, as long as their parts fit
    int chunks = a.B >= 2048 ? 1 : (2048 + a.B - 1) / a.B;
    if (chunks > (a.T + 3) / 4) chunks = (a.T + 3) / 4;
    const size_t room = ctx->ws_bytes / ((size_t)a.B * 2 * a.D * sizeof(float));
    if (chunks > 1 && (size_t)chunks > room) chunks = room > 1 ? (int)room : 1;
    const int per = (a.T + chunks - 1) / chunks;
    chunks = (a.T + per - 1) / per;
    if ((long)a.B * chunks > 0x7FFFFFFFl) {
        DP_SET_ERR(ctx, "too many examples for one launch");
        return DP_ERR_SHAPE;
    }
    float* part = chunks > 1 ? (float*)ctx->ws : grads;
    by_lanes(a.D, [&](auto lph) {
        constexpr int L = decltype(lph)::value;
        const dim3 grid((unsigned)(a.B * chunks));
        const size_t lds = 8 * (size_t)a.D * sizeof(float);
        if (a.dtype == DP_BF16) hipLaunchKernelGGL((qk_norm_grads_kernel<true, L>), grid, dim3(256), lds, ctx->stream, A, dyq, dyk, dq, dk, wanted, chunks, per, part);
        else hipLaunchKernelGGL((qk_norm_grads_kernel<false, L>), grid, dim3(256), lds, ctx->stream, A, dyq, dyk, dq, dk, wanted, chunks, per, part);
    });
    DP_LAUNCH_CHECK(ctx, "qk_norm_grads");
    if (chunks > 1) {
        hipLaunchKernelGGL(qk_join_kernel, dim3(a.B), dim3(256), 0, ctx->stream, part, chunks, 2 * a.D, grads);
        DP_LAUNCH_CHECK(ctx, "qk_join");
    }
    return DP_OK;
}
