// A relative position bias learned by buckets of distance, and every example's gradient of its table.
//
// A pair of a query at position p and a key at position k has distance k - p; a side's buckets are runs of distances (the last one open),
// so a bucket is a run of diagonals of the [queries x keys] plane.  Forward: a row of the bias is a window on one line of 2 T - 1 values
// that moves by one from row to row.  Gradient: the sums of the diagonals, then those of the buckets' runs.
//
// Roofline: HBM, both.  The forward writes H Tq Tk elements, the gradient reads L B H Tq Tk of them with one addition each.
#include "dp_common.h"

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));
typedef u32x4_t u32x4_a4 __attribute__((aligned(4)));

constexpr int MAX_SIDE = 128;    // buckets of a side
constexpr int REL_LAYERS = 128;  // layers per launch

struct Buckets {
    int start[MAX_SIDE];  // first distance of a side's bucket
    int n, both;
};

// The bucket of a key `rel` behind its query (negative: in front).
__device__ __forceinline__ int bucket_of(const Buckets& b, int rel) {
    const int dist = rel <= 0 ? -rel : b.both ? rel : 0;
    int lo = 0, hi = b.n;  // the last start that is not above the distance
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.start[mid] <= dist) lo = mid;
        else hi = mid;
    }
    return b.both && rel > 0 ? lo + b.n : lo;
}

constexpr int FWD_ROWS = 32, FWD_COLS = 256 * 8;

// bias[h][q][k] = table[bucket(k - (Tk - Tq + q))][h]: a workgroup writes 32 rows of 2,048 columns.  The line of values under the tile
// lies in LDS; a thread keeps the eight under its columns and takes in one more per row.
template <bool BF16>
__global__ __launch_bounds__(256) void relbias_kernel(const float* __restrict__ table, Buckets bk, int H, int Tq, int Tk, int row_tiles, int col_tiles, void* __restrict__ out) {
    __shared__ float line[FWD_ROWS + FWD_COLS];
    int b = blockIdx.x;
    const int ct = b % col_tiles;
    b /= col_tiles;
    const int rt = b % row_tiles, h = b / row_tiles;
    const int q0 = rt * FWD_ROWS, k0 = ct * FWD_COLS, rows = Tq - q0 < FWD_ROWS ? Tq - q0 : FWD_ROWS, cols = Tk - k0 < FWD_COLS ? Tk - k0 : FWD_COLS;
    // line[j]: distance j + base; row q0 + r, column k0 + c is line[c - r + rows - 1]
    const int base = k0 - (Tk - Tq + q0) - (rows - 1);
    for (int j = threadIdx.x; j < rows + cols - 1; j += 256) line[j] = table[(size_t)bucket_of(bk, j + base) * H + h];
    __syncthreads();
    const int c = threadIdx.x * 8;
    if (c >= cols) return;
    const int have = cols - c < 8 ? cols - c : 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < have ? line[c + e + rows - 1] : 0.f;
    size_t at = ((size_t)h * Tq + q0) * Tk + k0 + c;
    for (int r = 0; r < rows; ++r, at += Tk) {
        if (have == 8) {
            if constexpr (BF16) {
                typedef __bf16 bf16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));
                bf16x8_t w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (__bf16)v[e];
                *reinterpret_cast<bf16x8_a2*>((__bf16*)out + at) = w;
            } else {
                typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));
                f32x4_a4* o = reinterpret_cast<f32x4_a4*>((float*)out + at);
                o[0] = f32x4_t{v[0], v[1], v[2], v[3]};
                o[1] = f32x4_t{v[4], v[5], v[6], v[7]};
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < have) {
                    if constexpr (BF16) ((__bf16*)out)[at + e] = (__bf16)v[e];
                    else ((float*)out)[at + e] = v[e];
                }
        }
#pragma unroll
        for (int e = 7; e > 0; --e) v[e] = v[e - 1];
        if (r + 1 < rows) v[0] = line[c + rows - 2 - r];
    }
}

struct RelLayers {
    const void* x[REL_LAYERS];
    int n;
};

// How a workgroup's threads share the plane of one example and head, in blocks of 8 x 8: `wide` neighbouring threads take neighbouring
// blocks of a row of blocks; gr such groups take its rows of blocks in turn, `m` each, and gl of these the layers in turn.
struct RelPlan {
    int nb, rb;        // blocks in a row and in a column of the plane
    int splits, per;   // workgroups of a plane, rows of blocks of each
    int wide, gr, gl, m;
};

constexpr int SUMS = 15;  // diagonals of a block of 8 x 8

// part[i][bucket][h] (or, with several parts, part[slot][...]) = sums of the buckets.
//
// A thread walks down a band of blocks, its column of blocks one further with every row of blocks, so that the 15 diagonals it adds up stay
// the same ones: one addition an element, no exchange.  Where it steps over the last column it goes on with the band that begins in column 0
// (bands p and p - nb together have one block in every row of blocks).  The sums of both bands go to LDS and are joined there.
template <bool BF16>
__global__ __launch_bounds__(256) void relbias_grads_kernel(RelLayers t, Buckets bk, const int32_t* __restrict__ lengths, int causal, RelPlan pl, int B, int H, int Tq,
                                                            int Tk, float* __restrict__ part, int slot0) {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    constexpr int W = BF16 ? 4 : 8;  // words of eight elements
    extern __shared__ float lds[];
    float* const hold = lds;                        // [band before or after the step over][diagonal][thread]
    float* const diag = lds + 2 * SUMS * 256;       // [Tq + Tk - 1]
    const int D = Tq + Tk - 1, off = Tk - Tq, tid = threadIdx.x;
    const int s = blockIdx.x % pl.splits, mat = blockIdx.x / pl.splits, i = mat / H, h = mat - i * H;
    int len = Tk;
    if (lengths) len = min(max(lengths[i], 0), Tk);
    const int nq = min(max(len - off, 0), Tq);
    const int rb0 = s * pl.per, rb1 = min(rb0 + pl.per, (nq + 7) / 8);
    const int grp = tid / pl.wide, pp = tid - grp * pl.wide, lg = grp / pl.gr, rg = grp - lg * pl.gr;
    const bool works = lg < pl.gl;
    const int ra = rb0 + rg * pl.m, rz = min(ra + pl.m, rb1);
    // elements from the start of this plane to the end of the tensor (what a load may touch)
    const long left = ((long)B * H - mat) * Tq * Tk;
    const int room = left < 0x7FFFFFFF ? (int)left : 0x7FFFFFFF;

    for (int p0 = 0; p0 < pl.nb; p0 += pl.wide) {
        const int p = p0 + pp;
        float acc[SUMS];
#pragma unroll
        for (int e = 0; e < SUMS; ++e) acc[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * SUMS; ++e) hold[e * 256 + tid] = 0.f;
        int over = 0;
        if (works && p < pl.nb) {
            for (int rb = ra; rb < rz; ++rb) {
                int cb = rb + p;
                if (cb >= pl.nb) {
                    cb -= pl.nb;
                    if (!over) {
#pragma unroll
                        for (int e = 0; e < SUMS; ++e) {
                            hold[e * 256 + tid] = acc[e];
                            acc[e] = 0.f;
                        }
                        over = 1;
                    }
                }
                const int q0 = rb * 8, k0 = cb * 8, rows = nq - q0, cut = len - k0;  // (len is never above Tk)
                if (cut <= 0 || (causal && k0 > q0 + 7 + off)) continue;
                uint32_t mask[W];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if constexpr (BF16) mask[w] = cut >= 2 * w + 2 ? 0xFFFFFFFFu : cut == 2 * w + 1 ? 0xFFFFu : 0u;
                    else mask[w] = cut > w ? 0xFFFFFFFFu : 0u;
                }
                const int at = q0 * Tk + k0;
                for (int l = lg; l < t.n; l += pl.gl) {
                    const elem* x = (const elem*)t.x[l] + (size_t)mat * Tq * Tk + at;
                    uint32_t v[8][W];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
#pragma unroll
                        for (int w = 0; w < W; ++w) v[r][w] = 0u;
                        if (r >= rows) continue;
                        if (at + r * Tk + 8 <= room) {
                            if constexpr (BF16) {
                                const u32x4_t a = *reinterpret_cast<const u32x4_a2*>(x + r * Tk);
#pragma unroll
                                for (int w = 0; w < 4; ++w) v[r][w] = a[w];
                            } else {
                                const u32x4_t a = *reinterpret_cast<const u32x4_a4*>(x + r * Tk), b = *reinterpret_cast<const u32x4_a4*>(x + r * Tk + 4);
#pragma unroll
                                for (int w = 0; w < 4; ++w) {
                                    v[r][w] = a[w];
                                    v[r][4 + w] = b[w];
                                }
                            }
                        } else {  // the last elements of the tensor
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (e < cut) {
                                    if constexpr (BF16) v[r][e >> 1] |= (uint32_t)x[r * Tk + e] << (16 * (e & 1));
                                    else v[r][e] = __float_as_uint(x[r * Tk + e]);
                                }
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 8; ++r)
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            const uint32_t x2 = v[r][w] & mask[w];
                            if constexpr (BF16) {
                                acc[7 + 2 * w - r] += dp_bf16_lo(x2);
                                acc[8 + 2 * w - r] += dp_bf16_hi(x2);
                            } else {
                                acc[7 + w - r] += __uint_as_float(x2);
                            }
                        }
                }
            }
        }
#pragma unroll
        for (int e = 0; e < SUMS; ++e) hold[(over * SUMS + e) * 256 + tid] = acc[e];
        __syncthreads();
        // diag[j]: keys j - (Tq - 1) columns behind their row, i.e. rel = j - (Tk - 1)
        for (int j = tid; j < D; j += 256) {
            const int dd = j - (Tq - 1), band = dd >> 3, e = dd & 7;
            float sum = p0 ? diag[j] : 0.f;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const int b = band + side, ee = e + 7 - 8 * side, after = b < 0, q = (after ? b + pl.nb : b) - p0;
                if (ee < 0 || q < 0 || q >= pl.wide || q + p0 >= pl.nb) continue;
                for (int g = 0; g < pl.gr * pl.gl; ++g) sum += hold[(after * SUMS + ee) * 256 + g * pl.wide + q];
            }
            diag[j] = sum;
        }
        __syncthreads();
    }
    // the buckets' runs, a wave each
    const int lane = tid & 63, nbk = bk.both ? 2 * bk.n : bk.n, far = 1 << 30;
    for (int j = tid >> 6; j < nbk; j += 4) {
        const int b = j < bk.n ? j : j - bk.n;
        const int lo = bk.start[b], hi = b + 1 < bk.n ? bk.start[b + 1] : far;  // distances lo .. hi - 1
        int from, to;                                                          // rel from .. to
        if (j < bk.n) {
            from = 1 - hi;
            to = !bk.both && lo == 0 && hi > 0 ? far : -lo;
        } else {
            from = max(lo, 1);
            to = hi - 1;
        }
        if (causal) to = min(to, 0);
        const int a = max(from + Tk - 1, 0), z = min(to, D) + Tk - 1;
        float sum = 0.f;
        for (int k = a + lane; k <= z && k < D; k += 64) sum += diag[k];
        sum = dp_wave_sum(sum);
        if (lane == 0) part[(((size_t)(slot0 + s) * B + i) * nbk + j) * H + h] = sum;
    }
}

__global__ __launch_bounds__(256) void relbias_join_kernel(const float* __restrict__ part, int slots, size_t n, float* __restrict__ out) {
    const size_t k = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= n) return;
    float s = part[k];
    for (int j = 1; j < slots; ++j) s += part[j * n + k];
    out[k] = s;
}

Buckets make_buckets(int n, const int32_t* starts, int both) {
    Buckets b{};
    for (int j = 0; j < n; ++j) b.start[j] = starts[j];
    b.n = n;
    b.both = both ? 1 : 0;
    return b;
}

RelPlan rel_plan(int L, int Tq, int Tk, int splits) {
    RelPlan p;
    p.nb = (Tk + 7) / 8;
    p.rb = (Tq + 7) / 8;
    p.per = (p.rb + splits - 1) / splits;
    p.splits = (p.rb + p.per - 1) / p.per;
    p.wide = p.nb < 256 ? p.nb : 256;
    const int groups = 256 / p.wide;
    p.m = (p.per + groups - 1) / groups;
    p.gr = (p.per + p.m - 1) / p.m;
    p.gl = groups / p.gr < L ? groups / p.gr : L;
    return p;
}

}  // namespace

dp_status dpk_relbias(dp_ctx* ctx, const float* table, int n, const int32_t* starts, int both, int H, int Tq, int Tk, dp_dtype dt, void* out) {
    const Buckets bk = make_buckets(n, starts, both);
    const int row_tiles = (Tq + FWD_ROWS - 1) / FWD_ROWS, col_tiles = (Tk + FWD_COLS - 1) / FWD_COLS;
    const long grid = (long)H * row_tiles * col_tiles;
    if (grid > 0x7FFFFFFFl) {
        DP_SET_ERR(ctx, "H * Tq * Tk too large for one launch");
        return DP_ERR_SHAPE;
    }
    if (dt == DP_BF16) hipLaunchKernelGGL(relbias_kernel<true>, dim3((unsigned)grid), dim3(256), 0, ctx->stream, table, bk, H, Tq, Tk, row_tiles, col_tiles, out);
    else hipLaunchKernelGGL(relbias_kernel<false>, dim3((unsigned)grid), dim3(256), 0, ctx->stream, table, bk, H, Tq, Tk, row_tiles, col_tiles, out);
    DP_LAUNCH_CHECK(ctx, "relbias");
    return DP_OK;
}

dp_status dpk_relbias_grads(dp_ctx* ctx, int n_layers, const void* const* dS, dp_dtype dt, const int32_t* lengths, int causal, int n, const int32_t* starts, int both,
                            int B, int H, int Tq, int Tk, float* grads) {
    const Buckets bk = make_buckets(n, starts, both);
    const size_t out = (size_t)B * H * n * (both ? 2 : 1);
    const long planes = (long)B * H;
    const int launches = (n_layers + REL_LAYERS - 1) / REL_LAYERS;
    // workgroups of a plane: as many as fill the chip (five of a CU fit its LDS at T = 128), as long as their parts fit
    int splits = planes >= 1024 ? 1 : (int)(1024 / planes);
    const size_t room = ctx->ws_bytes / (out * sizeof(float));
    if ((size_t)splits * launches > room) splits = room / launches > 1 ? (int)(room / launches) : 1;
    RelPlan pl = rel_plan(n_layers < REL_LAYERS ? n_layers : REL_LAYERS, Tq, Tk, splits < (Tq + 7) / 8 ? splits : (Tq + 7) / 8);
    const int slots = pl.splits * launches;
    if (planes * pl.splits > 0x7FFFFFFFl) {
        DP_SET_ERR(ctx, "B * H = %ld is too large for one launch", planes);
        return DP_ERR_SHAPE;
    }
    if (slots > 1 && (size_t)slots > room) {
        DP_SET_ERR(ctx, "the workspace does not hold %d parts of the gradients", slots);
        return DP_ERR_WORKSPACE;
    }
    float* part = slots > 1 ? (float*)ctx->ws : grads;
    const size_t lds = (2 * SUMS * 256 + (size_t)(Tq + Tk - 1)) * sizeof(float);
    for (int l0 = 0; l0 < n_layers; l0 += REL_LAYERS) {
        RelLayers t{};
        t.n = n_layers - l0 < REL_LAYERS ? n_layers - l0 : REL_LAYERS;
        for (int l = 0; l < t.n; ++l) t.x[l] = dS[l0 + l];
        const dim3 grid((unsigned)(planes * pl.splits));
        const int slot0 = l0 / REL_LAYERS * pl.splits;
        auto launch = [&](auto kernel) {
            if (lds > 65536) DP_HIP_CHECK(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024));
            hipLaunchKernelGGL(kernel, grid, dim3(256), lds, ctx->stream, t, bk, lengths, causal, pl, B, H, Tq, Tk, part, slot0);
            return DP_OK;
        };
        const dp_status st = dt == DP_BF16 ? launch(relbias_grads_kernel<true>) : launch(relbias_grads_kernel<false>);
        if (st != DP_OK) return st;
        DP_LAUNCH_CHECK(ctx, "relbias_grads");
    }
    if (slots > 1) {
        const size_t blocks = (out + 255) / 256;
        if (blocks > 0x7FFFFFFF) {
            DP_SET_ERR(ctx, "B * H * buckets too large for one launch");
            return DP_ERR_SHAPE;
        }
        hipLaunchKernelGGL(relbias_join_kernel, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, part, slots, out, grads);
        DP_LAUNCH_CHECK(ctx, "relbias_join");
    }
    return DP_OK;
}
