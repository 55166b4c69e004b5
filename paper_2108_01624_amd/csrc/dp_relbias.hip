// A relative position bias learned by buckets of distance, and every example's gradient of its table.
//
// A pair of a query at position p and a key at position k has distance k - p; a side's buckets are runs of distances (the last one open),
// so a bucket is a run of diagonals of the [queries x keys] plane.  Forward: a row of the bias is a window on one line of 2 T - 1 values
// that moves by one from row to row.  Gradient: the sums of the diagonals, then those of the buckets' runs.
//
// Roofline: HBM, both.  The forward writes H Tq Tk elements, the gradient reads L B H Tq Tk of them with one addition each.
// Forward, 16 x 2,048 x 2,048: bf16 23 us (5.8 TB/s; 28 where the buffer is another from call to call), fp32 42 us (6.4); gradient, 24 layers x 128 x 16 x 128 x 128 bf16: 240 us (6.7 TB/s),
// 12 layers x 64 x 16 x 125 x 125: 72 us (5.3).
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

// The bucket of a key `rel` behind its query (negative: in front), by a side's n starts.
__device__ __forceinline__ int bucket_of(const int* start, int n, int both, int rel) {
    const int dist = rel <= 0 ? -rel : both ? rel : 0;
    int lo = 0, hi = n;  // the last start that is not above the distance: of most places of a long line the last of all
    if (dist >= start[n - 1]) lo = n - 1;
    else
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= dist) lo = mid;
            else hi = mid;
        }
    return both && rel > 0 ? lo + n : lo;
}

constexpr int FWD_ROWS = 16;

// bias[h][q][k] = table[bucket(k - (Tk - Tq + q))][h]: a workgroup writes 16 rows of 256 x 16 bytes.  The line of values under the tile lies in
// LDS; a thread keeps those under its columns and takes in one more per row.
template <bool BF16>
__global__ __launch_bounds__(256) void relbias_kernel(const float* __restrict__ table, Buckets bk, int H, int Tq, int Tk, int row_tiles, int col_tiles, void* __restrict__ out) {
    constexpr int E = BF16 ? 8 : 4, COLS = 256 * E;  // columns of a thread: 16 bytes
    typedef typename std::conditional<BF16, __bf16, float>::type elem;
    typedef elem pack __attribute__((ext_vector_type(E)));
    typedef pack pack_any __attribute__((aligned(sizeof(elem))));
    __shared__ float line[FWD_ROWS + COLS], value[2 * MAX_SIDE];
    __shared__ int start[MAX_SIDE];
    int b = blockIdx.x;
    const int ct = b % col_tiles;
    b /= col_tiles;
    const int rt = b % row_tiles, h = b / row_tiles;
    const int q0 = rt * FWD_ROWS, k0 = ct * COLS, rows = min(Tq - q0, FWD_ROWS), cols = min(Tk - k0, COLS);
    // line[j]: distance j + base; row q0 + r, column k0 + c is line[c - r + rows - 1]
    const int base = k0 - (Tk - Tq + q0) - (rows - 1);
    if ((int)threadIdx.x < bk.n) start[threadIdx.x] = bk.start[threadIdx.x];
    if ((int)threadIdx.x < (bk.both ? 2 * bk.n : bk.n)) value[threadIdx.x] = table[(size_t)threadIdx.x * H + h];
    __syncthreads();
    for (int j = threadIdx.x; j < rows + cols - 1; j += 256) line[j] = value[bucket_of(start, bk.n, bk.both, j + base)];
    __syncthreads();
    const int c = threadIdx.x * E;
    if (c >= cols) return;
    const int have = min(cols - c, E);
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < have ? line[c + e + rows - 1] : 0.f;
    elem* o = (elem*)out + ((size_t)h * Tq + q0) * Tk + k0 + c;
    for (int r = 0; r < rows; ++r, o += Tk) {
        if (have == E) {
            pack w;
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = (elem)v[e];
            *reinterpret_cast<pack_any*>(o) = w;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < have) o[e] = (elem)v[e];
        }
#pragma unroll
        for (int e = E - 1; e > 0; --e) v[e] = v[e - 1];
        if (r + 1 < rows) v[0] = line[c + rows - 2 - r];
    }
}

struct RelLayers {
    const void* x[REL_LAYERS];
    int n;
};

// How a workgroup's threads share what counts of a plane, in blocks of 8 x 8: `wide` neighbouring threads take neighbouring blocks of a row
// of blocks; gr such groups take the steps (rows of blocks, pairs of them under FOLD) in turn, `m` each, and gl of these the layers in turn.
struct RelPlan {
    int nb, np, steps;  // blocks in a row, threads for one (of which there may be more than `wide`), steps
    int used, per;      // workgroups that share the steps, and steps of each
    int wide, gr, gl, m;
};
// rows, cols: what counts of a plane that has up to splits workgroups for all_rows x all_cols; a short example has fewer to itself, by its share of
// the places.
template <bool FOLD, int NT>
__device__ __forceinline__ RelPlan rel_plan(int layers, int rows, int cols, int all_rows, int all_cols, int splits) {
    RelPlan p;
    p.nb = max((cols + 7) / 8, 1);
    p.np = FOLD ? p.nb + 1 : p.nb;
    p.steps = FOLD ? (p.nb + 1) / 2 : (rows + 7) / 8;
    p.used = splits;
    if (splits > 1 && cols < all_cols) {
        const float share = (float)rows * (float)cols / ((float)all_rows * (float)all_cols);
        p.used = min(max((int)ceilf(share * (float)splits), 1), splits);
    }
    p.per = max((int)((unsigned)(p.steps + p.used - 1) / (unsigned)p.used), 1);
    p.wide = min(p.np, NT);
    const unsigned groups = (unsigned)NT / (unsigned)p.wide;
    p.m = (unsigned)(p.per + groups - 1) / groups;
    p.gr = (unsigned)(p.per + p.m - 1) / (unsigned)p.m;
    p.gl = min((int)(groups / (unsigned)p.gr), layers);
    return p;
}

constexpr int SUMS = 15;  // diagonals of a block of 8 x 8
constexpr size_t MOST_LDS = (2 * SUMS * 256 + DP_REL_MAX_LINE) * sizeof(float);  // sums of 256 threads, and all diagonals
static_assert(MOST_LDS + 256 <= 160 * 1024, "the diagonals of a plane lie in a CU's local memory");

// part[i][bucket][h] (or, with several parts, part[slot][...]) = sums of the buckets.
//
// A thread walks down a band of blocks, its column of blocks one further with every row of blocks, so that the 15 diagonals it adds up stay
// the same ones: one addition an element, no exchange.  Where it steps over the last column it goes on with the band that begins in column 0
// (bands p and p - nb together have one block in every row of blocks).  The sums of both bands go to LDS and are joined there.
// FOLD, under a causal mask over a square: a step is a row of blocks s and the one as far from the end, nb - 1 - s, which have nb + 1 blocks that
// count together, a thread each: the first nb - s threads those of the lower row, of bands 0, -1, ..., the others those of the upper one, of bands
// -s .. 0.  Again a thread has two bands, one after the other, and half as many steps.  (6 layers x 8 x 16 x 512 x 512 bf16: 43 us, without a mask 70.)
//
// Bands in which every distance belongs to the last bucket of its side, those below near_lo and above near_hi, are not taken apart: their sums go to
// one number a side (4 x 16 x 1,024 x 1,024 of one layer, 2,047 diagonals of which 300 are near: 34 -> 30 us).
//
// bf16 loads are streamed (240 us, cached 269); of fp32 a thread's eight columns are two loads that share their lines, which streaming
// loses (6 layers of ragged examples of up to 509 tokens: 98 us cached, 115 streamed).
template <bool BF16, bool FOLD, int NT>
__global__ __launch_bounds__(NT) void relbias_grads_kernel(RelLayers t, Buckets bk, const int32_t* __restrict__ lengths, int causal, int splits, int near_lo, int near_hi, int B,
                                                           int H, int Tq, int Tk, float* __restrict__ part, int slot0) {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    constexpr int W = BF16 ? 4 : 8;  // words of eight elements
    extern __shared__ float lds[];
    const int off = Tk - Tq, tid = threadIdx.x;
    const int d_lo = max(8 * near_lo - 7, 1 - Tq), d_hi = min(8 * near_hi + 7, Tk - 1);  // columns minus rows of the near bands' diagonals
    float* const hold = lds;                 // [band before or after the step over][diagonal][thread]
    float* const diag = lds + 2 * SUMS * NT; // [d_hi - d_lo + 1]
    __shared__ float far_sum[2][NT / 64];
    const int s = blockIdx.x % (unsigned)splits, mat = blockIdx.x / (unsigned)splits, i = mat / H, h = mat - i * H;
    int len = Tk;
    if (lengths) len = min(max(lengths[i], 0), Tk);
    const int nq = min(max(len - off, 0), Tq);  // rows and columns that count: nq and len
    const RelPlan pl = rel_plan<FOLD, NT>(t.n, nq, len, Tq, Tk, splits);
    if (s >= pl.used) {
        const int nbk = bk.both ? 2 * bk.n : bk.n;
        for (int j = tid; j < nbk; j += NT) part[(((size_t)(slot0 + s) * B + i) * nbk + j) * H + h] = 0.f;
        return;
    }
    const int s0 = s * pl.per, s1 = min(s0 + pl.per, pl.steps);
    const int grp = tid / (unsigned)pl.wide, pp = tid - grp * pl.wide, lg = grp / (unsigned)pl.gr, rg = grp - lg * pl.gr;
    const bool works = lg < pl.gl;
    const int sa = s0 + rg * pl.m, sz = min(sa + pl.m, s1);
    // elements from the start of this plane to the end of the tensor (what a load may touch)
    const long left = ((long)B * H - mat) * Tq * Tk;
    const int room = left < 0x7FFFFFFF ? (int)left : 0x7FFFFFFF;

    float past = 0.f, future = 0.f;
    for (int p0 = 0; p0 < pl.np; p0 += pl.wide) {
        const int p = p0 + pp;
        float acc[SUMS];
        // the sums of this thread's band before or after its step over; those that it never comes to are zeros
        auto put = [&](int after) {
            const int band = after ? p - pl.nb : FOLD ? -p : p;
            if (band >= near_lo && band <= near_hi) {
#pragma unroll
                for (int e = 0; e < SUMS; ++e) hold[(after * SUMS + e) * NT + tid] = acc[e];
            } else {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < SUMS; ++e) sum += acc[e];
                if (band < near_lo) past += sum;
                else future += sum;
            }
        };
#pragma unroll
        for (int e = 0; e < SUMS; ++e) acc[e] = 0.f;
        put(0);
        put(1);
        int over = 0;
        if (works && p < pl.np) {
            for (int step = sa; step < sz; ++step) {
                int rb = step, cb = step + p;
                if (cb < pl.nb) {
                    if (FOLD) {
                        rb = pl.nb - 1 - step;
                        cb = rb - p;
                    }
                } else {
                    cb -= pl.nb;
                    if (!over) {
                        put(0);
#pragma unroll
                        for (int e = 0; e < SUMS; ++e) acc[e] = 0.f;
                        over = 1;
                    }
                }
                const int q0 = rb * 8, k0 = cb * 8, rows = nq - q0, cut = len - k0;  // (len is never above Tk)
                if (cut <= 0 || (FOLD ? over && 2 * step == pl.nb - 1 : causal && k0 > q0 + 7 + off)) continue;  // (a middle row is its own other)
                uint32_t mask[W];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if constexpr (BF16) mask[w] = cut >= 2 * w + 2 ? 0xFFFFFFFFu : cut == 2 * w + 1 ? 0xFFFFu : 0u;
                    else mask[w] = cut > w ? 0xFFFFFFFFu : 0u;
                }
                const int at = q0 * Tk + k0;
                for (int l = lg; l < t.n; l += pl.gl) {
                    // (where the layers are not shared out, theirs is a scalar load)
                    const void* base = pl.gl == 1 ? t.x[__builtin_amdgcn_readfirstlane(l)] : t.x[l];
                    const elem* x = (const elem*)base + (size_t)mat * Tq * Tk + at;
                    uint32_t v[8][W];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
#pragma unroll
                        for (int w = 0; w < W; ++w) v[r][w] = 0u;
                        if (r >= rows) continue;
                        if (at + r * Tk + 8 <= room) {
                            if constexpr (BF16) {
                                const u32x4_t a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(x + r * Tk));
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
        put(over);
        __syncthreads();
        // diag[j]: the diagonal of columns d_lo + j behind their rows
        for (int j = tid; j <= d_hi - d_lo; j += NT) {
            const int dd = d_lo + j, band = dd >> 3, e = dd & 7;
            float sum = p0 ? diag[j] : 0.f;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const int b = band + side, ee = e + 7 - 8 * side;
                if (ee < 0 || b < near_lo || b > near_hi) continue;
#pragma unroll
                for (int after = 0; after < 2; ++after) {
                    const int at = after ? b + pl.nb : FOLD ? -b : b, q = at - p0;  // the thread that has band b, before or after its step over
                    if (at < 0 || at >= pl.np || q < 0 || q >= pl.wide) continue;
                    for (int g = 0; g < pl.gr * pl.gl; ++g) sum += hold[(after * SUMS + ee) * NT + g * pl.wide + q];
                }
            }
            diag[j] = sum;
        }
        __syncthreads();
    }
    past = dp_lanes_sum<64>(past);
    future = dp_lanes_sum<64>(future);
    if ((tid & 63) == 0) {
        far_sum[0][tid >> 6] = past;
        far_sum[1][tid >> 6] = future;
    }
    __syncthreads();
    // the buckets' runs, sixteen lanes each
    const int lane = tid & 15, nbk = bk.both ? 2 * bk.n : bk.n, far = 1 << 30;
    for (int j = tid >> 4; j < nbk; j += NT / 16) {
        const int b = j < bk.n ? j : j - bk.n;
        const int lo = bk.start[b], hi = b + 1 < bk.n ? bk.start[b + 1] : far;  // distances lo .. hi - 1
        int from, to, whole = -1;                                              // rel from .. to; the side whose far bands belong to it
        if (j < bk.n) {
            const bool zero = !bk.both && lo == 0 && hi > 0;  // the keys behind the query too
            from = 1 - hi;
            to = zero ? far : -lo;
            if (j == bk.n - 1) whole = 0;
        } else {
            from = max(lo, 1);
            to = hi - 1;
            if (b == bk.n - 1) whole = 1;
        }
        const bool behind = !bk.both && lo == 0 && hi > 0 && !causal;
        if (causal) to = min(to, 0);
        const int a = max(from, d_lo - off) + off - d_lo, z = min(to, d_hi - off) + off - d_lo;  // (places in diag)
        float sum = 0.f;
#pragma unroll 4
        for (int k = a + lane; k <= z; k += 16) sum += diag[k];
        sum = dp_lanes_sum<16>(sum);
        for (int w = 0; w < NT / 64; ++w) {
            if (whole == 0) sum += far_sum[0][w];
            if (whole == 1 || behind) sum += far_sum[1][w];
        }
        if (lane == 0) part[(((size_t)(slot0 + s) * B + i) * nbk + j) * H + h] = sum;
    }
}

// out[k] = sum of the parts of k, sixteen lanes each.
__global__ __launch_bounds__(256) void relbias_join_kernel(const float* __restrict__ part, int slots, size_t n, float* __restrict__ out) {
    const size_t k = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (k >= n) return;
    float s = 0.f;
#pragma unroll 4
    for (int j = threadIdx.x & 15; j < slots; j += 16) s += part[j * n + k];
    s = dp_lanes_sum<16>(s);
    if ((threadIdx.x & 15) == 0) out[k] = s;
}

Buckets make_buckets(int n, const int32_t* starts, int both) {
    Buckets b{};
    for (int j = 0; j < n; ++j) b.start[j] = starts[j];
    b.n = n;
    b.both = both ? 1 : 0;
    return b;
}

}  // namespace

dp_status dpk_relbias(dp_ctx* ctx, const float* table, int n, const int32_t* starts, int both, int H, int Tq, int Tk, dp_dtype dt, void* out) {
    const Buckets bk = make_buckets(n, starts, both);
    const int cols = 256 * (dt == DP_BF16 ? 8 : 4), row_tiles = (Tq + FWD_ROWS - 1) / FWD_ROWS, col_tiles = (Tk + cols - 1) / cols;
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
    // workgroups of a plane: as many as fill the chip, four to a CU, as long as their parts fit (twice as many: 6 x 8 x 16 x 512 x 512 under a
    // causal mask 46 us instead of 43, half as many 46); twice as many where examples may be shorter, and need fewer (6 layers of 24 x 12 of up to 509 tokens, causal: 101 -> 94 us)
    const int aim = lengths ? 2048 : 1024;
    int splits = planes >= aim ? 1 : (int)(aim / planes);
    const bool fold = causal && Tq == Tk;
    const int steps = fold ? (Tq + 15) / 16 : (Tq + 7) / 8;
    if (lengths) {
        // Short examples leave the last workgroups of their planes empty.  Up to 8,192 where a thread then still has about two of its plane's steps, so that
        // the longest examples are not what all wait for (2 layers of 128 x 12 of up to 509 tokens, causal: 171 -> 155 us); and rounded up to an odd number,
        // so that the same part of a plane does not always come to the same XCD (2 layers of 16 x 16 x 1,024, causal: 128 us with 8, 112 with 9; 8 where
        // 7 had been, 6 layers of 24 x 12 x 509: 160 -> 211.  Planes in the inner order, which any number allows: 104 us instead of 94 under its mask).
        // A chain of four steps is thereby cut into three parts, and loses: 2 layers of 256 x 16 x 256 without a mask, bf16: 113 -> 121 us.
        const long across = (Tk + 7) / 8 + (fold ? 1 : 0), chain = steps / (across < 256 ? 256 / across : 1);
        const long more = chain / 2 < 8192 / planes ? chain / 2 : 8192 / planes;
        splits = (more > splits ? (int)more : splits) | 1;
    }
    const size_t room = ctx->ws_bytes / (out * sizeof(float));
    if ((size_t)splits * launches > room) splits = room / launches > 1 ? (int)(room / launches) : 1;
    if (splits > steps) splits = steps;
    const int slots = splits * launches;
    if (planes * splits > 0x7FFFFFFFl) {
        DP_SET_ERR(ctx, "B * H = %ld is too large for one launch", planes);
        return DP_ERR_SHAPE;
    }
    if (slots > 1 && (size_t)slots > room) {
        DP_SET_ERR(ctx, "the workspace does not hold %d parts of the gradients", slots);
        return DP_ERR_WORKSPACE;
    }
    float* part = slots > 1 ? (float*)ctx->ws : grads;
    // A band's distances: 8 b - 7 - off to 8 b + 7 - off.  Near are those that do not all lie from the last start on (without buckets of their own,
    // behind the query).
    const long off = Tk - Tq, last = starts[n - 1], behind = both && last > 1 ? last : 1;
    const long lo = (off - last - 7 >= 0 ? (off - last - 7) / 8 : -((last + 7 - off + 7) / 8)) + 1, hi = (behind + 7 + off + 7) / 8 - 1;
    const long rows = (Tq + 7) / 8, cols = (Tk + 7) / 8;
    const int near_lo = (int)(lo > -rows ? lo : -rows), near_hi = (int)(hi < cols ? hi : cols);
    const long d_lo = 8 * near_lo - 7 > 1 - Tq ? 8 * near_lo - 7 : 1 - Tq, d_hi = 8 * near_hi + 7 < Tk - 1 ? 8 * near_hi + 7 : Tk - 1;
    // a wave where it has a block for every lane at most (6 layers x 256 x 16 x 20 x 20: 18 us, four waves 28)
    const int threads = cols * steps <= 64 ? 64 : 256;
    const size_t lds = (2 * SUMS * threads + (size_t)(d_hi >= d_lo ? d_hi - d_lo + 1 : 0)) * sizeof(float);
    for (int l0 = 0; l0 < n_layers; l0 += REL_LAYERS) {
        RelLayers t{};
        t.n = n_layers - l0 < REL_LAYERS ? n_layers - l0 : REL_LAYERS;
        for (int l = 0; l < t.n; ++l) t.x[l] = dS[l0 + l];
        const dim3 grid((unsigned)(planes * splits));
        const int slot0 = l0 / REL_LAYERS * splits;
        auto launch = [&](auto kernel) {
            // (always the most that a launch can take, as contexts of several threads share the kernel; not a CU's 160 KiB, of which its static words are a part)
            if (lds > 65536) DP_HIP_CHECK(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)MOST_LDS));
            hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, ctx->stream, t, bk, lengths, causal, splits, near_lo, near_hi, B, H, Tq, Tk, part, slot0);
            return DP_OK;
        };
        dp_status st;
        if (dt == DP_BF16 && fold) st = threads == 64 ? launch(relbias_grads_kernel<true, true, 64>) : launch(relbias_grads_kernel<true, true, 256>);
        else if (dt == DP_BF16) st = threads == 64 ? launch(relbias_grads_kernel<true, false, 64>) : launch(relbias_grads_kernel<true, false, 256>);
        else if (fold) st = threads == 64 ? launch(relbias_grads_kernel<false, true, 64>) : launch(relbias_grads_kernel<false, true, 256>);
        else st = threads == 64 ? launch(relbias_grads_kernel<false, false, 64>) : launch(relbias_grads_kernel<false, false, 256>);
        if (st != DP_OK) return st;
        DP_LAUNCH_CHECK(ctx, "relbias_grads");
    }
    if (slots > 1) {
        const size_t blocks = (out + 15) / 16;
        if (blocks > 0x7FFFFFFF) {
            DP_SET_ERR(ctx, "B * H * buckets too large for one launch");
            return DP_ERR_SHAPE;
        }
        hipLaunchKernelGGL(relbias_join_kernel, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, part, slots, out, grads);
        DP_LAUNCH_CHECK(ctx, "relbias_join");
    }
    return DP_OK;
}
