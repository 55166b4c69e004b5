// C ABI entry points: argument checks, context management and dispatch to the kernel launchers.
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "dp_common.h"

namespace {

constexpr size_t DEFAULT_WORKSPACE = (size_t)512 << 20;
constexpr int CBUF_CAP = 1 << 20;
constexpr long MAX_ROWS = (long)INT_MAX - 4096;

#define REQUIRE_CTX(ctx) \
    if (!(ctx)) return DP_ERR_NULL

#define FAIL(ctx, code, ...)          \
    do {                              \
        DP_SET_ERR(ctx, __VA_ARGS__); \
        return code;                  \
    } while (0)

dp_status check_dtype(dp_ctx* ctx, dp_dtype dt) {
    if (dt != DP_F32 && dt != DP_BF16) FAIL(ctx, DP_ERR_DTYPE, "unknown dtype %d", (int)dt);
    return DP_OK;
}

dp_status check_tensor(dp_ctx* ctx, const char* name, const void* p, dp_dtype dt, int width) {
    if (!p) FAIL(ctx, DP_ERR_NULL, "%s is NULL", name);
    if (dt == DP_BF16) {
        if (width % 8) FAIL(ctx, DP_ERR_SHAPE, "%s: width %d is not a multiple of 8 (bf16)", name, width);
        if ((uintptr_t)p & 15) FAIL(ctx, DP_ERR_ALIGN, "%s is not 16-byte aligned (bf16)", name);
    } else if ((uintptr_t)p & 3) {
        FAIL(ctx, DP_ERR_ALIGN, "%s is not 4-byte aligned", name);
    }
    return DP_OK;
}

dp_status check_f32(dp_ctx* ctx, const char* name, const void* p) {
    if (!p) FAIL(ctx, DP_ERR_NULL, "%s is NULL", name);
    if ((uintptr_t)p & 3) FAIL(ctx, DP_ERR_ALIGN, "%s is not 4-byte aligned", name);
    return DP_OK;
}

dp_status check_bt(dp_ctx* ctx, int B, int T) {
    if (B < 0 || T < 0) FAIL(ctx, DP_ERR_SHAPE, "negative B or T");
    if ((long)B * T > MAX_ROWS) FAIL(ctx, DP_ERR_SHAPE, "B*T = %ld exceeds 2^31", (long)B * T);
    return DP_OK;
}

dp_status check_clip(dp_ctx* ctx, float C, int B) {
    if (!(C > 0.f) || !isfinite(C)) FAIL(ctx, DP_ERR_VALUE, "clip norm C must be positive and finite");
    if (B > ctx->cbuf_cap) FAIL(ctx, DP_ERR_WORKSPACE, "B = %d exceeds the clip-factor buffer (%d)", B, ctx->cbuf_cap);
    return DP_OK;
}

dp_status check_sum_width(dp_ctx* ctx, dp_dtype dt, int d_in, int d_out) {
    if (!dp_sum_width_ok(dt, d_in, d_out)) FAIL(ctx, DP_ERR_SHAPE, "a width above %d (bf16)", DP_BF16_MAX_WIDTH);
    return DP_OK;
}

#define TRY(expr)                    \
    do {                             \
        dp_status s__ = (expr);      \
        if (s__ != DP_OK) return s__; \
    } while (0)

// A range of memory, from its first byte to the one behind its last.
struct Span {
    uintptr_t from, to;
    bool output;
    bool meets(const Span& o) const { return from < o.to && o.from < to; }
};

Span block_span(const void* p, size_t bytes, bool output) { return {(uintptr_t)p, (uintptr_t)p + bytes, output}; }

// Whether one of n ranges that are written meets one that is read or (`apart`) another that is written.  in(l), out(l): range l (from == to: none).
// A flat buffer of outputs is seen through by one look at every range; ranges of outputs and inputs in any order are sorted.
template <typename In, typename Out>
dp_status spans_apart(dp_ctx* ctx, int n, const Span& also_read, In in, Out out, bool apart) {
    Span hull = {UINTPTR_MAX, 0, true};
    bool rising = true;
    for (int l = 0; l < n; ++l) {
        const Span o = out(l);
        if (o.from == o.to) continue;
        rising = rising && o.from >= hull.to;
        hull.from = o.from < hull.from ? o.from : hull.from;
        hull.to = o.to > hull.to ? o.to : hull.to;
    }
    if (hull.to == 0) return DP_OK;
    int within = also_read.meets(hull) ? 1 : 0;
    for (int l = 0; l < n; ++l) within += in(l).meets(hull) ? 1 : 0;
    if (within == 0 && (rising || !apart)) return DP_OK;
    Span* const s = (Span*)malloc((2 * (size_t)n + 1) * sizeof(Span));
    if (!s) FAIL(ctx, DP_ERR_HIP, "no host memory to compare the ranges of %d tensors", n);
    size_t m = 0;
    auto put = [&](const Span& x) {
        if (x.from != x.to) s[m++] = x;
    };
    put(also_read);
    for (int l = 0; l < n; ++l) {
        put(in(l));
        put(out(l));
    }
    std::sort(s, s + m, [](const Span& a, const Span& b) { return a.from < b.from; });
    uintptr_t read = 0, written = 0;  // ends of the ranges that begin before the next one
    bool meet = false;
    for (size_t k = 0; k < m && !meet; ++k) {
        meet = s[k].output ? read > s[k].from || (apart && written > s[k].from) : written > s[k].from;
        uintptr_t& end = s[k].output ? written : read;
        end = s[k].to > end ? s[k].to : end;
    }
    free(s);
    if (meet) FAIL(ctx, DP_ERR_VALUE, apart ? "an output overlaps an input, or another output" : "a sum overlaps an input");
    return DP_OK;
}

}  // namespace

extern "C" {

dp_status dp_create(dp_ctx** out, void* hip_stream, size_t workspace_bytes) {
    if (!out) return DP_ERR_NULL;
    dp_ctx* ctx = (dp_ctx*)calloc(1, sizeof(dp_ctx));
    if (!ctx) return DP_ERR_HIP;
    ctx->stream = (hipStream_t)hip_stream;
    ctx->ws_bytes = workspace_bytes ? workspace_bytes : DEFAULT_WORKSPACE;
    ctx->cbuf_cap = CBUF_CAP;
    ctx->prof = (dp_prof_rec*)calloc(DP_PROF_CAP, sizeof(dp_prof_rec));
    if (!ctx->prof) {
        free(ctx);
        return DP_ERR_HIP;
    }
    hipError_t e = hipGetDevice(&ctx->device);
    float* static_scratch = nullptr;  // looked up here so that dp_noise_adamw_snr_static finds it ready on this device
    if (e == hipSuccess && dpk_static_scratch(&static_scratch) != DP_OK) e = hipErrorInvalidSymbol;
    if (e == hipSuccess) e = hipMalloc((void**)&ctx->ws, ctx->ws_bytes);
    constexpr size_t WORDS = 256;  // the error word and, in a line of its own, the ticket
    if (e == hipSuccess) e = hipMalloc((void**)&ctx->err_word, WORDS);
    if (e == hipSuccess) e = hipMalloc((void**)&ctx->cbuf, (size_t)ctx->cbuf_cap * sizeof(float));
    if (e == hipSuccess) e = hipMemset(ctx->err_word, 0, WORDS);
    if (e == hipSuccess) ctx->ticket = (uint32_t*)ctx->err_word + 32;
    if (e != hipSuccess) {
        dp_forget_error();
        if (ctx->ws) (void)hipFree(ctx->ws);
        if (ctx->err_word) (void)hipFree(ctx->err_word);
        if (ctx->cbuf) (void)hipFree(ctx->cbuf);
        free(ctx->prof);
        free(ctx);
        return DP_ERR_HIP;
    }
    *out = ctx;
    return DP_OK;
}

dp_status dp_destroy(dp_ctx* ctx) {
    REQUIRE_CTX(ctx);
    (void)hipStreamSynchronize(ctx->stream);
    (void)hipFree(ctx->ws);
    (void)hipFree(ctx->err_word);
    (void)hipFree(ctx->cbuf);
    for (int i = 0; i < ctx->prof_made; ++i) {
        (void)hipEventDestroy(ctx->prof[i].start);
        (void)hipEventDestroy(ctx->prof[i].stop);
    }
    free(ctx->prof);
    free(ctx);
    return DP_OK;
}

dp_status dp_profile_enable(dp_ctx* ctx, int enable) {
    REQUIRE_CTX(ctx);
    DP_HIP_CHECK(ctx, hipStreamSynchronize(ctx->stream));
    ctx->prof_on = enable ? 1 : 0;
    ctx->prof_n = 0;
    return DP_OK;
}

dp_status dp_profile_read(dp_ctx* ctx, dp_prof_kind kind, double* ms_total, uint64_t* launches, double* work_total) {
    REQUIRE_CTX(ctx);
    if ((int)kind < 0 || (int)kind > (int)DP_PROF_ADAMW) FAIL(ctx, DP_ERR_DTYPE, "unknown profile kind %d", (int)kind);
    DP_HIP_CHECK(ctx, hipStreamSynchronize(ctx->stream));
    double ms = 0.0, work = 0.0;
    uint64_t cnt = 0;
    int keep = 0;
    for (int i = 0; i < ctx->prof_n; ++i) {
        dp_prof_rec r = ctx->prof[i];
        if (r.kind == (int)kind) {
            float t = 0.f;
            DP_HIP_CHECK(ctx, hipEventElapsedTime(&t, r.start, r.stop));
            ms += t;
            work += r.work;
            ++cnt;
        }
    }
    // compact: drop the records just read, keep the others (event objects are swapped, never leaked)
    for (int i = 0; i < ctx->prof_n; ++i) {
        if (ctx->prof[i].kind != (int)kind) {
            if (i != keep) {
                dp_prof_rec t = ctx->prof[keep];
                ctx->prof[keep] = ctx->prof[i];
                ctx->prof[i] = t;
            }
            ++keep;
        }
    }
    ctx->prof_n = keep;
    if (ms_total) *ms_total = ms;
    if (launches) *launches = cnt;
    if (work_total) *work_total = work;
    return DP_OK;
}

dp_status dp_profile_mfma_ceiling(dp_ctx* ctx, int iters, int launches, double* tflops) {
    REQUIRE_CTX(ctx);
    if (!tflops) FAIL(ctx, DP_ERR_NULL, "tflops is NULL");
    if (iters < 1 || iters > (1 << 20) || launches < 1 || launches > 1024) FAIL(ctx, DP_ERR_VALUE, "iters in [1, 2^20], launches in [1, 1024]");
    return dpk_mfma_ceiling(ctx, iters, launches, tflops);
}

dp_status dp_sync(dp_ctx* ctx) {
    REQUIRE_CTX(ctx);
    DP_HIP_CHECK(ctx, hipStreamSynchronize(ctx->stream));
    int w = 0;
    DP_HIP_CHECK(ctx, hipMemcpy(&w, ctx->err_word, sizeof(int), hipMemcpyDeviceToHost));
    if (w) {
        DP_HIP_CHECK(ctx, hipMemset(ctx->err_word, 0, sizeof(int)));
        if (w & DP_ERRBIT_INDEX) FAIL(ctx, DP_ERR_INDEX, "a token id outside [0, V), or a position outside its table, was met on the device");
        FAIL(ctx, DP_ERR_VALUE, "a per-example squared norm was NaN or overflowed fp32: the sums it entered hold NaN");
    }
    return DP_OK;
}

const char* dp_status_str(dp_status s) {
    switch (s) {
        case DP_OK: return "DP_OK";
        case DP_ERR_NULL: return "DP_ERR_NULL";
        case DP_ERR_SHAPE: return "DP_ERR_SHAPE";
        case DP_ERR_DTYPE: return "DP_ERR_DTYPE";
        case DP_ERR_ALIGN: return "DP_ERR_ALIGN";
        case DP_ERR_VALUE: return "DP_ERR_VALUE";
        case DP_ERR_INDEX: return "DP_ERR_INDEX";
        case DP_ERR_WORKSPACE: return "DP_ERR_WORKSPACE";
        case DP_ERR_HIP: return "DP_ERR_HIP";
    }
    return "DP_ERR_UNKNOWN";
}

const char* dp_last_error(const dp_ctx* ctx) { return ctx ? ctx->msg : "no context"; }

dp_status dp_gram_unit_plan(int T, uint32_t* units, int capacity, int* n_units) {
    if (!units || !n_units) return DP_ERR_NULL;
    if (capacity < 0) return DP_ERR_SHAPE;
    return dpk_gram_unit_plan(T, units, capacity, n_units);
}

dp_status dp_dense_sum_plan(dp_dtype dtype, int n_layers, int B, int T, int d_in, int d_out, size_t workspace_bytes, int32_t* plan) {
    if (!plan) return DP_ERR_NULL;
    if (dtype != DP_F32 && dtype != DP_BF16) return DP_ERR_DTYPE;
    if (n_layers < 1 || B < 1 || T < 1 || d_in < 1 || d_out < 1 || (long)B * T > MAX_ROWS) return DP_ERR_SHAPE;
    if (dtype == DP_BF16 && (d_in % 8 || d_out % 8)) return DP_ERR_SHAPE;
    if (!dp_sum_width_ok(dtype, d_in, d_out)) return DP_ERR_SHAPE;
    return dpk_dense_sum_plan(dtype, n_layers, B, T, d_in, d_out, workspace_bytes ? workspace_bytes : DEFAULT_WORKSPACE, plan);
}

dp_status dp_choose_path(int T, int d_in, int d_out, dp_dtype dtype, dp_path* out) {
    if (!out) return DP_ERR_NULL;
    if (dtype != DP_F32 && dtype != DP_BF16) return DP_ERR_DTYPE;
    if (T < 0 || d_in < 0 || d_out < 0) return DP_ERR_SHAPE;
    // flops of the symmetric Gram form, T(T+1)/2 * (d_in + d_out) multiply-adds per example, against those
    // of materialising the d_in x d_out gradient, T * d_in * d_out.
    const double gram = 0.5 * ((double)T + 1.0) * ((double)d_in + (double)d_out);
    const double mat = (double)d_in * (double)d_out;
    *out = gram <= mat ? DP_PATH_GRAM : DP_PATH_MATERIALISE;
    return DP_OK;
}

dp_status dp_batch_size_schedule(uint64_t step, uint64_t b_start, uint64_t b_end, uint64_t ramp_steps,
                                 uint32_t n_increments, uint64_t* out) {
    if (!out) return DP_ERR_NULL;
    if (step == 0 || n_increments == 0 || ramp_steps < n_increments || b_end < b_start) return DP_ERR_VALUE;
    // k jumps have happened once k/n_increments of the ramp's steps are complete (step t has t - 1 behind it)
    const unsigned __int128 done = (unsigned __int128)(step - 1) * n_increments;
    const uint64_t k = (uint64_t)(done / ramp_steps);
    *out = k >= n_increments ? b_end : b_start + k * ((b_end - b_start) / n_increments);
    return DP_OK;
}

dp_status dp_lr_schedule(uint64_t step, double peak, uint64_t warmup_steps, uint64_t total_steps, double* out) {
    if (!out) return DP_ERR_NULL;
    if (step == 0 || total_steps == 0 || total_steps < warmup_steps || !isfinite(peak)) return DP_ERR_VALUE;
    if (step <= warmup_steps) {
        *out = peak * (double)step / (double)warmup_steps;
    } else if (step >= total_steps) {
        *out = 0.0;
    } else {
        const double frac = (double)(total_steps - step) / (double)(total_steps - warmup_steps);
        *out = peak * frac * frac;
    }
    return DP_OK;
}

// ln of one term of the sampled-Gaussian moment sum; -inf for a vanishing factor
static double rdp_log_term(double q, double sigma, int alpha, int k) {
    const double lq = q > 0.0 ? log(q) : -INFINITY, l1q = q < 1.0 ? log1p(-q) : -INFINITY;
    double t = lgamma(alpha + 1.0) - lgamma(k + 1.0) - lgamma(alpha - k + 1.0);
    if (k > 0) t += k * lq;
    if (alpha - k > 0) t += (alpha - k) * l1q;
    return t + ((double)k * k - k) / (2.0 * sigma * sigma);
}

dp_status dp_rdp_sampled_gaussian(double q, double sigma, int alpha, double* out) {
    if (!out) return DP_ERR_NULL;
    if (!(q >= 0.0 && q <= 1.0) || !(sigma > 0.0) || !isfinite(sigma) || alpha < 2) return DP_ERR_VALUE;
    // log-sum-exp over the alpha + 1 terms
    double mx = -INFINITY;
    for (int k = 0; k <= alpha; ++k) mx = fmax(mx, rdp_log_term(q, sigma, alpha, k));
    double acc = 0.0;
    for (int k = 0; k <= alpha; ++k) acc += exp(rdp_log_term(q, sigma, alpha, k) - mx);
    *out = (mx + log(acc)) / (alpha - 1.0);
    return DP_OK;
}

dp_status dp_rdp_epsilon(const double* q, const uint64_t* steps, int n_phases, double sigma, double delta, int max_alpha,
                         double* eps, int* best_alpha) {
    if (!q || !steps || !eps) return DP_ERR_NULL;
    if (n_phases < 0 || !(delta > 0.0 && delta < 1.0) || max_alpha < 2) return DP_ERR_VALUE;
    double best = INFINITY;
    int arg = 0;
    for (int alpha = 2; alpha <= max_alpha; ++alpha) {
        double rdp = 0.0;
        for (int p = 0; p < n_phases; ++p) {
            double e;
            const dp_status st = dp_rdp_sampled_gaussian(q[p], sigma, alpha, &e);
            if (st != DP_OK) return st;
            rdp += (double)steps[p] * e;
        }
        const double cand = rdp + log(1.0 / delta) / (alpha - 1.0);
        if (cand < best) {
            best = cand;
            arg = alpha;
        }
    }
    *eps = best;
    if (best_alpha) *best_alpha = arg;
    return DP_OK;
}

dp_status dp_rdp_noise_multiplier(const double* q, const uint64_t* steps, int n_phases, double eps_target, double delta,
                                  int max_alpha, double rel_tol, double* sigma) {
    if (!sigma) return DP_ERR_NULL;
    if (!(eps_target > 0.0) || !(rel_tol > 0.0 && rel_tol < 1.0)) return DP_ERR_VALUE;
    // the guarantee shrinks as sigma grows: bracket the target from sigma = 1 by doubling / halving, then bisect
    double e, hi = 1.0;
    for (;;) {
        const dp_status st = dp_rdp_epsilon(q, steps, n_phases, hi, delta, max_alpha, &e, nullptr);
        if (st != DP_OK) return st;
        if (e <= eps_target) break;
        hi *= 2.0;
        if (hi > 1048576.0) return DP_ERR_VALUE;  // the conversion term of the largest order alone is above the target
    }
    double lo = hi / 2.0;
    for (;;) {
        const dp_status st = dp_rdp_epsilon(q, steps, n_phases, lo, delta, max_alpha, &e, nullptr);
        if (st != DP_OK) return st;
        if (e > eps_target) break;
        hi = lo;
        lo = lo / 2.0;
        if (lo < 1.0 / 1024.0) {  // no noise to speak of is needed (no steps, or nothing is ever sampled)
            *sigma = hi;
            return DP_OK;
        }
    }
    while (hi - lo > rel_tol * hi) {
        const double mid = 0.5 * (lo + hi);
        const dp_status st = dp_rdp_epsilon(q, steps, n_phases, mid, delta, max_alpha, &e, nullptr);
        if (st != DP_OK) return st;
        if (e <= eps_target) hi = mid;
        else lo = mid;
    }
    *sigma = hi;
    return DP_OK;
}

// DP_PATH_AUTO: fewer operations, or, where that leaves the chip idle, the path that fills it.
static dp_path choose_dense_path(const dp_ctx* ctx, int n, int B, int T, int d_in, int d_out, dp_dtype dtype) {
    dp_path path;
    dp_choose_path(T, d_in, d_out, dtype, &path);
    return path == DP_PATH_GRAM && dtype == DP_BF16 && dpk_materialise_sooner(ctx, n, B, T, d_in, d_out) ? DP_PATH_MATERIALISE : path;
}

dp_status dp_sqnorms_dense(dp_ctx* ctx, const void* A, const void* G, dp_dtype dtype, int B, int T, int d_in,
                           int d_out, int has_bias, dp_path path, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    if (path != DP_PATH_AUTO && path != DP_PATH_GRAM && path != DP_PATH_MATERIALISE)
        FAIL(ctx, DP_ERR_DTYPE, "unknown path %d", (int)path);
    TRY(check_bt(ctx, B, T));
    if (d_in < 0 || d_out < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer width");
    TRY(check_tensor(ctx, "A", A, dtype, d_in));
    TRY(check_tensor(ctx, "G", G, dtype, d_out));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    if (B == 0 || T == 0 || d_out == 0) return DP_OK;
    if (d_in == 0) {  // no weights; only the bias term is left
        if (has_bias) return dpk_colstat_sqnorms(ctx, nullptr, G, dtype, B, T, d_out, 0, 1, sqnorms);
        return DP_OK;
    }
    if (path == DP_PATH_AUTO) path = choose_dense_path(ctx, 1, B, T, d_in, d_out, dtype);
    if (path == DP_PATH_GRAM) return dpk_gram_sqnorms(ctx, A, G, dtype, B, T, d_in, d_out, has_bias, sqnorms);
    return dpk_materialise_sqnorms_batched(ctx, 1, &A, &G, dtype, B, T, d_in, d_out, has_bias, sqnorms);
}

dp_status dp_sqnorms_dense_batched(dp_ctx* ctx, int n_layers, const void* const* A, const void* const* G, dp_dtype dtype,
                                   int B, int T, int d_in, int d_out, int has_bias, dp_path path, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    if (path != DP_PATH_AUTO && path != DP_PATH_GRAM && path != DP_PATH_MATERIALISE)
        FAIL(ctx, DP_ERR_DTYPE, "unknown path %d", (int)path);
    TRY(check_bt(ctx, B, T));
    if (n_layers < 0 || d_in < 0 || d_out < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer count or width");
    if (n_layers == 0) return DP_OK;
    if (!A || !G) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_tensor(ctx, "A[l]", A[l], dtype, d_in));
        TRY(check_tensor(ctx, "G[l]", G[l], dtype, d_out));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    if (B == 0 || T == 0 || d_out == 0) return DP_OK;
    if (path == DP_PATH_AUTO && d_in > 0) path = choose_dense_path(ctx, n_layers, B, T, d_in, d_out, dtype);
    if (path == DP_PATH_GRAM && d_in > 0)
        return dpk_gram_sqnorms_batched(ctx, n_layers, A, G, dtype, B, T, d_in, d_out, has_bias, sqnorms);
    if (path == DP_PATH_MATERIALISE && d_in > 0)
        return dpk_materialise_sqnorms_batched(ctx, n_layers, A, G, dtype, B, T, d_in, d_out, has_bias, sqnorms);
    for (int l = 0; l < n_layers; ++l)
        TRY(dp_sqnorms_dense(ctx, A[l], G[l], dtype, B, T, d_in, d_out, has_bias, path, sqnorms));
    return DP_OK;
}

dp_status dp_sqnorms_dense_shared(dp_ctx* ctx, int n_groups, const void* const* A, int n_out, const void* const* G,
                                  dp_dtype dtype, int B, int T, int d_in, int d_out, int has_bias, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (n_groups < 0 || n_out < 1 || d_in < 0 || d_out < 0) FAIL(ctx, DP_ERR_SHAPE, "negative count or width");
    if (n_groups == 0) return DP_OK;
    if (!A || !G) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int g = 0; g < n_groups; ++g) {
        TRY(check_tensor(ctx, "A[g]", A[g], dtype, d_in));
        for (int j = 0; j < n_out; ++j) TRY(check_tensor(ctx, "G[g][j]", G[(size_t)g * n_out + j], dtype, d_out));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    if (B == 0 || T == 0 || d_out == 0) return DP_OK;
    dp_path path = DP_PATH_GRAM;
    if (d_in > 0) dp_choose_path(T, d_in, n_out * d_out, dtype, &path);  // one A A^T serves n_out output Grams
    if (d_in > 0 && path == DP_PATH_GRAM)
        return dpk_gram_sqnorms_shared(ctx, n_groups, A, n_out, G, dtype, B, T, d_in, d_out, has_bias, sqnorms);
    for (int g = 0; g < n_groups; ++g)
        for (int j = 0; j < n_out; ++j)
            TRY(dp_sqnorms_dense(ctx, A[g], G[(size_t)g * n_out + j], dtype, B, T, d_in, d_out, has_bias, DP_PATH_AUTO, sqnorms));
    return DP_OK;
}

dp_status dp_sqnorms_layernorm(dp_ctx* ctx, const void* Xhat, const void* G, dp_dtype dtype, int B, int T, int d,
                               float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative width");
    TRY(check_tensor(ctx, "Xhat", Xhat, dtype, d));
    TRY(check_tensor(ctx, "G", G, dtype, d));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    return dpk_colstat_sqnorms(ctx, Xhat, G, dtype, B, T, d, 1, 1, sqnorms);
}

dp_status dp_sqnorms_embedding(dp_ctx* ctx, const int32_t* ids, const void* G, dp_dtype dtype, int B, int T, int d,
                               int V, int distinct_per_example, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d < 0 || V <= 0) FAIL(ctx, DP_ERR_SHAPE, "width must be >= 0 and V > 0");
    TRY(check_f32(ctx, "ids", ids));
    TRY(check_tensor(ctx, "G", G, dtype, d));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    return dpk_embedding_sqnorms(ctx, ids, G, dtype, B, T, d, V, distinct_per_example, sqnorms);
}

dp_status dp_clip_factors(dp_ctx* ctx, const float* sqnorms, int B, float C, float* c) {
    REQUIRE_CTX(ctx);
    if (B < 0) FAIL(ctx, DP_ERR_SHAPE, "negative B");
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_f32(ctx, "c", c));
    if (!(C > 0.f) || !isfinite(C)) FAIL(ctx, DP_ERR_VALUE, "clip norm C must be positive and finite");
    if (B == 0) return DP_OK;
    return dpk_clip_factors(ctx, sqnorms, B, C, c);
}

// Tensors of held gradients; `out` may be NULL (a call without outputs).  SUMS: outputs are a unit's fp32 sums, which may share memory; otherwise of
// the inputs' size and type, each apart from all others or in place of its input.
enum HeldOut { HELD_NONE, HELD_SUMS, HELD_SCALED };
static dp_status check_grads(dp_ctx* ctx, int n, const void* const* X, const uint64_t* counts, dp_dtype dtype, int B, const float* sqnorms, const void* const* out,
                             HeldOut kind) {
    TRY(check_dtype(ctx, dtype));
    if (n < 0 || B < 0) FAIL(ctx, DP_ERR_SHAPE, "negative count");
    if (n > 0 && (!X || !counts)) FAIL(ctx, DP_ERR_NULL, "a table is NULL");
    if (B == 0) return DP_OK;  // (tensors of no elements have no address)
    const size_t elem = dtype == DP_BF16 ? 2 : 4, out_elem = kind == HELD_SUMS ? 4 : elem;
    for (int l = 0; l < n; ++l) {
        if (counts[l] == 0) continue;
        if (counts[l] > (B > 1 ? 1ull << 31 : 1ull << 59)) FAIL(ctx, DP_ERR_SHAPE, "counts[%d] is too large", l);
        if (!X[l]) FAIL(ctx, DP_ERR_NULL, "X[%d] is NULL", l);
        if ((uintptr_t)X[l] & (elem - 1)) FAIL(ctx, DP_ERR_ALIGN, "X[%d] is not aligned to its elements", l);
        if (kind == HELD_NONE) continue;
        if (!out[l]) FAIL(ctx, DP_ERR_NULL, "output %d is NULL", l);
        if ((uintptr_t)out[l] & (out_elem - 1)) FAIL(ctx, DP_ERR_ALIGN, "output %d is not aligned to its elements", l);
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    const Span norms = {(uintptr_t)sqnorms, (uintptr_t)(sqnorms + B), kind == HELD_NONE};
    auto in = [&](int l) -> Span { return {(uintptr_t)X[l], counts[l] ? (uintptr_t)X[l] + counts[l] * B * elem : (uintptr_t)X[l], false}; };
    if (kind == HELD_NONE) {
        for (int l = 0; l < n; ++l)
            if (counts[l] && in(l).meets(norms)) FAIL(ctx, DP_ERR_VALUE, "sqnorms overlaps X[%d]", l);
        return DP_OK;
    }
    if (kind == HELD_SUMS)
        return spans_apart(ctx, n, norms, in, [&](int l) -> Span { return {(uintptr_t)out[l], (uintptr_t)out[l] + counts[l] * 4, true}; }, false);
    // (in place: the output alone stands for both)
    return spans_apart(ctx, n, norms, [&](int l) -> Span { return X[l] == out[l] ? Span{0, 0, false} : in(l); },
                       [&](int l) -> Span { return {(uintptr_t)out[l], (uintptr_t)out[l] + counts[l] * B * elem, true}; }, true);
}

dp_status dp_sqnorms_grads(dp_ctx* ctx, int n_layers, const void* const* X, const uint64_t* counts, dp_dtype dtype, int B, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_grads(ctx, n_layers, X, counts, dtype, B, sqnorms, nullptr, HELD_NONE));
    if (B == 0 || n_layers == 0) return DP_OK;
    return dpk_held_sqnorms(ctx, n_layers, X, counts, dtype, B, sqnorms);
}

dp_status dp_clip_accumulate_grads(dp_ctx* ctx, int n_layers, const void* const* X, const uint64_t* counts, dp_dtype dtype, int B, float C,
                                   const float* sqnorms, float* const* sums) {
    REQUIRE_CTX(ctx);
    if (n_layers > 0 && !sums) FAIL(ctx, DP_ERR_NULL, "a table is NULL");
    TRY(check_grads(ctx, n_layers, X, counts, dtype, B, sqnorms, (const void* const*)sums, HELD_SUMS));
    TRY(check_clip(ctx, C, 0));
    if (B == 0 || n_layers == 0) return DP_OK;
    return dpk_held_sums(ctx, n_layers, X, counts, dtype, B, C, sqnorms, sums);
}

dp_status dp_clip_grads(dp_ctx* ctx, int n_layers, const void* const* X, const uint64_t* counts, dp_dtype dtype, int B, float C,
                        const float* sqnorms, void* const* Y) {
    REQUIRE_CTX(ctx);
    if (n_layers > 0 && !Y) FAIL(ctx, DP_ERR_NULL, "a table is NULL");
    TRY(check_grads(ctx, n_layers, X, counts, dtype, B, sqnorms, Y, HELD_SCALED));
    TRY(check_clip(ctx, C, 0));
    if (B == 0 || n_layers == 0) return DP_OK;
    return dpk_held_scale(ctx, n_layers, X, counts, dtype, B, C, sqnorms, Y);
}

// d^m e^j < r^j e^m for whole numbers, by comparing products of 32-bit words (at most 128 factors of 30 bits: 120 words).
static bool bucket_below(uint32_t d, uint32_t e, uint32_t r, int m, int j) {
    struct Product {
        uint32_t w[128] = {1};
        int n = 1;  // words in use
        void times(uint32_t f) {
            uint64_t carry = 0;
            for (int k = 0; k < n; ++k) {
                carry += (uint64_t)w[k] * f;
                w[k] = (uint32_t)carry;
                carry >>= 32;
            }
            if (carry && n < 128) w[n++] = (uint32_t)carry;
        }
    } a, b;
    for (int k = 0; k < m; ++k) {
        a.times(d);
        b.times(e);
    }
    for (int k = 0; k < j; ++k) {
        a.times(e);
        b.times(r);
    }
    if (a.n != b.n) return a.n < b.n;
    for (int k = a.n - 1; k >= 0; --k)
        if (a.w[k] != b.w[k]) return a.w[k] < b.w[k];
    return false;
}

dp_status dp_relative_buckets(int n, int max_distance, int32_t* starts) {
    if (!starts) return DP_ERR_NULL;
    if (n < 2 || n > DP_REL_MAX_SIDE || max_distance <= n / 2 || max_distance > (1 << 30)) return DP_ERR_VALUE;
    const int e = n / 2, m = n - e;
    for (int j = 0; j < e; ++j) starts[j] = j;
    for (int j = 0; j < m; ++j) {
        int lo = e, hi = max_distance;  // the first distance in [lo, hi] that is not below (at max_distance: 1 >= ..., j < m)
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (bucket_below((uint32_t)mid, (uint32_t)e, (uint32_t)max_distance, m, j)) lo = mid + 1;
            else hi = mid;
        }
        starts[e + j] = lo;
    }
    return DP_OK;
}

static dp_status check_relative(dp_ctx* ctx, int n, const int32_t* starts, dp_dtype dtype, int H, int Tq, int Tk) {
    TRY(check_dtype(ctx, dtype));
    if (!starts) FAIL(ctx, DP_ERR_NULL, "starts is NULL");
    if (n < 1 || n > DP_REL_MAX_SIDE) FAIL(ctx, DP_ERR_SHAPE, "%d buckets: 1 to %d of a side", n, DP_REL_MAX_SIDE);
    for (int j = 0; j < n; ++j)
        if (starts[j] < (j ? starts[j - 1] : 0) || starts[j] > (1 << 30) || (j == 0 && starts[0] != 0))
            FAIL(ctx, DP_ERR_VALUE, "starts[%d] = %d: they begin at 0, do not fall and do not exceed 2^30", j, starts[j]);
    if (H < 0 || Tq < 0 || Tk < Tq || Tk > (1 << 30)) FAIL(ctx, DP_ERR_SHAPE, "H = %d, Tq = %d, Tk = %d: 0 <= H, 0 <= Tq <= Tk <= 2^30", H, Tq, Tk);
    return DP_OK;
}

dp_status dp_relative_bias(dp_ctx* ctx, const float* table, int n, const int32_t* starts, int bidirectional, int H, int Tq, int Tk,
                           dp_dtype dtype, void* bias) {
    REQUIRE_CTX(ctx);
    TRY(check_relative(ctx, n, starts, dtype, H, Tq, Tk));
    if (H == 0 || Tq == 0) return DP_OK;
    TRY(check_f32(ctx, "table", table));
    if (!bias) FAIL(ctx, DP_ERR_NULL, "bias is NULL");
    const size_t e = dtype == DP_BF16 ? 2 : 4;
    if ((uintptr_t)bias & (e - 1)) FAIL(ctx, DP_ERR_ALIGN, "bias is not aligned to its elements");
    if (block_span(bias, (size_t)H * Tq * Tk * e, true).meets(block_span(table, (size_t)n * (bidirectional ? 2 : 1) * H * sizeof(float), false)))
        FAIL(ctx, DP_ERR_VALUE, "bias overlaps the table");
    return dpk_relbias(ctx, table, n, starts, bidirectional != 0, H, Tq, Tk, dtype, bias);
}

dp_status dp_relative_bias_grads(dp_ctx* ctx, int n_layers, const void* const* dS, dp_dtype dtype, const int32_t* lengths, int causal, int n,
                                 const int32_t* starts, int bidirectional, int B, int H, int Tq, int Tk, float* grads) {
    REQUIRE_CTX(ctx);
    TRY(check_relative(ctx, n, starts, dtype, H, Tq, Tk));
    if (n_layers < 0 || B < 0) FAIL(ctx, DP_ERR_SHAPE, "negative count");
    if (Tq + Tk - 1 > DP_REL_MAX_LINE) FAIL(ctx, DP_ERR_SHAPE, "Tq + Tk = %d exceeds %d", Tq + Tk, DP_REL_MAX_LINE + 1);
    if (B == 0 || H == 0) return DP_OK;
    TRY(check_f32(ctx, "grads", grads));
    const uint64_t out = (uint64_t)B * H * n * (bidirectional ? 2 : 1);
    if (n_layers == 0 || Tq == 0) return dpk_zero_f32(ctx, grads, out);
    if (!dS) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    const size_t e = dtype == DP_BF16 ? 2 : 4;
    for (int l = 0; l < n_layers; ++l) {
        if (!dS[l]) FAIL(ctx, DP_ERR_NULL, "dS[%d] is NULL", l);
        if ((uintptr_t)dS[l] & (e - 1)) FAIL(ctx, DP_ERR_ALIGN, "dS[%d] is not aligned to its elements", l);
    }
    if (lengths) TRY(check_f32(ctx, "lengths", lengths));
    const Span written = block_span(grads, out * sizeof(float), true);
    for (int l = 0; l < n_layers; ++l)
        if (written.meets(block_span(dS[l], (size_t)B * H * Tq * Tk * e, false))) FAIL(ctx, DP_ERR_VALUE, "grads overlaps dS[%d]", l);
    if (lengths && written.meets(block_span(lengths, (size_t)B * sizeof(int32_t), false))) FAIL(ctx, DP_ERR_VALUE, "grads overlaps lengths");
    return dpk_relbias_grads(ctx, n_layers, dS, dtype, lengths, causal != 0, n, starts, bidirectional != 0, B, H, Tq, Tk, grads);
}

static dp_status check_qk(dp_ctx* ctx, const dp_qk_args& a) {
    TRY(check_dtype(ctx, a.dtype));
    TRY(check_bt(ctx, a.B, a.T));
    if (a.Hq < 0 || a.Hk < 0 || (long)a.Hq + a.Hk > (1 << 20)) FAIL(ctx, DP_ERR_SHAPE, "Hq = %d, Hk = %d: 0 to 2^20 heads", a.Hq, a.Hk);
    if (a.D < 8 || a.D > 512 || a.D % 8) FAIL(ctx, DP_ERR_SHAPE, "D = %d: a multiple of 8 in [8, 512]", a.D);
    if (a.R < 0 || a.R > a.D || a.R % 8) FAIL(ctx, DP_ERR_SHAPE, "R = %d: a multiple of 8 in [0, D]", a.R);
    if (!(a.eps >= FLT_MIN) || !isfinite(a.eps)) FAIL(ctx, DP_ERR_VALUE, "eps must be a positive normal number");
    const uintptr_t low = a.dtype == DP_BF16 ? 1 : 3;
    for (int s = 0; s < 2; ++s) {
        const int H = s ? a.Hk : a.Hq;
        const void* x = s ? a.k : a.q;
        const int64_t ld = s ? a.ldk : a.ldq;
        if (H == 0 || a.B == 0 || a.T == 0) continue;
        if (!x) FAIL(ctx, DP_ERR_NULL, "%s is NULL", s ? "k" : "q");
        if ((uintptr_t)x & low) FAIL(ctx, DP_ERR_ALIGN, "%s is not aligned to its elements", s ? "k" : "q");
        if (ld < (int64_t)H * a.D || ld > (1ll << 32)) FAIL(ctx, DP_ERR_SHAPE, "%s: tokens %lld numbers apart, %lld are needed", s ? "ldk" : "ldq", (long long)ld, (long long)H * a.D);
        TRY(check_f32(ctx, s ? "gain_k" : "gain_q", s ? a.gain_k : a.gain_q));
    }
    if (a.n_pos < 0 || (a.R > 0 && a.n_pos == 0 && a.B > 0 && a.T > 0)) FAIL(ctx, DP_ERR_SHAPE, "n_pos = %d: a table of positions is needed", a.n_pos);
    if (a.R > 0 && a.n_pos > 0) {
        TRY(check_f32(ctx, "cos", a.cos));
        TRY(check_f32(ctx, "sin", a.sin));
    }
    if (a.R > 0 && a.positions) TRY(check_f32(ctx, "positions", a.positions));
    return DP_OK;
}

// The range of memory that `tokens` tokens of `width` numbers lie in, `ld` numbers apart.
static Span tokens_span(const void* p, long tokens, int64_t ld, long width, size_t elem, bool output) {
    return {(uintptr_t)p, (uintptr_t)p + ((size_t)(tokens - 1) * ld + width) * elem, output};
}

// Outputs of heads (of the queries, of the keys; ldq, ldk numbers from token to token) and `grads`, if there are any: aligned, and apart from each other
// and from what is read.
static dp_status check_qk_out(dp_ctx* ctx, const dp_qk_args& a, const char* const names[2], const void* const y[2], const int64_t ld[2], const void* dyq, const void* dyk,
                              const float* grads) {
    const size_t e = a.dtype == DP_BF16 ? 2 : 4;
    const long n = (long)a.B * a.T, w[2] = {(long)a.Hq * a.D, (long)a.Hk * a.D};
    auto block = [](const void* p, size_t bytes) { return block_span(p, bytes, false); };
    Span read[9], out[3];
    int n_read = 0, n_out = 0;
    if (w[0]) read[n_read++] = tokens_span(a.q, n, a.ldq, w[0], e, false);
    if (w[1]) read[n_read++] = tokens_span(a.k, n, a.ldk, w[1], e, false);
    if (w[0] && dyq) read[n_read++] = tokens_span(dyq, n, w[0], w[0], e, false);
    if (w[1] && dyk) read[n_read++] = tokens_span(dyk, n, w[1], w[1], e, false);
    if (w[0]) read[n_read++] = block(a.gain_q, a.D * sizeof(float));
    if (w[1]) read[n_read++] = block(a.gain_k, a.D * sizeof(float));
    if (a.R) read[n_read++] = block(a.cos, (size_t)a.n_pos * (a.R / 2) * sizeof(float));
    if (a.R) read[n_read++] = block(a.sin, (size_t)a.n_pos * (a.R / 2) * sizeof(float));
    if (a.R && a.positions) read[n_read++] = block(a.positions, n * sizeof(int32_t));
    int heads[2];  // place of y[s] in out
    for (int s = 0; s < 2; ++s) {
        heads[s] = -1;
        if (!y || !w[s]) continue;
        if (!y[s]) FAIL(ctx, DP_ERR_NULL, "%s is NULL", names[s]);
        if ((uintptr_t)y[s] & (e - 1)) FAIL(ctx, DP_ERR_ALIGN, "%s is not aligned to its elements", names[s]);
        heads[s] = n_out;
        out[n_out++] = tokens_span(y[s], n, ld[s], w[s], e, true);
    }
    if (grads) out[n_out++] = block(grads, (size_t)a.B * 2 * a.D * sizeof(float));
    for (int i = 0; i < n_out; ++i) {
        const char* name = i == heads[0] ? names[0] : i == heads[1] ? names[1] : "grads";
        for (int j = 0; j < n_read; ++j)
            if (out[i].meets(read[j])) FAIL(ctx, DP_ERR_VALUE, "%s overlaps an input", name);
        for (int j = 0; j < i; ++j) {
            if (!out[i].meets(out[j])) continue;
            if (i == heads[1] && j == heads[0] && ld[0] == ld[1]) {  // other columns of the same rows
                const int low = (uintptr_t)y[0] <= (uintptr_t)y[1] ? 0 : 1;
                const int64_t column = (int64_t)(((uintptr_t)y[1 - low] - (uintptr_t)y[low]) / e) % ld[0];
                if (column >= w[low] && column + w[1 - low] <= ld[0]) continue;
            }
            FAIL(ctx, DP_ERR_VALUE, "%s overlaps another output", name);
        }
    }
    return DP_OK;
}

dp_status dp_qk_norm(dp_ctx* ctx, const void* q, const void* k, dp_dtype dtype, int64_t ldq, int64_t ldk, const float* gain_q,
                     const float* gain_k, const float* cos, const float* sin, int n_pos, const int32_t* positions, int interleaved, int B,
                     int T, int Hq, int Hk, int D, int R, float eps, void* yq, void* yk) {
    REQUIRE_CTX(ctx);
    const dp_qk_args a = {q, k, dtype, ldq, ldk, gain_q, gain_k, cos, sin, n_pos, positions, interleaved != 0, B, T, Hq, Hk, D, R, eps};
    TRY(check_qk(ctx, a));
    if (B == 0 || T == 0 || Hq + Hk == 0) return DP_OK;
    const char* const names[2] = {"yq", "yk"};
    const void* const y[2] = {yq, yk};
    const int64_t ld[2] = {(int64_t)Hq * D, (int64_t)Hk * D};
    TRY(check_qk_out(ctx, a, names, y, ld, nullptr, nullptr, nullptr));
    return dpk_qk_norm(ctx, a, yq, yk);
}

dp_status dp_qk_norm_grads(dp_ctx* ctx, const void* q, const void* k, dp_dtype dtype, int64_t ldq, int64_t ldk, const float* gain_q,
                           const float* gain_k, const float* cos, const float* sin, int n_pos, const int32_t* positions, int interleaved,
                           int B, int T, int Hq, int Hk, int D, int R, float eps, const void* dyq, const void* dyk, float* grads, void* dq,
                           void* dk) {
    REQUIRE_CTX(ctx);
    const dp_qk_args a = {q, k, dtype, ldq, ldk, gain_q, gain_k, cos, sin, n_pos, positions, interleaved != 0, B, T, Hq, Hk, D, R, eps};
    TRY(check_qk(ctx, a));
    if (B == 0) return DP_OK;
    TRY(check_f32(ctx, "grads", grads));
    if (T == 0 || Hq + Hk == 0) return dpk_zero_f32(ctx, grads, (uint64_t)B * 2 * D);
    const uintptr_t low = dtype == DP_BF16 ? 1 : 3;
    if ((Hq && !dyq) || (Hk && !dyk)) FAIL(ctx, DP_ERR_NULL, "dyq or dyk is NULL");
    if ((Hq && ((uintptr_t)dyq & low)) || (Hk && ((uintptr_t)dyk & low))) FAIL(ctx, DP_ERR_ALIGN, "dyq or dyk is not aligned to its elements");
    const bool wanted = (Hq && dq) || (Hk && dk);
    const char* const names[2] = {"dq", "dk"};
    const void* const y[2] = {dq, dk};
    const int64_t ld[2] = {ldq, ldk};
    TRY(check_qk_out(ctx, a, names, wanted ? y : nullptr, ld, dyq, dyk, grads));
    return dpk_qk_norm_grads(ctx, a, dyq, dyk, grads, dq, dk, wanted);
}

dp_status dp_clip_accumulate_dense(dp_ctx* ctx, const void* A, const void* G, dp_dtype dtype, int B, int T, int d_in,
                                   int d_out, float C, const float* sqnorms, float* sum_W, float* sum_b) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d_in < 0 || d_out < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer width");
    TRY(check_tensor(ctx, "A", A, dtype, d_in));
    TRY(check_tensor(ctx, "G", G, dtype, d_out));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_f32(ctx, "sum_W", sum_W));
    if (sum_b) TRY(check_f32(ctx, "sum_b", sum_b));
    if (dtype == DP_BF16 && ((uintptr_t)sum_W & 15)) FAIL(ctx, DP_ERR_ALIGN, "sum_W is not 16-byte aligned");
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d_out == 0) return DP_OK;
    TRY(check_sum_width(ctx, dtype, d_in, d_out));
    return dpk_weighted_gemm(ctx, A, G, dtype, B, T, d_in, d_out, sqnorms, C, sum_W, sum_b);
}

dp_status dp_clip_accumulate_dense_batched(dp_ctx* ctx, int n_layers, const void* const* A, const void* const* G,
                                           dp_dtype dtype, int B, int T, int d_in, int d_out, float C,
                                           const float* sqnorms, float* const* sum_W, float* const* sum_b) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (n_layers < 0 || d_in < 0 || d_out < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer count or width");
    if (n_layers == 0) return DP_OK;
    if (!A || !G || !sum_W) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_tensor(ctx, "A[l]", A[l], dtype, d_in));
        TRY(check_tensor(ctx, "G[l]", G[l], dtype, d_out));
        TRY(check_f32(ctx, "sum_W[l]", sum_W[l]));
        if (dtype == DP_BF16 && ((uintptr_t)sum_W[l] & 15)) FAIL(ctx, DP_ERR_ALIGN, "sum_W[%d] is not 16-byte aligned", l);
        if (sum_b && sum_b[l]) TRY(check_f32(ctx, "sum_b[l]", sum_b[l]));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d_out == 0) return DP_OK;
    TRY(check_sum_width(ctx, dtype, d_in, d_out));
    return dpk_weighted_gemm_batched(ctx, n_layers, A, G, dtype, B, T, d_in, d_out, sqnorms, C, sum_W, sum_b);
}

dp_status dp_clip_accumulate_layernorm(dp_ctx* ctx, const void* Xhat, const void* G, dp_dtype dtype, int B, int T,
                                       int d, float C, const float* sqnorms, float* sum_gamma, float* sum_beta) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative width");
    TRY(check_tensor(ctx, "Xhat", Xhat, dtype, d));
    TRY(check_tensor(ctx, "G", G, dtype, d));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_f32(ctx, "sum_gamma", sum_gamma));
    TRY(check_f32(ctx, "sum_beta", sum_beta));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d == 0) return DP_OK;
    return dpk_colstat_sums(ctx, Xhat, G, dtype, B, T, d, sqnorms, C, sum_gamma, sum_beta);
}

dp_status dp_sqnorms_layernorm_batched(dp_ctx* ctx, int n_layers, const void* const* Xhat, const void* const* G,
                                       dp_dtype dtype, int B, int T, int d, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (n_layers < 0 || d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer count or width");
    if (n_layers == 0) return DP_OK;
    if (!Xhat || !G) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_tensor(ctx, "Xhat[l]", Xhat[l], dtype, d));
        TRY(check_tensor(ctx, "G[l]", G[l], dtype, d));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    return dpk_colstat_sqnorms_batched(ctx, n_layers, Xhat, G, dtype, B, T, d, 1, 1, sqnorms, nullptr);
}

dp_status dp_sqnorms_layernorm_keep(dp_ctx* ctx, int n_layers, const void* const* Xhat, const void* const* G, dp_dtype dtype,
                                    int B, int T, int d, float* sqnorms, float* const* grads) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (n_layers < 0 || d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer count or width");
    if (d % 4) FAIL(ctx, DP_ERR_SHAPE, "width %d is not a multiple of 4", d);
    if (n_layers == 0) return DP_OK;
    if (!Xhat || !G || !grads) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_tensor(ctx, "Xhat[l]", Xhat[l], dtype, d));
        TRY(check_tensor(ctx, "G[l]", G[l], dtype, d));
        TRY(check_f32(ctx, "grads[l]", grads[l]));
        if ((uintptr_t)grads[l] & 15) FAIL(ctx, DP_ERR_ALIGN, "grads[%d] is not 16-byte aligned", l);
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    if (B == 0 || d == 0) return DP_OK;
    if (T == 0) {  // no tokens: every example's gradient is zero
        for (int l = 0; l < n_layers; ++l) TRY(dpk_zero_f32(ctx, grads[l], (uint64_t)B * 2 * d));
        return DP_OK;
    }
    return dpk_colstat_sqnorms_batched(ctx, n_layers, Xhat, G, dtype, B, T, d, 1, 1, sqnorms, grads);
}

dp_status dp_clip_accumulate_layernorm_kept(dp_ctx* ctx, int n_layers, float* const* grads, int B, int d, float C,
                                            const float* sqnorms, float* const* sum_gamma, float* const* sum_beta) {
    REQUIRE_CTX(ctx);
    if (B < 0 || n_layers < 0 || d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative count or width");
    if (d % 4) FAIL(ctx, DP_ERR_SHAPE, "width %d is not a multiple of 4", d);
    if (n_layers == 0) return DP_OK;
    if (!grads || !sum_gamma || !sum_beta) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_f32(ctx, "grads[l]", grads[l]));
        TRY(check_f32(ctx, "sum_gamma[l]", sum_gamma[l]));
        TRY(check_f32(ctx, "sum_beta[l]", sum_beta[l]));
        if (((uintptr_t)grads[l] | (uintptr_t)sum_gamma[l] | (uintptr_t)sum_beta[l]) & 15)
            FAIL(ctx, DP_ERR_ALIGN, "grads, sum_gamma and sum_beta must be 16-byte aligned (layer %d)", l);
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || d == 0) return DP_OK;
    return dpk_kept_sums_batched(ctx, n_layers, grads, B, d, sqnorms, C, sum_gamma, sum_beta);
}

dp_status dp_clip_accumulate_layernorm_batched(dp_ctx* ctx, int n_layers, const void* const* Xhat, const void* const* G,
                                               dp_dtype dtype, int B, int T, int d, float C, const float* sqnorms,
                                               float* const* sum_gamma, float* const* sum_beta) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (n_layers < 0 || d < 0) FAIL(ctx, DP_ERR_SHAPE, "negative layer count or width");
    if (n_layers == 0) return DP_OK;
    if (!Xhat || !G || !sum_gamma || !sum_beta) FAIL(ctx, DP_ERR_NULL, "a pointer table is NULL");
    for (int l = 0; l < n_layers; ++l) {
        TRY(check_tensor(ctx, "Xhat[l]", Xhat[l], dtype, d));
        TRY(check_tensor(ctx, "G[l]", G[l], dtype, d));
        TRY(check_f32(ctx, "sum_gamma[l]", sum_gamma[l]));
        TRY(check_f32(ctx, "sum_beta[l]", sum_beta[l]));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d == 0) return DP_OK;
    return dpk_colstat_sums_batched(ctx, n_layers, Xhat, G, dtype, B, T, d, sqnorms, C, sum_gamma, sum_beta);
}

dp_status dp_clip_accumulate_embedding(dp_ctx* ctx, const int32_t* ids, const void* G, dp_dtype dtype, int B, int T,
                                       int d, int V, float C, const float* sqnorms, float* sum_E) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d < 0 || V <= 0) FAIL(ctx, DP_ERR_SHAPE, "width must be >= 0 and V > 0");
    TRY(check_f32(ctx, "ids", ids));
    TRY(check_tensor(ctx, "G", G, dtype, d));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_f32(ctx, "sum_E", sum_E));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d == 0) return DP_OK;
    return dpk_embedding_sums(ctx, ids, G, dtype, B, T, d, V, sqnorms, C, sum_E);
}

dp_status dp_clip_accumulate_positions(dp_ctx* ctx, const void* G, dp_dtype dtype, int B, int T, int d, float C,
                                       const float* sqnorms, float* sum_E) {
    REQUIRE_CTX(ctx);
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    if (d < 0) FAIL(ctx, DP_ERR_SHAPE, "width must be >= 0");
    TRY(check_tensor(ctx, "G", G, dtype, d));
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    TRY(check_f32(ctx, "sum_E", sum_E));
    TRY(check_clip(ctx, C, B));
    if (B == 0 || T == 0 || d == 0) return DP_OK;
    if ((long)T * d > 0x7FFFFFFFl) FAIL(ctx, DP_ERR_SHAPE, "T * d too large");
    // token t of every example adds to row t: the first T rows of the table, read as one vector of T*d entries,
    // receive sum_i c_i * (example i's gradient read as one row of T*d entries): a weighted column sum over B rows
    return dpk_colstat_sums(ctx, nullptr, G, dtype, B, 1, T * d, sqnorms, C, nullptr, sum_E);
}

static dp_status check_tied(dp_ctx* ctx, const int32_t* ids, const void* dY, const void* H, const void* dL,
                            dp_dtype dtype, int B, int T, int M, int d, int V, const float* sqnorms) {
    TRY(check_dtype(ctx, dtype));
    TRY(check_bt(ctx, B, T));
    TRY(check_bt(ctx, B, M));
    if (d < 0 || V <= 0) FAIL(ctx, DP_ERR_SHAPE, "width must be >= 0 and V > 0");
    if ((long)M * V > (long)INT_MAX) FAIL(ctx, DP_ERR_SHAPE, "M * V = %ld exceeds 2^31", (long)M * V);
    TRY(check_f32(ctx, "ids", ids));
    TRY(check_tensor(ctx, "dY", dY, dtype, d));
    if (M > 0) {
        TRY(check_tensor(ctx, "H", H, dtype, d));
        TRY(check_tensor(ctx, "dL", dL, dtype, V));
    }
    TRY(check_f32(ctx, "sqnorms", sqnorms));
    return DP_OK;
}

dp_status dp_sqnorms_tied_embedding(dp_ctx* ctx, const int32_t* ids, const void* dY, const void* H, const void* dL,
                                    dp_dtype dtype, int B, int T, int M, int d, int V, float* sqnorms) {
    REQUIRE_CTX(ctx);
    TRY(check_tied(ctx, ids, dY, H, dL, dtype, B, T, M, d, V, sqnorms));
    if (B == 0 || d == 0) return DP_OK;
    if (T > 0) TRY(dpk_embedding_sqnorms(ctx, ids, dY, dtype, B, T, d, V, 0, sqnorms));
    if (M == 0) return DP_OK;
    // the output projection as a dense layer with weight E: "input" dL_i [M, V], "output gradient" H_i [M, d];
    // M is far below both widths, so the Gram form <dL dL^T, H H^T> is the cheap one, if not always the quick one
    if (dtype == DP_BF16 && dpk_materialise_sooner(ctx, 1, B, M, V, d)) TRY(dpk_materialise_sqnorms_batched(ctx, 1, &dL, &H, dtype, B, M, V, d, 0, sqnorms));
    else TRY(dpk_gram_sqnorms(ctx, dL, H, dtype, B, M, V, d, 0, sqnorms));
    return dpk_tied_cross_sqnorms(ctx, ids, dY, H, dL, dtype, B, T, M, d, V, sqnorms);
}

dp_status dp_clip_accumulate_tied_embedding(dp_ctx* ctx, const int32_t* ids, const void* dY, const void* H,
                                            const void* dL, dp_dtype dtype, int B, int T, int M, int d, int V, float C,
                                            const float* sqnorms, float* sum_E) {
    REQUIRE_CTX(ctx);
    TRY(check_tied(ctx, ids, dY, H, dL, dtype, B, T, M, d, V, sqnorms));
    TRY(check_f32(ctx, "sum_E", sum_E));
    if (dtype == DP_BF16 && ((uintptr_t)sum_E & 15)) FAIL(ctx, DP_ERR_ALIGN, "sum_E is not 16-byte aligned");
    TRY(check_clip(ctx, C, B));
    if (B == 0 || d == 0) return DP_OK;
    if (M > 0) TRY(check_sum_width(ctx, dtype, V, d));  // before anything is added to sum_E
    if (T > 0) TRY(dpk_embedding_sums(ctx, ids, dY, dtype, B, T, d, V, sqnorms, C, sum_E));
    if (M == 0) return DP_OK;
    // the output projection's sum is a dense sum with input dL [B, M, V] and output gradient H [B, M, d]
    return dpk_weighted_gemm(ctx, dL, H, dtype, B, M, V, d, sqnorms, C, sum_E, nullptr);
}

// Argument checks of the update; *why is set to a static text on failure.
static dp_status check_update_args(const float* params, const float* m, const float* v, const float* sum, uint64_t n,
                                   uint64_t elem_offset, float sigma, float C, uint64_t step, uint64_t batch_size, float lr,
                                   float beta1, float beta2, float eps, float weight_decay, const char** why) {
#define UPD_FAIL(code, text) \
    do {                     \
        *why = text;         \
        return code;         \
    } while (0)
    if (!params || !m || !v || !sum) UPD_FAIL(DP_ERR_NULL, "params, m, v or sum is NULL");
    if (((uintptr_t)params | (uintptr_t)m | (uintptr_t)v | (uintptr_t)sum) & 3) UPD_FAIL(DP_ERR_ALIGN, "params, m, v and sum must be 4-byte aligned");
    if (!(sigma >= 0.f) || !isfinite(sigma)) UPD_FAIL(DP_ERR_VALUE, "sigma must be >= 0 and finite");
    if (!(C > 0.f) || !isfinite(C)) UPD_FAIL(DP_ERR_VALUE, "clip norm C must be positive and finite");
    if (batch_size == 0) UPD_FAIL(DP_ERR_VALUE, "batch_size must be positive");
    if (step == 0) UPD_FAIL(DP_ERR_VALUE, "step counts from 1");
    if (!(beta1 >= 0.f && beta1 < 1.f) || !(beta2 >= 0.f && beta2 < 1.f)) UPD_FAIL(DP_ERR_VALUE, "beta outside [0, 1)");
    if (!(eps >= 0.f) || !isfinite(eps)) UPD_FAIL(DP_ERR_VALUE, "eps must be >= 0 and finite");
    if (!isfinite(lr) || !isfinite(weight_decay)) UPD_FAIL(DP_ERR_VALUE, "lr and weight_decay must be finite");
    if (elem_offset + n < elem_offset) UPD_FAIL(DP_ERR_SHAPE, "elem_offset + n overflows");
#undef UPD_FAIL
    return DP_OK;
}

static dp_status noise_adamw_checked(dp_ctx* ctx, float* params, float* m, float* v, float* sum, uint64_t n,
                                     uint64_t elem_offset, float sigma, float C, uint64_t seed, uint64_t step,
                                     uint64_t batch_size, float lr, float beta1, float beta2, float eps,
                                     float weight_decay, int zero_sum, float* sq_out) {
    const char* why = "";
    const dp_status st = check_update_args(params, m, v, sum, n, elem_offset, sigma, C, step, batch_size, lr, beta1, beta2,
                                           eps, weight_decay, &why);
    if (st != DP_OK) FAIL(ctx, st, "%s", why);
    return dpk_noise_adamw(ctx, params, m, v, sum, n, elem_offset, sigma, C, seed, step, batch_size, lr, beta1, beta2,
                           eps, weight_decay, zero_sum, sq_out);
}

dp_status dp_noise_adamw(dp_ctx* ctx, float* params, float* m, float* v, float* sum, uint64_t n,
                         uint64_t elem_offset, float sigma, float C, uint64_t seed, uint64_t step,
                         uint64_t batch_size, float lr, float beta1, float beta2, float eps, float weight_decay,
                         int zero_sum) {
    REQUIRE_CTX(ctx);
    return noise_adamw_checked(ctx, params, m, v, sum, n, elem_offset, sigma, C, seed, step, batch_size, lr, beta1,
                               beta2, eps, weight_decay, zero_sum, nullptr);
}

dp_status dp_noise_adamw_snr(dp_ctx* ctx, float* params, float* m, float* v, float* sum, uint64_t n,
                             uint64_t elem_offset, float sigma, float C, uint64_t seed, uint64_t step,
                             uint64_t batch_size, float lr, float beta1, float beta2, float eps, float weight_decay,
                             int zero_sum, float* snr_sq) {
    REQUIRE_CTX(ctx);
    if (!snr_sq) FAIL(ctx, DP_ERR_NULL, "snr_sq is NULL");
    if ((uintptr_t)snr_sq & 3) FAIL(ctx, DP_ERR_ALIGN, "snr_sq must be 4-byte aligned");
    return noise_adamw_checked(ctx, params, m, v, sum, n, elem_offset, sigma, C, seed, step, batch_size, lr, beta1,
                               beta2, eps, weight_decay, zero_sum, snr_sq);
}

dp_status dp_noise_adamw_snr_static(void* hip_stream, float* params, float* m, float* v, float* sum, uint64_t n,
                                    uint64_t elem_offset, float sigma, float C, uint64_t seed, uint64_t step,
                                    uint64_t batch_size, float lr, float beta1, float beta2, float eps, float weight_decay,
                                    int zero_sum, float* snr_sq) {
    if (!snr_sq) return DP_ERR_NULL;
    if ((uintptr_t)snr_sq & 3) return DP_ERR_ALIGN;
    const char* why = "";
    const dp_status st = check_update_args(params, m, v, sum, n, elem_offset, sigma, C, step, batch_size, lr, beta1, beta2,
                                           eps, weight_decay, &why);
    if (st != DP_OK) return st;
    return dpk_noise_adamw_snr_static((hipStream_t)hip_stream, params, m, v, sum, n, elem_offset, sigma, C, seed, step,
                                      batch_size, lr, beta1, beta2, eps, weight_decay, zero_sum, snr_sq);
}

dp_status dp_zero_f32(dp_ctx* ctx, float* p, uint64_t n) {
    REQUIRE_CTX(ctx);
    TRY(check_f32(ctx, "p", p));
    return dpk_zero_f32(ctx, p, n);
}

dp_status dp_philox_u32(dp_ctx* ctx, uint32_t* out, uint64_t n, uint64_t elem_offset, uint64_t seed, uint64_t step) {
    REQUIRE_CTX(ctx);
    TRY(check_f32(ctx, "out", out));
    if (elem_offset + n < elem_offset) FAIL(ctx, DP_ERR_SHAPE, "elem_offset + n overflows");
    return dpk_philox_u32(ctx, out, n, elem_offset, seed, step);
}

dp_status dp_normal_f32(dp_ctx* ctx, float* out, uint64_t n, uint64_t elem_offset, uint64_t seed, uint64_t step) {
    REQUIRE_CTX(ctx);
    TRY(check_f32(ctx, "out", out));
    if (elem_offset + n < elem_offset) FAIL(ctx, DP_ERR_SHAPE, "elem_offset + n overflows");
    return dpk_normal_f32(ctx, out, n, elem_offset, seed, step);
}

}  // extern "C"
