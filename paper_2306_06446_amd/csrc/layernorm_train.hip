// LayerNorm of training (Eq. 2) with its statistics and the router's logits, and its gradient with the residual's and the router's.
//
//   xh = (x - mean) rstd,  y = xh gamma + beta,  logits = y wg + bg
//   h = dy + dlogits wg^T,  g = h gamma,  dx = dres + rstd (g - <g> - xh <g xh>),  <.> the mean over the row
//   dgamma = sum_t h xh,  dbeta = sum_t h,  dwg = sum_t y dlogits,  dbg = sum_t dlogits
#include "common.h"
#include "layernorm.h"
#include "row_types.h"

namespace {

using namespace sa;

constexpr int kThreads = 256;
constexpr int kMaxColumns = 8192;

struct NormArgs {
    const void *x;
    long T;
    int E;
    const float *gamma, *beta;
    float eps;
    void *y;                 // optional outputs
    float *mean, *rstd;
    const float *wg, *bg;    // [E, n], [n]
    int n;
    float *logits;           // [T, n], or null
};

struct NormGradArgs {
    const void *dy, *x;
    long T;
    int E;
    const float *gamma, *beta;
    const float *mean, *rstd;
    const void *dres;        // or null
    const float *dlogits, *wg;       // null: no router
    int n;
    void *dx;
    float *partial;          // [parts][2 + n][E], then [parts][n]
    float *dgamma, *dbeta, *dwg, *dbg;
    int accumulate;
};

// Sum over the workgroup's threads, in all of them; `red` holds one value per wavefront.
__device__ inline float block_sum(float v, float *red) {
    v = group_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < kThreads / 64; ++w) s += red[w];
    return s;
}

template <class X, class Y>
__global__ __launch_bounds__(kThreads) void train_norm_kernel(NormArgs a) {
    __shared__ float red[kThreads / 64];
    const size_t t = blockIdx.x;
    const X *x = static_cast<const X *>(a.x) + t * a.E;
    float s = 0.0f;
    for (int j = threadIdx.x; j < a.E; j += kThreads) s += load_elem(x + j);
    const float mean = block_sum(s, red) / (float)a.E;
    s = 0.0f;
    for (int j = threadIdx.x; j < a.E; j += kThreads) {
        const float d = load_elem(x + j) - mean;
        s += d * d;
    }
    const float rstd = 1.0f / __builtin_sqrtf(block_sum(s, red) / (float)a.E + a.eps);
    float part[kMaxExperts] = {};
    for (int j = threadIdx.x; j < a.E; j += kThreads) {
        if (!a.y && !a.logits) break;
        const float y = (load_elem(x + j) - mean) * rstd * a.gamma[j] + a.beta[j];
        if (a.y) store_elem(static_cast<Y *>(a.y) + t * a.E + j, y);
        if (a.logits) {
#pragma unroll
            for (int e = 0; e < kMaxExperts; ++e)
                if (e < a.n) part[e] = __builtin_fmaf(y, a.wg[(size_t)j * a.n + e], part[e]);
        }
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[t] = mean;
        if (a.rstd) a.rstd[t] = rstd;
    }
    if (a.logits) {
#pragma unroll
        for (int e = 0; e < kMaxExperts; ++e) {
            if (e >= a.n) break;
            const float l = block_sum(part[e], red);
            if (threadIdx.x == 0) a.logits[t * a.n + e] = l + a.bg[e];
        }
    }
}

// dy with the router's share
template <class Y>
__device__ inline float incoming(const NormGradArgs &a, size_t t, int j) {
    float h = load_elem(static_cast<const Y *>(a.dy) + t * a.E + j);
    if (a.dlogits)
        for (int e = 0; e < a.n; ++e) h = __builtin_fmaf(a.dlogits[t * a.n + e], a.wg[(size_t)j * a.n + e], h);
    return h;
}

template <class X, class Y>
__global__ __launch_bounds__(kThreads) void norm_grad_rows_kernel(NormGradArgs a, float eps) {
    __shared__ float red[kThreads / 64];
    const size_t t = blockIdx.x;
    const X *x = static_cast<const X *>(a.x) + t * a.E;
    float mean, rstd, s = 0.0f;
    if (a.mean) {
        mean = a.mean[t], rstd = a.rstd[t];
    } else {
        for (int j = threadIdx.x; j < a.E; j += kThreads) s += load_elem(x + j);
        mean = block_sum(s, red) / (float)a.E;
        s = 0.0f;
        for (int j = threadIdx.x; j < a.E; j += kThreads) {
            const float d = load_elem(x + j) - mean;
            s += d * d;
        }
        rstd = 1.0f / __builtin_sqrtf(block_sum(s, red) / (float)a.E + eps);
    }
    float s0 = 0.0f, s1 = 0.0f;
    for (int j = threadIdx.x; j < a.E; j += kThreads) {
        const float g = incoming<Y>(a, t, j) * a.gamma[j];
        s0 += g;
        s1 += g * ((load_elem(x + j) - mean) * rstd);
    }
    const float c0 = block_sum(s0, red) / (float)a.E, c1 = block_sum(s1, red) / (float)a.E;
    for (int j = threadIdx.x; j < a.E; j += kThreads) {
        const float g = incoming<Y>(a, t, j) * a.gamma[j], xh = (load_elem(x + j) - mean) * rstd;
        float d = rstd * (g - c0 - xh * c1);
        if (a.dres) d += load_elem(static_cast<const X *>(a.dres) + t * a.E + j);
        store_elem(static_cast<X *>(a.dx) + t * a.E + j, d);
    }
}

// Columns' sums over a range of rows.
template <class X, class Y>
__global__ __launch_bounds__(kThreads) void norm_grad_columns_kernel(NormGradArgs a, long rows_per_part) {
    const int j = blockIdx.x * kThreads + threadIdx.x;
    const long t0 = (long)blockIdx.y * rows_per_part, t1 = t0 + rows_per_part < a.T ? t0 + rows_per_part : a.T;
    const int n = a.dlogits ? a.n : 0;
    if (j < a.E) {
        float sum[2 + kMaxExperts] = {};
        for (long t = t0; t < t1; ++t) {
            const float h = incoming<Y>(a, t, j);
            const float xh = (load_elem(static_cast<const X *>(a.x) + (size_t)t * a.E + j) - a.mean[t]) * a.rstd[t];
            sum[0] = __builtin_fmaf(h, xh, sum[0]);
            sum[1] += h;
            if (a.dwg) {
                const float y = xh * a.gamma[j] + a.beta[j];
                for (int e = 0; e < n; ++e) sum[2 + e] = __builtin_fmaf(y, a.dlogits[(size_t)t * n + e], sum[2 + e]);
            }
        }
        float *p = a.partial + (size_t)blockIdx.y * (2 + n) * a.E + j;
        for (int q = 0; q < 2 + n; ++q) p[(size_t)q * a.E] = sum[q];
    }
    if (blockIdx.x == 0 && (int)threadIdx.x < n) {
        float s = 0.0f;
        for (long t = t0; t < t1; ++t) s += a.dlogits[(size_t)t * n + threadIdx.x];
        a.partial[(size_t)gridDim.y * (2 + n) * a.E + (size_t)blockIdx.y * n + threadIdx.x] = s;
    }
}

__global__ __launch_bounds__(kThreads) void norm_grad_sum_kernel(NormGradArgs a, int parts) {
    const int n = a.dlogits ? a.n : 0, i = blockIdx.x * kThreads + threadIdx.x, q = i / a.E, j = i % a.E;
    if (q < 2 + n) {
        float s = 0.0f;
        for (int p = 0; p < parts; ++p) s += a.partial[(size_t)p * (2 + n) * a.E + i];
        float *out = q == 0 ? a.dgamma + j : q == 1 ? a.dbeta + j : a.dwg ? a.dwg + (size_t)j * n + (q - 2) : nullptr;
        if (out) *out = a.accumulate ? *out + s : s;
    } else if (i - (2 + n) * a.E < n && a.dbg) {
        const int e = i - (2 + n) * a.E;
        float s = 0.0f;
        for (int p = 0; p < parts; ++p) s += a.partial[(size_t)parts * (2 + n) * a.E + (size_t)p * n + e];
        a.dbg[e] = a.accumulate ? a.dbg[e] + s : s;
    }
}

// Rows in at most 256 ranges.
int grad_parts(long T) {
    const long parts = (T + 63) / 64;
    return (int)(parts < 256 ? parts : 256);
}

struct GradLayout {
    size_t mean, rstd, partial, total;
};

GradLayout grad_layout(long T, int E, int n) {
    GradLayout L;
    const size_t rows = ((size_t)T * 4 + 255) / 256 * 256, parts = (size_t)grad_parts(T);
    L.mean = 0, L.rstd = rows, L.partial = 2 * rows;
    L.total = L.partial + (parts * (2 + n) * E * 4 + parts * n * 4 + 255) / 256 * 256;
    return L;
}

template <class X, class Y>
struct RunNorm {
    static int run(const NormArgs &a, hipStream_t st) {
        train_norm_kernel<X, Y><<<dim3((unsigned)a.T), dim3(kThreads), 0, st>>>(a);
        return check_launch("sa_layernorm");
    }
};

template <class X, class Y>
struct RunNormGrad {
    static int run(NormGradArgs &a, float eps, uint8_t *ws, hipStream_t st) {
        if (a.dgamma) {
            // the sums over rows first: dx may take the place of what they read
            const int n = a.dlogits ? a.n : 0, parts = grad_parts(a.T);
            const GradLayout L = grad_layout(a.T, a.E, n);
            a.partial = reinterpret_cast<float *>(ws + L.partial);
            if (!a.mean) {
                NormArgs f{};
                f.x = a.x, f.T = a.T, f.E = a.E, f.eps = eps;
                f.mean = reinterpret_cast<float *>(ws + L.mean), f.rstd = reinterpret_cast<float *>(ws + L.rstd);
                const int rc = RunNorm<X, Y>::run(f, st);
                if (rc != SA_OK) return rc;
                a.mean = f.mean, a.rstd = f.rstd;
            }
            const long per = (a.T + parts - 1) / parts;
            norm_grad_columns_kernel<X, Y><<<dim3((unsigned)((a.E + kThreads - 1) / kThreads), (unsigned)parts), dim3(kThreads), 0, st>>>(a, per);
            int rc = check_launch("sa_layernorm_backward(columns)");
            if (rc != SA_OK) return rc;
            const int total = (2 + n) * a.E + n;
            norm_grad_sum_kernel<<<dim3((unsigned)((total + kThreads - 1) / kThreads)), dim3(kThreads), 0, st>>>(a, parts);
            rc = check_launch("sa_layernorm_backward(sums)");
            if (rc != SA_OK) return rc;
        }
        norm_grad_rows_kernel<X, Y><<<dim3((unsigned)a.T), dim3(kThreads), 0, st>>>(a, eps);
        return check_launch("sa_layernorm_backward(rows)");
    }
};

int check_sizes(const char *what, long T, int E, bool route, int n_experts) {
    SA_REQUIRE(T >= 0 && E > 0, SA_ERR_INVALID, "%s: T < 0 or E <= 0", what);
    SA_REQUIRE(E <= kMaxColumns, SA_ERR_UNSUPPORTED, "%s: rows of more than %d elements are not built", what, kMaxColumns);
    SA_REQUIRE(T < (1L << 31), SA_ERR_SHAPE, "%s: T >= 2^31", what);
    if (route) SA_REQUIRE(n_experts >= 2 && n_experts <= kMaxExperts, SA_ERR_SHAPE, "%s: 2 to 8 experts (got %d)", what, n_experts);
    return SA_OK;
}

}  // namespace

extern "C" int sa_layernorm(const void *x, int x_type, long T, int E, const float *gamma, const float *beta, float eps,
                            void *y_or_null, int y_type, float *mean_or_null, float *rstd_or_null, const float *wg_or_null,
                            const float *bg_or_null, int n_experts, float *logits_or_null, void *stream) {
    sa::clear_error();
    const bool route = logits_or_null != nullptr;
    int rc = sa::check_row_types("sa_layernorm", x_type, y_type);
    if (rc == SA_OK) rc = check_sizes("sa_layernorm", T, E, route, n_experts);
    if (rc != SA_OK || T == 0) return rc;
    SA_REQUIRE(x && gamma && beta, SA_ERR_INVALID, "sa_layernorm: NULL buffer");
    SA_REQUIRE(!route || (wg_or_null && bg_or_null), SA_ERR_INVALID, "sa_layernorm: logits need wg and bg");
    SA_REQUIRE(y_or_null || mean_or_null || rstd_or_null || route, SA_ERR_INVALID, "sa_layernorm: no output requested");
    SA_REQUIRE(sa::aligned16(x) && sa::aligned16(gamma) && sa::aligned16(beta) && sa::aligned16(y_or_null) &&
                   sa::aligned16(mean_or_null) && sa::aligned16(rstd_or_null) && sa::aligned16(wg_or_null) &&
                   sa::aligned16(bg_or_null) && sa::aligned16(logits_or_null),
               SA_ERR_ALIGN, "sa_layernorm: pointers must be 16-byte aligned");
    const NormArgs a{x, T, E, gamma, beta, eps, y_or_null, mean_or_null, rstd_or_null, wg_or_null, bg_or_null, route ? n_experts : 0,
                     logits_or_null};
    return sa::for_row_types<RunNorm>(x_type, y_type, a, sa::as_stream(stream));
}

extern "C" size_t sa_layernorm_backward_workspace_bytes(long T, int E, int n_experts) {
    if (T <= 0 || E <= 0 || E > kMaxColumns || T >= (1L << 31)) return 0;
    if (n_experts != 0 && (n_experts < 2 || n_experts > sa::kMaxExperts)) return 0;
    return grad_layout(T, E, n_experts).total;
}

extern "C" int sa_layernorm_backward(const void *dy, int y_type, const void *x, int x_type, long T, int E, const float *gamma,
                                     const float *beta_or_null, float eps, const float *mean_or_null, const float *rstd_or_null,
                                     const void *dres_or_null, const float *dlogits_or_null, const float *wg_or_null, int n_experts,
                                     void *dx, float *dgamma_or_null, float *dbeta_or_null, float *dwg_or_null, float *dbg_or_null,
                                     int accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    sa::clear_error();
    const bool route = dlogits_or_null != nullptr, params = dgamma_or_null != nullptr;
    int rc = sa::check_row_types("sa_layernorm_backward", x_type, y_type);
    if (rc == SA_OK) rc = check_sizes("sa_layernorm_backward", T, E, route || dwg_or_null, n_experts);
    if (rc != SA_OK) return rc;
    SA_REQUIRE((dbeta_or_null != nullptr) == params, SA_ERR_INVALID, "sa_layernorm_backward: dgamma and dbeta go together");
    SA_REQUIRE((dwg_or_null != nullptr) == (dbg_or_null != nullptr), SA_ERR_INVALID, "sa_layernorm_backward: dwg and dbg go together");
    SA_REQUIRE(dwg_or_null == nullptr || (params && (route || T == 0)), SA_ERR_INVALID,
               "sa_layernorm_backward: dwg and dbg need dlogits, dgamma and dbeta");
    SA_REQUIRE((mean_or_null != nullptr) == (rstd_or_null != nullptr), SA_ERR_INVALID, "sa_layernorm_backward: mean and rstd go together");
    SA_REQUIRE(sa::aligned16(dy) && sa::aligned16(x) && sa::aligned16(gamma) && sa::aligned16(beta_or_null) &&
                   sa::aligned16(mean_or_null) && sa::aligned16(rstd_or_null) && sa::aligned16(dres_or_null) &&
                   sa::aligned16(dlogits_or_null) && sa::aligned16(wg_or_null) && sa::aligned16(dx) && sa::aligned16(dgamma_or_null) &&
                   sa::aligned16(dbeta_or_null) && sa::aligned16(dwg_or_null) && sa::aligned16(dbg_or_null) && sa::aligned16(workspace),
               SA_ERR_ALIGN, "sa_layernorm_backward: pointers must be 16-byte aligned");
    hipStream_t st = sa::as_stream(stream);
    if (T == 0) {
        // sums over no rows
        if (accumulate) return SA_OK;
        float *const out[4] = {dgamma_or_null, dbeta_or_null, dwg_or_null, dbg_or_null};
        const size_t words[4] = {(size_t)E, (size_t)E, (size_t)E * n_experts, (size_t)n_experts};
        for (int i = 0; i < 4 && rc == SA_OK; ++i)
            if (out[i]) rc = sa::launch_zero(out[i], words[i] * 4, st);
        return rc;
    }
    SA_REQUIRE(dy && x && gamma && dx, SA_ERR_INVALID, "sa_layernorm_backward: NULL buffer");
    SA_REQUIRE(!route || wg_or_null, SA_ERR_INVALID, "sa_layernorm_backward: dlogits need wg");
    SA_REQUIRE(!dwg_or_null || beta_or_null, SA_ERR_INVALID, "sa_layernorm_backward: dwg needs beta");
    if (params) {
        const size_t need = sa_layernorm_backward_workspace_bytes(T, E, route ? n_experts : 0);
        SA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SA_ERR_WORKSPACE,
                   "sa_layernorm_backward: workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    }
    NormGradArgs a{};
    a.dy = dy, a.x = x, a.T = T, a.E = E, a.gamma = gamma, a.beta = beta_or_null, a.mean = mean_or_null, a.rstd = rstd_or_null;
    a.dres = dres_or_null, a.dlogits = dlogits_or_null, a.wg = wg_or_null, a.n = route ? n_experts : 0, a.dx = dx;
    a.dgamma = dgamma_or_null, a.dbeta = dbeta_or_null, a.dwg = dwg_or_null, a.dbg = dbg_or_null, a.accumulate = accumulate;
    return sa::for_row_types<RunNormGrad>(x_type, y_type, a, eps, static_cast<uint8_t *>(workspace), st);
}
