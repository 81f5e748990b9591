// LayerNorm of training (Eq. 2) with its statistics and the router's logits, and its gradient with the residual's and the router's.
//
//   xh = (x - mean) rstd,  y = xh gamma + beta,  logits = y wg + bg
//   h = dy + dlogits wg^T,  g = h gamma,  dx = dres + rstd (g - <g> - xh <g xh>),  <.> the mean over the row
//   dgamma = sum_t h xh,  dbeta = sum_t h,  dwg = sum_t y dlogits,  dbg = sum_t dlogits
#include "layernorm_train.h"

namespace sa {

template <class X, class Y, class S, int ROUTE>
__global__ __launch_bounds__(S::THREADS) void train_norm_kernel(NormArgs a) {
    constexpr int VEC = S::VEC, CH = S::CH, HELD = ROUTE > kStreamed ? ROUTE : 0, PR = HELD ? HELD : 1, PC = HELD ? CH : 1;
    __shared__ float red[S::LANES > 64 ? PR : 1][2][S::WAVES];
    const int g = threadIdx.x / S::LANES, l = threadIdx.x % S::LANES;
    const RowPlace<S> p(l, a.E);
    RowSums<S, 1> sum{red};
    float gm[CH][VEC], bt[CH][VEC], w[PR][PC][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int j = p.at[c] + i;
            gm[c][i] = a.gamma ? a.gamma[j] : 0.0f;
            bt[c][i] = a.gamma ? a.beta[j] : 0.0f;
#pragma unroll
            for (int e = 0; e < HELD; ++e) w[e][c][i] = e < a.n && p.mine(c, i) ? a.wg[(size_t)j * a.n + e] : 0.0f;
        }
    const long stride = (long)gridDim.x * S::GROUPS;
    auto load = [&](Piece<X, VEC> (&x)[CH], long t) {
        const X *row = static_cast<const X *>(a.x) + (size_t)(t < a.T ? t : a.T - 1) * a.E;
#pragma unroll
        for (int c = 0; c < CH; ++c) x[c].load(row + p.at[c]);
    };
    Piece<X, VEC> nxt[CH], x[CH];
    long t0 = (long)blockIdx.x * S::GROUPS;
    load(nxt, t0 + g);
    for (; t0 < a.T; t0 += stride) {
        const long t = t0 + g;
#pragma unroll
        for (int c = 0; c < CH; ++c) x[c] = nxt[c];
        if (t0 + stride < a.T) load(nxt, t + stride);
        float s[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0] += p.mine(c, i) ? x[c][i] : 0.0f;
        sum(s);
        const float mean = s[0] / (float)a.E;
        s[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = x[c][i] - mean;
                s[0] = p.mine(c, i) ? __builtin_fmaf(d, d, s[0]) : s[0];
            }
        sum(s);
        const float rstd = 1.0f / __builtin_sqrtf(s[0] / (float)a.E + a.eps);
        float y[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[c][i] = __builtin_fmaf((x[c][i] - mean) * rstd, gm[c][i], bt[c][i]);
            if (a.y && t < a.T && p.any(c))
                store_piece<Y, VEC>(static_cast<Y *>(a.y) + (size_t)t * a.E + p.at[c], y[c], c < S::FULL ? 0 : p.skip[c]);
        }
        if (l == 0 && t < a.T) {
            if (a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd;
        }
        if constexpr (HELD > 0) {
            float part[HELD];
#pragma unroll
            for (int e = 0; e < HELD; ++e) {
                part[e] = 0.0f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) part[e] = __builtin_fmaf(y[c][i], w[e][c][i], part[e]);
            }
            RowSums<S, HELD> all{red, sum.turn};
            all(part, a.n);
            sum.turn = all.turn;
            if (l == 0 && t < a.T) {
#pragma unroll
                for (int e = 0; e < HELD; ++e)
                    if (e < a.n) a.logits[(size_t)t * a.n + e] = part[e] + a.bg[e];
            }
        }
        if constexpr (ROUTE == kStreamed) {
#pragma unroll 1
            for (int e = 0; e < a.n; ++e) {
                s[0] = 0.0f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        s[0] = p.mine(c, i) ? __builtin_fmaf(y[c][i], a.wg[(size_t)(p.at[c] + i) * a.n + e], s[0]) : s[0];
                sum(s);
                if (l == 0 && t < a.T) a.logits[(size_t)t * a.n + e] = s[0] + a.bg[e];
            }
        }
    }
}

template <class X, class Y>
int launch_norm_rows(const NormArgs &a, hipStream_t st) {
    constexpr int VEC = row_vec<X, Y>();
    auto rows = [&](auto shape, auto route) {
        using S = decltype(shape);
        // up to 4 workgroups to a CU, the same number of steps in each
        const long cap = 1024 * 256 / S::THREADS;
        const long steps = (a.T + S::GROUPS * cap - 1) / (S::GROUPS * cap);
        const long blocks = (a.T + S::GROUPS * steps - 1) / (S::GROUPS * steps);
        train_norm_kernel<X, Y, S, decltype(route)::value><<<dim3((unsigned)blocks), dim3(S::THREADS), 0, st>>>(a);
        return check_launch("sa_layernorm");
    };
    auto with = [&](auto route) { return [&rows, route](auto shape) { return rows(shape, route); }; };
    if (!a.logits) return by_shape<VEC>(a.E, with(std::integral_constant<int, 0>()));
    if (a.n == 2) return by_shape<VEC>(a.E, with(std::integral_constant<int, 2>()));
    if (a.E > kMaxRoute8Columns) return by_wide_shape<VEC>(a.E, with(std::integral_constant<int, kStreamed>()));
    return by_shape_route8<VEC>(a.E, with(std::integral_constant<int, kMaxExperts>()));
}

}  // namespace sa

namespace {

using namespace sa;

// The parts' sums, in fp64 and in ascending order: 16 threads to four columns.
__global__ __launch_bounds__(256) void norm_grad_sum_kernel(NormGradArgs a, int parts) {
    constexpr int kSlices = 16;
    __shared__ double red[kSlices][64];
    const int n = a.dlogits ? a.n : 0, columns = padded_columns(a.E), all = (2 + n) * columns;
    const int slice = threadIdx.x >> 4, quad = threadIdx.x & 15, at = (int)blockIdx.x * 64 + quad * 4;
    const bool last = blockIdx.x == gridDim.x - 1;           // has room for the router's bias behind the columns
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    const float *from = nullptr;
    size_t step = 0;
    if (at < all) from = a.partial + at, step = (size_t)all;
    else if (last && quad >= 14 && a.dbg) from = a.partial_dbg + (quad - 14) * 4, step = kMaxExperts;
    if (from) {
#pragma unroll 8
        for (int k = slice; k < parts; k += kSlices) {
            const float4 v = *reinterpret_cast<const float4 *>(from + k * step);
            s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[slice][quad * 4 + i] = s[i];
    __syncthreads();
    if (threadIdx.x >= 64) return;
    double sum = 0.0;
    for (int k = 0; k < kSlices; ++k) sum += red[k][threadIdx.x];
    const int i = (int)blockIdx.x * 64 + threadIdx.x, q = i / columns, j = i % columns;
    float *out = nullptr;
    if (i < all) {
        if (j < a.E) out = q == 0 ? a.dgamma + j : q == 1 ? a.dbeta + j : a.dwg ? a.dwg + (size_t)j * n + (q - 2) : nullptr;
    } else if (last && a.dbg && threadIdx.x >= 56 && (int)threadIdx.x - 56 < n) {
        out = a.dbg + (threadIdx.x - 56);
    }
    if (out) *out = (a.accumulate ? *out : 0.0f) + (float)sum;
}

// Router weights [E, n] to [n, columns]: rows that are read again for every token (kStreamed).
__global__ __launch_bounds__(256) void router_rows_kernel(const float *wg, int E, int n, float *rows) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < E * n) rows[(size_t)(i % n) * padded_columns(E) + i / n] = wg[i];
}

struct GradLayout {
    size_t partial, dbg, weights, mean, rstd, total;
};

GradLayout grad_layout(long T, int E, int n) {
    GradLayout L;
    auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    const size_t parts = (size_t)(T < kMaxGradParts ? T : kMaxGradParts), columns = (size_t)padded_columns(E);
    const bool streamed = n > 2 && E > kMaxRoute8Columns;
    L.partial = 0;
    L.dbg = up(parts * (2 + n) * columns * 4);
    L.weights = L.dbg + up(n ? parts * kMaxExperts * 4 : 0);
    L.mean = L.weights + up(streamed ? n * columns * 4 : 0);
    L.rstd = L.mean + up(streamed ? (size_t)T * 4 : 0);
    L.total = L.rstd + up(streamed ? (size_t)T * 4 : 0);
    return L;
}

template <class X, class Y>
struct RunNorm {
    static int run(const NormArgs &a, hipStream_t st) { return launch_norm_rows<X, Y>(a, st); }
};

template <class X, class Y>
struct RunNormGrad {
    static int run(NormGradArgs &a, uint8_t *ws, hipStream_t st) {
        const int n = a.dlogits ? a.n : 0;
        const bool streamed = n > 2 && a.E > kMaxRoute8Columns;
        a.weights = a.wg, a.by_expert = 1, a.by_column = n;
        if (a.dgamma) {
            const GradLayout L = grad_layout(a.T, a.E, n);
            a.partial = reinterpret_cast<float *>(ws + L.partial);
            a.partial_dbg = reinterpret_cast<float *>(ws + L.dbg);
            if (streamed) {
                float *rows = reinterpret_cast<float *>(ws + L.weights);
                router_rows_kernel<<<dim3((unsigned)((a.E * n + 255) / 256)), dim3(256), 0, st>>>(a.wg, a.E, n, rows);
                int rc = check_launch("sa_layernorm_backward(router's rows)");
                if (rc != SA_OK) return rc;
                a.weights = rows, a.by_expert = padded_columns(a.E), a.by_column = 1;
                if (!a.mean && a.dwg) {
                    NormArgs f{};
                    f.x = a.x, f.T = a.T, f.E = a.E, f.eps = a.eps;
                    f.mean = reinterpret_cast<float *>(ws + L.mean), f.rstd = reinterpret_cast<float *>(ws + L.rstd);
                    rc = launch_norm_rows<X, Y>(f, st);
                    if (rc != SA_OK) return rc;
                    a.mean = f.mean, a.rstd = f.rstd;
                }
            }
        }
        int parts = 0;
        const int rc = launch_norm_grad_rows<X, Y>(a, &parts, st);
        if (rc != SA_OK || !a.dgamma) return rc;
        const int blocks = ((2 + n) * padded_columns(a.E) + kMaxExperts + 63) / 64;
        norm_grad_sum_kernel<<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, parts);
        return check_launch("sa_layernorm_backward(sums)");
    }
};

int check_sizes(const char *what, long T, int E, bool route, int n_experts) {
    SA_REQUIRE(T >= 0 && E > 0, SA_ERR_INVALID, "%s: T < 0 or E <= 0", what);
    SA_REQUIRE(E <= kMaxNormColumns, SA_ERR_UNSUPPORTED, "%s: rows of more than %d elements are not built", what, kMaxNormColumns);
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
    if (T <= 0 || E <= 0 || E > kMaxNormColumns || T >= (1L << 31)) return 0;
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
    a.eps = eps;
    a.dres = dres_or_null, a.dlogits = dlogits_or_null, a.wg = wg_or_null, a.n = route ? n_experts : 0, a.dx = dx;
    a.dgamma = dgamma_or_null, a.dbeta = dbeta_or_null, a.dwg = dwg_or_null, a.dbg = dbg_or_null, a.accumulate = accumulate;
    return sa::for_row_types<RunNormGrad>(x_type, y_type, a, static_cast<uint8_t *>(workspace), st);
}
