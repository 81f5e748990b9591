// LayerNorm of training (Eq. 2) with its statistics and the router's logits, and its gradient with the residual's and the router's.
//
//   xh = (x - mean) rstd,  y = xh gamma + beta,  logits = y wg + bg
//   h = dy + dlogits wg^T,  g = h gamma,  dx = dres + rstd (g - <g> - xh <g xh>),  <.> the mean over the row
//   dgamma = sum_t h xh,  dbeta = sum_t h,  dwg = sum_t y dlogits,  dbg = sum_t dlogits
//
// The forward pass: a row stays in the registers of the lanes that share it (row_types.h), so x is read once: mean, centred squares, results.
// What bounds it: memory, 4 to 8 bytes an element; a wavefront keeps a row ahead in flight and waits for no store.  Measured: 12608 x 768
// fp32 to fp16 with the router of two 10.3 us (5.7 TB/s, part of it out of the memory-side cache; 37 as a workgroup to a row that reads it
// three times), 100000 x 1024 bf16 73 us (5.6), 35714 x 5600 fp16 161 (4.9), 5003 x 4099 bf16, rows that begin anywhere, 18.5 (4.4).
// Eight experts: 20000 x 768 27 to 30 us (3.1 to 3.4 TB/s), 20000 x 8000 bf16 178 to 211 (3.0 to 3.6), 131072 x 64 bf16 16.4 (2.4): two
// wavefronts to a SIMD are too few to hide memory behind.  Of rows from 769 elements on the weights take a lane's registers (96 to 128 of them),
// of narrow ones the tile that they come through takes the LDS (67.6 KB whatever the width); the products themselves are few, 0.25 GFLOP of
// 20000 x 768.
#include "layernorm_train.h"

namespace sa {

// TRAIN: y, mean and rstd are all wanted (else each is asked about).
constexpr int kNormWaves = 4;                // of a workgroup of rows of one wavefront or less
template <class X, class Y, class S, int ROUTE, bool TRAIN>
__global__ __launch_bounds__(S::WIDE ? 512 : 64 * kNormWaves) void train_norm_kernel(NormArgs a) {
    constexpr int VEC = S::VEC, CH = S::CH, HELD = ROUTE, PR = HELD ? HELD : 1, PC = HELD ? CH : 1;
    // Of many experts whose rows have whole wavefronts, lane l has the logit of expert l / 8, of every eighth step: eight rows leave at a time.
    constexpr bool EIGHT = HELD == kMaxExperts && S::LANES >= 64;
    constexpr int PERIOD = EIGHT ? 8 : S::PERIOD;
    __shared__ __align__(16) float red[S::WIDE ? PR : 1][2][8], tile[HELD == kMaxExperts ? kRouterTileFloats : 1];
    const RowPlace<S> p(a.E);
    const int g = p.g, l = p.l, groups = S::WIDE ? p.groups : 64 * kNormWaves / S::LANES;
    const float per = 1.0f / (float)a.E;
    RowSums<S, PR> sum(red, p);
    const long stride = (long)gridDim.x * groups;
    auto load = [&](Piece<X, VEC> (&x)[CH], long t) {
        const X *row = static_cast<const X *>(a.x) + (size_t)(t < a.T ? t : a.T - 1) * a.E;
#pragma unroll
        for (int c = 0; c < CH; ++c) x[c].load(row + p.at[c]);
    };
    Piece<X, VEC> nxt[CH], x[CH];
    long t0 = (long)blockIdx.x * groups;
    load(nxt, t0 + g);
    float gm[CH][VEC], bt[CH][VEC], w[PR][PC][VEC], bias[EIGHT ? 1 : PR];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_columns<VEC>(gm[c], a.gamma + p.at[c]);
        load_columns<VEC>(bt[c], a.beta + p.at[c]);
        if constexpr (HELD == 2) load_router_pair<VEC, PC>(w, c, a.wg + 2 * (size_t)p.at[c]);
    }
    if constexpr (HELD == kMaxExperts) load_router<S, PR>(w, p, a.wg, a.E, a.n, tile);
#pragma unroll
    for (int e = 0; e < HELD; ++e)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[e][c][i] = p.own(c, i, w[e][c][i]);
    const int expert = l >> 3;           // (EIGHT)
    if constexpr (EIGHT) {
        bias[0] = a.bg[expert < a.n ? expert : 0];
    } else {
#pragma unroll
        for (int e = 0; e < HELD; ++e) bias[e] = a.bg[HELD == 2 || e < a.n ? e : 0];
    }
    // What there is one of to a row is kept, a step to a lane, and leaves for PERIOD rows at a time: every step then stores the same
    // number of pieces, and a wait for the next row leaves the last row's stores in flight (one counter, in order).
    float kept_mean = 0.0f, kept_rstd = 0.0f, kept[EIGHT ? 1 : PR] = {};
    const long t_first = (long)blockIdx.x * groups + g;
    auto flush = [&](long steps) {       // the last 1 to PERIOD of `steps` steps
        if (l >= (EIGHT ? 64 : PERIOD)) return;
        const long k = (steps - 1) / PERIOD * PERIOD + (l & (PERIOD - 1)), t = t_first + k * stride;
        if (k >= steps || t >= a.T) return;
        if (l < PERIOD) {
            if (TRAIN || a.mean) a.mean[t] = kept_mean;
            if (TRAIN || a.rstd) a.rstd[t] = kept_rstd;
        }
        if constexpr (EIGHT) {
            if (expert < a.n) a.logits[(size_t)t * a.n + expert] = kept[0];
        } else {
#pragma unroll
            for (int e = 0; e < HELD; ++e)
                if (HELD == 2 || e < a.n) a.logits[(size_t)t * a.n + e] = kept[e];
        }
    };
    auto work = [&](const Piece<X, VEC> (&x)[CH], long t, bool row_ok, long step) {
        float s[1] = {0.0f};
        if constexpr (S::WIDE) {
#pragma unroll
            for (int c = 0; c < CH; ++c) arrived(x[c]);      // y may be in the place of x
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0] += p.own(c, i, x[c][i]);
        sum(s);
        const float mean = s[0] * per;
        s[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = p.own(c, i, x[c][i] - mean);
                s[0] = __builtin_fmaf(d, d, s[0]);
            }
        sum(s);
        const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(s[0], per, a.eps));
        const bool keep = (int)(step & (PERIOD - 1)) == (EIGHT ? l & 7 : l);
        kept_mean = keep ? mean : kept_mean;
        kept_rstd = keep ? rstd : kept_rstd;
        float y[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[c][i] = __builtin_fmaf((x[c][i] - mean) * rstd, gm[c][i], bt[c][i]);
            if (row_ok && (TRAIN || a.y)) stream_piece<Y, VEC>(static_cast<Y *>(a.y) + (size_t)t * a.E + p.at[c], y[c]);
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
            if constexpr (EIGHT) {
                float logit = eight_sums(part);
                if constexpr (S::WIDE) {
                    if ((l & 7) == 0) red[(l >> 3) & 7][sum.turn][threadIdx.x >> 6] = logit;
                    __syncthreads();
                    logit = sum.of(expert & 7);
                    sum.turn ^= 1;
                }
                kept[0] = keep ? logit + bias[0] : kept[0];
            } else {
                sum(part);
#pragma unroll
                for (int e = 0; e < HELD; ++e) kept[e] = keep ? part[e] + bias[e] : kept[e];
            }
        }
    };
    long step = 0;
    for (; t0 + groups <= a.T; t0 += stride) {
#pragma unroll
        for (int c = 0; c < CH; ++c) x[c] = nxt[c];
        load(nxt, t0 + g + stride);
        work(x, t0 + g, true, step++);
        if ((step & (PERIOD - 1)) == 0) flush(step);
    }
    if (t0 < a.T) {
        work(nxt, t0 + g, t0 + g < a.T, step++);
        flush(step);
    } else if ((step & (PERIOD - 1)) != 0) {
        flush(step);
    }
}

template <class X, class Y>
int launch_norm_rows(const NormArgs &a, hipStream_t st) {
    constexpr int VEC = row_vec<X, Y>();
    auto rows = [&](auto shape, auto route) {
        using S = decltype(shape);
        // 16 wavefronts to a CU, 32 where several wait for each other at every row (in two rounds where the registers have room for 16), 8
        // with the weights of many experts, each with as many rows as it takes.  16 is as many as there is room for, up to 128 registers, but
        // for rows of 16 elements to a lane, fp32 in, with a router of two and not all outputs: 129 to 131 registers, 12 wavefronts, and a
        // second round for the rest.
        const int threads = S::threads(a.E, kNormWaves);
        const long groups = S::groups(a.E, kNormWaves), steps = (a.T + groups - 1) / groups;
        const long cap = 256 * (decltype(route)::value == kMaxExperts ? 512 : S::WIDE ? 2048 : 1024) / threads;
        const dim3 grid((unsigned)(steps < cap ? steps : cap)), block((unsigned)threads);
        if (a.y && a.mean && a.rstd)
            train_norm_kernel<X, Y, S, decltype(route)::value, true><<<grid, block, 0, st>>>(a);
        else
            train_norm_kernel<X, Y, S, decltype(route)::value, false><<<grid, block, 0, st>>>(a);
        return check_launch("sa_layernorm");
    };
    auto with = [&](auto route) { return [&rows, route](auto shape) { return rows(shape, route); }; };
    if (!a.logits) return by_shape<VEC, true>(a.E, with(std::integral_constant<int, 0>()));
    if (a.n == 2) return by_shape<VEC, true>(a.E, with(std::integral_constant<int, 2>()));
    return by_shape<VEC, true>(a.E, with(std::integral_constant<int, kMaxExperts>()));
}

}  // namespace sa

namespace {

using namespace sa;

// The parts' sums in fp64, in a fixed order: 64 threads to four columns, whose loads (8 to a thread) are all in flight at once, for up to 512
// parts at a time.
constexpr int kSumColumns = 16;              // of a workgroup
__global__ __launch_bounds__(256) void norm_grad_sum_kernel(NormGradArgs a, int parts) {
    constexpr int kSlices = 256 / (kSumColumns / 4);
    constexpr int kEach = kGradParts / kSlices;
    __shared__ double red[4][kSumColumns];
    const int n = a.dlogits ? a.n : 0, columns = padded_columns(a.E), all = (2 + n) * columns;
    const int slice = threadIdx.x / 4, quad = threadIdx.x & 3, at = (int)blockIdx.x * kSumColumns + quad * 4;
    const bool last = blockIdx.x == gridDim.x - 1;           // the router's bias is behind the columns, in the last 8 places
    const float *from = a.partial;
    size_t step = (size_t)all;
    bool any = at < all;
    if (any) from += at;
    else if (last && quad >= 2 && a.dbg) any = true, from = a.partial_dbg + (quad - 2) * 4, step = kMaxExperts;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int first = 0; first < parts; first += kGradParts) {
        float4 v[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int part = first + slice + k * kSlices;
            v[k] = any && part < parts ? *reinterpret_cast<const float4 *>(from + part * step) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) s[0] += v[k].x, s[1] += v[k].y, s[2] += v[k].z, s[3] += v[k].w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int off = 4; off < 64; off *= 2) s[i] += __shfl_xor(s[i], off, 64);
        if ((threadIdx.x & 63) < 4) red[threadIdx.x >> 6][quad * 4 + i] = s[i];
    }
    __syncthreads();
    if (threadIdx.x >= kSumColumns) return;
    const double sum = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
    const int i = (int)blockIdx.x * kSumColumns + threadIdx.x, q = i / columns, j = i % columns;
    const int bias = (int)threadIdx.x - (kSumColumns - kMaxExperts);
    float *out = nullptr;
    if (i < all) {
        if (j < a.E) out = q == 0 ? a.dgamma + j : q == 1 ? a.dbeta + j : a.dwg ? a.dwg + (size_t)j * n + (q - 2) : nullptr;
    } else if (last && a.dbg && bias >= 0 && bias < n) {
        out = a.dbg + bias;
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

bool needs_weights(int E, int n) { return n > 2 && E > kMaxRoute8Columns; }
GradLayout grad_layout(long T, int E, int n, bool params) {
    GradLayout L;
    auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    const size_t parts = params ? (size_t)max_grad_parts(T, E) : 0, columns = (size_t)padded_columns(E);
    const bool streamed = needs_weights(E, n);
    L.partial = 0;
    L.dbg = up(parts * (2 + n) * columns * 4);
    L.weights = L.dbg + up(n ? parts * kMaxExperts * 4 : 0);
    L.mean = L.weights + up(streamed ? n * columns * 4 : 0);
    L.rstd = L.mean + up(streamed && params ? (size_t)T * 4 : 0);
    L.total = L.rstd + up(streamed && params ? (size_t)T * 4 : 0);
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
        const bool streamed = needs_weights(a.E, n);
        const GradLayout L = grad_layout(a.T, a.E, n, a.dgamma != nullptr);
        if (a.dgamma) {
            a.partial = reinterpret_cast<float *>(ws + L.partial);
            a.partial_dbg = reinterpret_cast<float *>(ws + L.dbg);
        }
        if (streamed) {
            float *rows = reinterpret_cast<float *>(ws + L.weights);
            router_rows_kernel<<<dim3((unsigned)((a.E * n + 255) / 256)), dim3(256), 0, st>>>(a.wg, a.E, n, rows);
            int rc = check_launch("sa_layernorm_backward(router's rows)");
            if (rc != SA_OK) return rc;
            a.weights = rows;
            if (!a.mean && a.dwg) {
                NormArgs f{};
                f.x = a.x, f.T = a.T, f.E = a.E, f.eps = a.eps, f.gamma = a.gamma, f.beta = a.gamma;
                f.mean = reinterpret_cast<float *>(ws + L.mean), f.rstd = reinterpret_cast<float *>(ws + L.rstd);
                rc = launch_norm_rows<X, Y>(f, st);
                if (rc != SA_OK) return rc;
                a.mean = f.mean, a.rstd = f.rstd;
            }
        }
        int parts = 0;
        const int rc = launch_norm_grad_rows<X, Y>(a, &parts, st);
        if (rc != SA_OK || !a.dgamma) return rc;
        const int blocks = ((2 + n) * padded_columns(a.E) + kMaxExperts + kSumColumns - 1) / kSumColumns;
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
    return grad_layout(T, E, n_experts, true).total;
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
    const size_t need = grad_layout(T, E, route ? n_experts : 0, params).total;
    if (need > 0) {
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
