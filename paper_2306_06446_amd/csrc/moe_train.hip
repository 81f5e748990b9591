// What trains the router: the balance loss of Eq. 4 with its gradient and the tokens of each expert, and the gradient of the gated
// combine behind a top-1 dispatch (Sec. 4.2).
//
//   p = softmax(l), o(i) the best expert but i, d_i = (p_i - p_o(i)) / std, q_i = Phi(d_i)
//   u_i = alpha_i sum_t p_i, v_i = alpha_i sum_t q_i, losses SCV(u), SCV(v), SCV(u) = mean((u - m)^2) / m^2, m = mean(u)
//   dSCV / du_i = 2 (u_i - sum u^2 / sum u) / (n m^2)
//   with c and f the gradients of the sums of p and q:  a = c + J^T (f phi(d) / std),  J p_i = p_i - p_o(i),  dl = p (a - <p, a>)
#include "common.h"
#include "layernorm.h"
#include "row_types.h"

namespace {

using namespace sa;

constexpr int kMaxE = kMaxExperts;
constexpr int kTok = 256;                // tokens per workgroup

// A token's routing: p, and for each expert the normal deviate of its distance to the best of the others.
struct TokenRouting {
    float p[kMaxE], z[kMaxE];
    int first, second;                   // largest and second largest logit, ties to the lowest index
};

__device__ inline TokenRouting route_token(const float *l, int E, float inv_noise_std) {
    TokenRouting r;
    float v[kMaxE];
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) v[e] = e < E ? l[e] : 0.0f;
    float l0 = v[0], l1 = v[1];
    r.first = 0, r.second = 1;
    if (l1 > l0) { const float t = l0; l0 = l1; l1 = t; r.first = 1, r.second = 0; }
#pragma unroll
    for (int e = 2; e < kMaxE; ++e) {
        if (e >= E) break;
        if (v[e] > l0) { l1 = l0, r.second = r.first, l0 = v[e], r.first = e; }
        else if (v[e] > l1) { l1 = v[e], r.second = e; }
    }
    float den = 0.0f;
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        r.p[e] = e < E ? expf(v[e] - l0) : 0.0f;
        den += r.p[e];
    }
    const float inv = 1.0f / den;
    float p0 = 0.0f, p1 = 0.0f;
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        r.p[e] *= inv;
        if (e == r.first) p0 = r.p[e];
        if (e == r.second) p1 = r.p[e];
    }
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) r.z[e] = (r.p[e] - (e == r.first ? p1 : p0)) * inv_noise_std;
    return r;
}

struct BalanceArgs {
    const float *logits;
    long T;
    int E;
    const uint8_t *valid;
    const float *alpha;
    float noise_std;
    const float *dlosses;
    float *losses, *sums;
    int32_t *counts;
    float *dlogits;
    int accumulate;
    double *partial;         // [blocks][2 * kMaxE]: sums of p, of q
    int32_t *partial_counts; // [blocks][kMaxE]
    float *coeff;            // [2 * kMaxE]: c, f
};

__device__ inline double wave_sum_d(double v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

__global__ __launch_bounds__(kTok) void balance_sums_kernel(BalanceArgs a) {
    __shared__ double red[kTok / 64][2 * kMaxE];
    __shared__ int32_t cnt[kTok / 64][kMaxE];
    const long t = (long)blockIdx.x * kTok + threadIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool in = t < a.T && (!a.valid || a.valid[t] != 0);
    TokenRouting r;
    r.first = -1;
    if (in) r = route_token(a.logits + (size_t)t * a.E, a.E, 1.0f / a.noise_std);
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        if (e >= a.E) break;
        const double sp = wave_sum_d(in ? (double)r.p[e] : 0.0);
        const double sq = wave_sum_d(in ? 0.5 * (double)erfcf(r.z[e] * -0.70710678118654752f) : 0.0);
        const int c = __popcll(__ballot(r.first == e));
        if (lane == 0) red[wave][e] = sp, red[wave][kMaxE + e] = sq, cnt[wave][e] = c;
    }
    __syncthreads();
    const int i = threadIdx.x, e = i % kMaxE;
    if (i < 2 * kMaxE && e < a.E) {
        double s = 0.0;
        for (int w = 0; w < kTok / 64; ++w) s += red[w][i];
        a.partial[(size_t)blockIdx.x * 2 * kMaxE + i] = s;
        if (i < kMaxE) {
            int c = 0;
            for (int w = 0; w < kTok / 64; ++w) c += cnt[w][i];
            a.partial_counts[(size_t)blockIdx.x * kMaxE + i] = c;
        }
    }
}

__global__ __launch_bounds__(64) void balance_losses_kernel(BalanceArgs a, long blocks) {
    __shared__ double u[2 * kMaxE];
    const int i = threadIdx.x, e = i % kMaxE, kind = i / kMaxE;
    if (kind < 2 && e < a.E) {
        double s = 0.0;
        for (long b = 0; b < blocks; ++b) s += a.partial[(size_t)b * 2 * kMaxE + i];
        u[i] = s * (double)a.alpha[e];
        if (a.sums) a.sums[kind * a.E + e] = (float)u[i];
    } else if (kind == 2 && e < a.E && a.counts) {
        int c = 0;
        for (long b = 0; b < blocks; ++b) c += a.partial_counts[(size_t)b * kMaxE + e];
        a.counts[e] = c;
    }
    __syncthreads();
    if (kind < 2 && e < a.E) {
        double sum = 0.0, squares = 0.0, var = 0.0;
        for (int k = 0; k < a.E; ++k) sum += u[kind * kMaxE + k], squares += u[kind * kMaxE + k] * u[kind * kMaxE + k];
        const double m = sum / a.E;
        for (int k = 0; k < a.E; ++k) var += (u[kind * kMaxE + k] - m) * (u[kind * kMaxE + k] - m);
        const bool none = m == 0.0;
        if (e == 0) a.losses[kind] = none ? 0.0f : (float)(var / a.E / (m * m));
        a.coeff[i] = none ? 0.0f : (float)(2.0 / (a.E * m * m) * (u[i] - squares / sum) * (double)a.alpha[e] * (double)a.dlosses[kind]);
    }
}

__global__ __launch_bounds__(kTok) void balance_grad_kernel(BalanceArgs a) {
    const long t = (long)blockIdx.x * kTok + threadIdx.x;
    if (t >= a.T) return;
    float *dl = a.dlogits + (size_t)t * a.E;
    if (a.valid && a.valid[t] == 0) {
        if (!a.accumulate)
            for (int e = 0; e < a.E; ++e) dl[e] = 0.0f;
        return;
    }
    const TokenRouting r = route_token(a.logits + (size_t)t * a.E, a.E, 1.0f / a.noise_std);
    const float peak = 0.39894228040143268f / a.noise_std;
    float up[kMaxE], to_first = 0.0f, to_second = 0.0f;
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        up[e] = 0.0f;
        if (e >= a.E) continue;
        const float f = a.coeff[kMaxE + e] * peak * expf(-0.5f * r.z[e] * r.z[e]);
        up[e] = a.coeff[e] + f;
        if (e == r.first) to_second -= f; else to_first -= f;
    }
    float mean = 0.0f;
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        up[e] += (e == r.first ? to_first : 0.0f) + (e == r.second ? to_second : 0.0f);
        mean = __builtin_fmaf(r.p[e], up[e], mean);
    }
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) {
        if (e >= a.E) break;
        const float d = r.p[e] * (up[e] - mean);
        dl[e] = a.accumulate ? dl[e] + d : d;
    }
}

long balance_blocks(long T) { return (T + kTok - 1) / kTok; }
size_t balance_workspace(long T) {
    return (size_t)balance_blocks(T) * (2 * kMaxE * 8 + kMaxE * 4) + 256;
}

struct CombineGradArgs {
    const void *dy, *src;
    RowSel sel;
    const float *gate, *logits;
    int n, E;
    void *dsrc;
    float *dgate, *dlogits;
};

template <class T>
__device__ inline float load_elem(const T *p) { return (float)*p; }
template <class T>
__device__ inline void store_elem(T *p, float v) { *p = (T)v; }

// A wavefront to a row.
template <class Y, class S>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
    const int32_t *rows;
    long n_rows;
    resolve_rows(a.sel, rows, n_rows);
    const long i = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (i >= n_rows) return;
    const size_t r = rows ? (size_t)rows[i] : (size_t)i;
    const float gate = a.gate ? a.gate[r] : 1.0f;
    const Y *dy = static_cast<const Y *>(a.dy) + r * a.E;
    const bool dot = a.dgate || a.dlogits;
    float s = 0.0f;
    for (int j = lane; j < a.E; j += 64) {
        const float d = load_elem(dy + j);
        if (dot) s = __builtin_fmaf(d, load_elem(static_cast<const S *>(a.src) + (size_t)i * a.E + j), s);
        if (a.dsrc) store_elem(static_cast<S *>(a.dsrc) + (size_t)i * a.E + j, gate * d);
    }
    if (!dot) return;
    s = group_sum<64>(s);
    if (lane != 0) return;
    if (a.dgate) a.dgate[r] = s;
    if (a.dlogits) {
        const TokenRouting t = route_token(a.logits + r * a.n, a.n, 1.0f);
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < kMaxE; ++e)
            if (e == t.first) top = t.p[e];
#pragma unroll
        for (int e = 0; e < kMaxE; ++e) {
            if (e >= a.n) break;
            a.dlogits[r * a.n + e] = s * top * ((e == t.first ? 1.0f : 0.0f) - t.p[e]);
        }
    }
}

template <class Y, class S>
struct RunCombineGrad {
    static int run(const CombineGradArgs &a, hipStream_t st) {
        combine_grad_kernel<Y, S><<<dim3((unsigned)((a.sel.max_rows + 3) / 4)), dim3(256), 0, st>>>(a);
        return check_launch("sa_combine_rows_backward");
    }
};

}  // namespace

extern "C" size_t sa_moe_balance_loss_grad_workspace_bytes(long T, int E) {
    if (T < 0 || T >= (1L << 31) || E < 2 || E > kMaxE) return 0;
    return balance_workspace(T);
}

extern "C" int sa_moe_balance_loss_grad(const float *logits, long T, int E, const uint8_t *valid_or_null, const float *alpha,
                                        float noise_std, const float *dlosses, float *losses, float *sums_or_null,
                                        int32_t *counts_or_null, float *dlogits, int accumulate, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    sa::clear_error();
    SA_REQUIRE(T >= 0, SA_ERR_INVALID, "sa_moe_balance_loss_grad: T < 0");
    SA_REQUIRE(T < (1L << 31), SA_ERR_SHAPE, "sa_moe_balance_loss_grad: T >= 2^31");
    SA_REQUIRE(E >= 2 && E <= kMaxE, SA_ERR_SHAPE, "sa_moe_balance_loss_grad: 2 to 8 experts (got %d)", E);
    SA_REQUIRE(noise_std > 0.0f && __builtin_isfinite(noise_std), SA_ERR_INVALID,
               "sa_moe_balance_loss_grad: noise_std must be positive and finite");
    SA_REQUIRE(alpha && dlosses && losses && (T == 0 || (logits && dlogits)), SA_ERR_INVALID, "sa_moe_balance_loss_grad: NULL buffer");
    SA_REQUIRE(sa::aligned16(logits) && sa::aligned16(valid_or_null) && sa::aligned16(alpha) && sa::aligned16(dlosses) &&
                   sa::aligned16(losses) && sa::aligned16(sums_or_null) && sa::aligned16(counts_or_null) && sa::aligned16(dlogits) &&
                   sa::aligned16(workspace),
               SA_ERR_ALIGN, "sa_moe_balance_loss_grad: pointers must be 16-byte aligned");
    const size_t need = balance_workspace(T);
    SA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SA_ERR_WORKSPACE,
               "sa_moe_balance_loss_grad: workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    hipStream_t st = sa::as_stream(stream);
    const long blocks = balance_blocks(T);
    BalanceArgs a{logits, T, E, valid_or_null, alpha, noise_std, dlosses, losses, sums_or_null, counts_or_null, dlogits, accumulate};
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.coeff = reinterpret_cast<float *>(ws);
    a.partial = reinterpret_cast<double *>(ws + 256);
    a.partial_counts = reinterpret_cast<int32_t *>(ws + 256 + (size_t)blocks * 2 * kMaxE * 8);
    int rc;
    if (T > 0) {
        balance_sums_kernel<<<dim3((unsigned)blocks), dim3(kTok), 0, st>>>(a);
        rc = sa::check_launch("sa_moe_balance_loss_grad(sums)");
        if (rc != SA_OK) return rc;
    }
    balance_losses_kernel<<<dim3(1), dim3(64), 0, st>>>(a, blocks);
    rc = sa::check_launch("sa_moe_balance_loss_grad(losses)");
    if (rc != SA_OK || T == 0) return rc;
    balance_grad_kernel<<<dim3((unsigned)blocks), dim3(kTok), 0, st>>>(a);
    return sa::check_launch("sa_moe_balance_loss_grad(gradient)");
}

extern "C" int sa_combine_rows_backward(const void *dy, int y_type, const void *src_or_null, int src_type, const sa_rows *rows,
                                        const float *gate_or_null, const float *logits_or_null, int n_experts, int E,
                                        void *dsrc_or_null, float *dgate_or_null, float *dlogits_or_null, void *stream) {
    sa::clear_error();
    sa::RowSel sel;
    int rc = sa::validate_rows(rows, &sel);
    if (rc == SA_OK) rc = sa::check_row_types("sa_combine_rows_backward", y_type, src_type);
    if (rc != SA_OK) return rc;
    SA_REQUIRE(E > 0, SA_ERR_SHAPE, "sa_combine_rows_backward: E must be positive");
    SA_REQUIRE(!dlogits_or_null || (n_experts >= 2 && n_experts <= kMaxE), SA_ERR_SHAPE,
               "sa_combine_rows_backward: 2 to 8 experts (got %d)", n_experts);
    if (sel.max_rows == 0) return SA_OK;
    SA_REQUIRE(dy, SA_ERR_INVALID, "sa_combine_rows_backward: NULL buffer");
    SA_REQUIRE(dsrc_or_null || dgate_or_null || dlogits_or_null, SA_ERR_INVALID, "sa_combine_rows_backward: no output requested");
    SA_REQUIRE(src_or_null || !(dgate_or_null || dlogits_or_null), SA_ERR_INVALID, "sa_combine_rows_backward: dgate and dlogits need src");
    SA_REQUIRE(!dlogits_or_null || (logits_or_null && gate_or_null), SA_ERR_INVALID,
               "sa_combine_rows_backward: dlogits need logits and gate");
    SA_REQUIRE(sa::aligned16(dy) && sa::aligned16(src_or_null) && sa::aligned16(gate_or_null) && sa::aligned16(logits_or_null) &&
                   sa::aligned16(dsrc_or_null) && sa::aligned16(dgate_or_null) && sa::aligned16(dlogits_or_null) &&
                   sa::aligned4(sel.rows) && sa::aligned4(sel.counts),
               SA_ERR_ALIGN, "sa_combine_rows_backward: pointers must be 16-byte aligned");
    const CombineGradArgs a{dy, src_or_null, sel, gate_or_null, logits_or_null, n_experts, E, dsrc_or_null, dgate_or_null, dlogits_or_null};
    return sa::for_row_types<RunCombineGrad>(y_type, src_type, a, sa::as_stream(stream));
}
