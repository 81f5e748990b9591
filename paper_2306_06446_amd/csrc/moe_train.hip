// What trains the router: the balance loss of Eq. 4 with its gradient and the tokens of each expert, and the gradient of the gated
// combine behind a top-1 dispatch (Sec. 4.2).
//
//   p = softmax(l), o(i) the best expert but i, d_i = (p_i - p_o(i)) / std, q_i = Phi(d_i)
//   u_i = alpha_i sum_t p_i, v_i = alpha_i sum_t q_i, losses SCV(u), SCV(v), SCV(u) = mean((u - m)^2) / m^2, m = mean(u)
//   dSCV / du_i = 2 (u_i - sum u^2 / sum u) / (n m^2)
//   with c and f the gradients of the sums of p and q:  a = c + J^T (f phi(d) / std),  J p_i = p_i - p_o(i),  dl = p (a - <p, a>)
#include <type_traits>

#include "common.h"
#include "row_types.h"

namespace {

using namespace sa;

constexpr int kMaxE = kMaxExperts;

// A token's routing: p, and for each expert the normal deviate of its distance to the best of the others.
template <int E>
struct TokenRouting {
    float p[E], z[E];
    int first, second;                   // largest and second largest logit, ties to the lowest index
};

template <int E>
__device__ inline TokenRouting<E> route_token(const float *l, float inv_noise_std) {
    TokenRouting<E> r;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = l[e];
    float l0 = v[0], l1 = v[1];
    r.first = 0, r.second = 1;
    if (l1 > l0) { const float t = l0; l0 = l1; l1 = t; r.first = 1, r.second = 0; }
#pragma unroll
    for (int e = 2; e < E; ++e) {
        const bool best = v[e] > l0, next = v[e] > l1;
        r.second = best ? r.first : next ? e : r.second;
        l1 = best ? l0 : next ? v[e] : l1;
        r.first = best ? e : r.first;
        l0 = best ? v[e] : l0;
    }
    float den = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        r.p[e] = expf(v[e] - l0);
        den += r.p[e];
    }
    const float inv = 1.0f / den;
    float p0 = 0.0f, p1 = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        r.p[e] *= inv;
        p0 = e == r.first ? r.p[e] : p0;
        p1 = e == r.second ? r.p[e] : p1;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) r.z[e] = (r.p[e] - (e == r.first ? p1 : p0)) * inv_noise_std;
    return r;
}

struct BalanceArgs {
    const float *logits;
    long T;
    const uint8_t *valid;
    const float *alpha;
    float noise_std;
    const float *dlosses;
    float *losses, *sums;
    int32_t *counts;
    float *dlogits;
    int accumulate;
    double *partial;         // [2 E][parts]: sums of p, of q
    int32_t *partial_counts; // [E][parts]
    int parts;
};

template <int CTRL>
__device__ inline double dpp_add_d(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
    return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over a wavefront in all of its lanes, the most distant lanes first (as group_sum<64>, in fp64).
__device__ inline double wave_sum_d(double v) {
    v += __shfl_xor(v, 32, 64);
    v += __shfl_xor(v, 16, 64);
    v = dpp_add_d<0x128>(v);
    v = dpp_add_d<0x124>(v);
    v = dpp_add_d<0x122>(v);
    return dpp_add_d<0x121>(v);
}

// Sums over the tokens first, first + step, ... of every thread of WAVES wavefronts, in thread 0.. of LDS: red[2 E], cnt[E].
template <int E, int WAVES>
struct TokenSums {
    double red[2 * E][WAVES];
    int32_t cnt[E][WAVES];
};
template <int E, int WAVES>
__device__ inline void sum_tokens(const BalanceArgs &a, long first, long step, TokenSums<E, WAVES> &s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double sp[E], sq[E];
    int cnt[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sp[e] = sq[e] = 0.0, cnt[e] = 0;
    for (long t = first; t < a.T; t += step) {
        if (a.valid && a.valid[t] == 0) continue;
        const TokenRouting<E> r = route_token<E>(a.logits + (size_t)t * E, 1.0f / a.noise_std);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sp[e] += (double)r.p[e];
            sq[e] += (double)(0.5f * erfcf(r.z[e] * -0.70710678118654752f));
            cnt[e] += r.first == e ? 1 : 0;
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const double p = wave_sum_d(sp[e]), q = wave_sum_d(sq[e]);
        int c = cnt[e];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
        if (lane == 0) s.red[e][wave] = p, s.red[E + e][wave] = q, s.cnt[e][wave] = c;
    }
    __syncthreads();
}

// The losses and, in coeff, the gradients of the sums of p and of q, from the sums u of alpha p and alpha q (LDS).
template <int E>
__device__ inline void losses_of(const BalanceArgs &a, const double (&u)[2 * E], float (&coeff)[2 * E], bool write) {
    const int i = threadIdx.x, kind = i / E, e = i % E;
    if (i < 2 * E) {
        double sum = 0.0, squares = 0.0, var = 0.0;
#pragma unroll
        for (int k = 0; k < E; ++k) sum += u[kind * E + k], squares += u[kind * E + k] * u[kind * E + k];
        const double m = sum / E;
#pragma unroll
        for (int k = 0; k < E; ++k) var += (u[kind * E + k] - m) * (u[kind * E + k] - m);
        const bool none = m == 0.0;
        coeff[i] = none ? 0.0f : (float)(2.0 / (E * m * m) * (u[i] - squares / sum) * (double)a.alpha[e] * (double)a.dlosses[kind]);
        if (write) {
            if (e == 0) a.losses[kind] = none ? 0.0f : (float)(var / E / (m * m));
            if (a.sums) a.sums[i] = (float)u[i];
        }
    }
}

template <int E>
__device__ inline void grad_tokens(const BalanceArgs &a, long first, long step, const float (&coeff)[2 * E]) {
    const float peak = 0.39894228040143268f / a.noise_std;
    float c[E], f0[E];
#pragma unroll
    for (int e = 0; e < E; ++e) c[e] = coeff[e], f0[e] = coeff[E + e] * peak;
    for (long t = first; t < a.T; t += step) {
        float *dl = a.dlogits + (size_t)t * E;
        if (a.valid && a.valid[t] == 0) {
            if (!a.accumulate) {
#pragma unroll
                for (int e = 0; e < E; ++e) dl[e] = 0.0f;
            }
            continue;
        }
        const TokenRouting<E> r = route_token<E>(a.logits + (size_t)t * E, 1.0f / a.noise_std);
        float up[E], to_first = 0.0f, to_second = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float f = f0[e] * expf(-0.5f * r.z[e] * r.z[e]);
            up[e] = c[e] + f;
            to_second -= e == r.first ? f : 0.0f;
            to_first -= e == r.first ? 0.0f : f;
        }
        float mean = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            up[e] += e == r.first ? to_first : e == r.second ? to_second : 0.0f;
            mean = __builtin_fmaf(r.p[e], up[e], mean);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = r.p[e] * (up[e] - mean);
            dl[e] = a.accumulate ? dl[e] + d : d;
        }
    }
}

constexpr int kSumThreads = 512, kSumWaves = kSumThreads / 64, kMaxSumParts = 256, kMaxGradBlocks = 512;
constexpr int kOneThreads = 1024;
constexpr long kOneLogits = 2048;        // up to this many, all of it in one workgroup

template <int E>
__global__ __launch_bounds__(kSumThreads) void balance_sums_kernel(BalanceArgs a) {
    __shared__ TokenSums<E, kSumWaves> s;
    sum_tokens<E, kSumWaves>(a, (long)blockIdx.x * kSumThreads + threadIdx.x, (long)a.parts * kSumThreads, s);
    const int i = threadIdx.x;
    if (i < 2 * E) {
        double v = 0.0;
        for (int w = 0; w < kSumWaves; ++w) v += s.red[i][w];
        a.partial[(size_t)i * a.parts + blockIdx.x] = v;
    } else if (i < 3 * E) {
        int c = 0;
        for (int w = 0; w < kSumWaves; ++w) c += s.cnt[i - 2 * E][w];
        a.partial_counts[(size_t)(i - 2 * E) * a.parts + blockIdx.x] = c;
    }
}

// Every workgroup adds up the parts (a few KB out of the caches) rather than wait for a launch that does.
template <int E>
__global__ __launch_bounds__(kSumThreads) void balance_grad_kernel(BalanceArgs a) {
    __shared__ double u[2 * E];
    __shared__ float coeff[2 * E];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int v = wave; v < 3 * E; v += kSumWaves) {
        if (v < 2 * E) {
            double sum = 0.0;
            for (int k = lane; k < a.parts; k += 64) sum += a.partial[(size_t)v * a.parts + k];
            sum = wave_sum_d(sum);
            if (lane == 0) u[v] = sum * (double)a.alpha[v % E];
        } else if (blockIdx.x == 0 && a.counts) {
            int c = 0;
            for (int k = lane; k < a.parts; k += 64) c += a.partial_counts[(size_t)(v - 2 * E) * a.parts + k];
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
            if (lane == 0) a.counts[v - 2 * E] = c;
        }
    }
    __syncthreads();
    losses_of<E>(a, u, coeff, blockIdx.x == 0);
    __syncthreads();
    grad_tokens<E>(a, (long)blockIdx.x * kSumThreads + threadIdx.x, (long)gridDim.x * kSumThreads, coeff);
}

template <int E>
__global__ __launch_bounds__(kOneThreads) void balance_one_kernel(BalanceArgs a) {
    __shared__ TokenSums<E, kOneThreads / 64> s;
    __shared__ double u[2 * E];
    __shared__ float coeff[2 * E];
    sum_tokens<E, kOneThreads / 64>(a, threadIdx.x, kOneThreads, s);
    const int i = threadIdx.x;
    if (i < 2 * E) {
        double v = 0.0;
        for (int w = 0; w < kOneThreads / 64; ++w) v += s.red[i][w];
        u[i] = v * (double)a.alpha[i % E];
    } else if (i < 3 * E && a.counts) {
        int c = 0;
        for (int w = 0; w < kOneThreads / 64; ++w) c += s.cnt[i - 2 * E][w];
        a.counts[i - 2 * E] = c;
    }
    __syncthreads();
    losses_of<E>(a, u, coeff, true);
    __syncthreads();
    grad_tokens<E>(a, threadIdx.x, kOneThreads, coeff);
}

int balance_parts(long T) {
    const long parts = (T + kSumThreads - 1) / kSumThreads;
    return (int)(parts < kMaxSumParts ? parts : kMaxSumParts);
}
size_t balance_workspace(long T) { return (size_t)balance_parts(T) * kMaxE * (2 * 8 + 4) + 256; }

template <int E>
int launch_balance(const BalanceArgs &a, hipStream_t st) {
    if (a.T * E <= kOneLogits) {
        balance_one_kernel<E><<<dim3(1), dim3(kOneThreads), 0, st>>>(a);
        return check_launch("sa_moe_balance_loss_grad(one launch)");
    }
    balance_sums_kernel<E><<<dim3((unsigned)a.parts), dim3(kSumThreads), 0, st>>>(a);
    const int rc = check_launch("sa_moe_balance_loss_grad(sums)");
    if (rc != SA_OK) return rc;
    const long blocks = (a.T + kSumThreads - 1) / kSumThreads;
    balance_grad_kernel<E><<<dim3((unsigned)(blocks < kMaxGradBlocks ? blocks : kMaxGradBlocks)), dim3(kSumThreads), 0, st>>>(a);
    return check_launch("sa_moe_balance_loss_grad(gradient)");
}

// f(std::integral_constant<int, E>()) for E experts.
template <class F>
int by_experts(int E, F &&f) {
    switch (E) {
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 4: return f(std::integral_constant<int, 4>());
        case 5: return f(std::integral_constant<int, 5>());
        case 6: return f(std::integral_constant<int, 6>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, kMaxE>());
    }
}

struct CombineGradArgs {
    const void *dy, *src;
    RowSel sel;
    const float *gate, *logits;
    int n, E;
    void *dsrc;
    float *dgate, *dlogits;
};

// Maximum over aligned groups of 16 lanes.
__device__ inline float max16(float v) {
#define SA_MAX_STEP(CTRL) \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)))
    SA_MAX_STEP(0x128);
    SA_MAX_STEP(0x124);
    SA_MAX_STEP(0x122);
    SA_MAX_STEP(0x121);
#undef SA_MAX_STEP
    return v;
}

// 16 to 64 lanes to a row, which they walk over in blocks of S::COLUMNS columns; an expert of its routing to a lane.
template <class Y, class X, class S>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
    constexpr int VEC = S::VEC, CH = S::CH;
    const int32_t *rows;
    long n_rows;
    resolve_rows(a.sel, rows, n_rows);
    const int g = threadIdx.x / S::LANES, l = threadIdx.x % S::LANES;
    const bool dot = a.dgate || a.dlogits;
    const long stride = (long)gridDim.x * S::GROUPS;
    for (long i = (long)blockIdx.x * S::GROUPS + g; i < n_rows; i += stride) {
        const size_t r = rows ? (size_t)rows[i] : (size_t)i;
        const float gate = a.gate ? a.gate[r] : 1.0f;
        const Y *dy = static_cast<const Y *>(a.dy) + r * a.E;
        const X *src = static_cast<const X *>(a.src) + (size_t)i * a.E;
        X *dsrc = static_cast<X *>(a.dsrc) + (size_t)i * a.E;
        float s = 0.0f;
        for (int j0 = 0; j0 < a.E; j0 += S::COLUMNS) {
            Piece<Y, VEC> d[CH];
            Piece<X, VEC> v[CH];
            int at[CH], skip[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j = j0 + (c * S::LANES + l) * VEC;
                at[c] = j + VEC <= a.E ? j : a.E - VEC;
                skip[c] = j - at[c];
                d[c].load(dy + at[c]);
                if (dot) v[c].load(src + at[c]);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float out[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    if (dot) s = k >= skip[c] ? __builtin_fmaf(d[c][k], v[c][k], s) : s;
                    out[k] = gate * d[c][k];
                }
                // elements that two lanes hold are written by both, the same bits
                if (a.dsrc) store_piece<X, VEC>(dsrc + at[c], out);
            }
        }
        if (!dot) continue;
        s = group_sum<S::LANES>(s);
        if (a.dgate && l == 0) a.dgate[r] = s;
        if (a.dlogits) {
            // p_first = 1 / den, the largest exponent being 0
            const float v = l < a.n ? a.logits[r * a.n + l] : -__builtin_inff();
            const float top = max16(v);
            const uint64_t best = __ballot(l < a.n && v == top) >> (threadIdx.x & 63 & ~(S::LANES - 1));
            const float e = l < a.n ? expf(v - top) : 0.0f;
            const float inv = 1.0f / group_sum<16>(e);
            if (l < a.n) a.dlogits[r * a.n + l] = s * inv * ((l == __ffsll((unsigned long long)(best & 0xFFFF)) - 1 ? 1.0f : 0.0f) - e * inv);
        }
    }
}

template <class Y, class X>
struct RunCombineGrad {
    static int run(const CombineGradArgs &a, hipStream_t st) {
        constexpr int VEC = row_vec<Y, X>();
        auto rows = [&](auto shape) {
            using S = decltype(shape);
            // 8 workgroups to a CU; the rows there are may be fewer than max_rows
            const long blocks = (a.sel.max_rows + S::GROUPS - 1) / S::GROUPS;
            combine_grad_kernel<Y, X, S><<<dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st>>>(a);
            return check_launch("sa_combine_rows_backward");
        };
        if (a.E < VEC) return rows(RowShape<1, 1, 16, 0>());
        if (a.E <= 16 * VEC) return rows(RowShape<VEC, 1, 16, 0>());
        if (a.E <= 32 * VEC) return rows(RowShape<VEC, 1, 32, 0>());
        if (a.E <= 64 * VEC) return rows(RowShape<VEC, 1, 64, 0>());
        return rows(RowShape<VEC, 8 / VEC, 64, 0>());
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
    BalanceArgs a{logits, T, valid_or_null, alpha, noise_std, dlosses, losses, sums_or_null, counts_or_null, dlogits, accumulate};
    a.parts = balance_parts(T);
    a.partial = static_cast<double *>(workspace);
    a.partial_counts = reinterpret_cast<int32_t *>(a.partial + (size_t)a.parts * 2 * kMaxE);
    return by_experts(E, [&](auto experts) { return launch_balance<decltype(experts)::value>(a, sa::as_stream(stream)); });
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
