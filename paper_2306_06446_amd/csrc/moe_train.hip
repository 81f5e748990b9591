// What trains the router: the balance loss of Eq. 4 with its gradient and the tokens of each expert, and the gradient of the gated
// combine behind a top-1 dispatch (Sec. 4.2).
//
//   p = softmax(l), o(i) the best expert but i, d_i = (p_i - p_o(i)) / std, q_i = Phi(d_i)
//   u_i = alpha_i sum_t p_i, v_i = alpha_i sum_t q_i, losses SCV(u), SCV(v), SCV(u) = mean((u - m)^2) / m^2, m = mean(u)
//   dSCV / du_i = 2 (u_i - sum u^2 / sum u) / (n m^2)
//   with c and f the gradients of the sums of p and q:  a = c + J^T (f phi(d) / std),  J p_i = p_i - p_o(i),  dl = p (a - <p, a>)
//
// The loss: every token's gradient needs the sums over all tokens, so logits are read twice, the second time out of the caches: a launch
// that leaves sums of up to 512 parts in fp64, and one of which every workgroup adds those up.  What bounds it: latency.  A million tokens of
// two experts 11.1 us (16 MB, 3.1 us at a copy's rate), 5.8 and 7.0 of the two launches on the device: some 5 are what two launches take in any
// case, the rest is four tokens to a thread one behind the other, with one ahead under way.  131072 of eight 10.3, one token to a thread, of
// which the instructions of 8 exponentials, distributions and densities are some 3.  Up to 1024 tokens one workgroup does all of it: 2.7 us on
// the device (two launches: 7).
//
// The combine's gradient: one pass, a dot product and a product a row.  What bounds it: memory, 12608 x 768 fp16 under fp32 14.6 us
// (5.3 TB/s), 50021 x 500 bf16, rows of 1000 bytes in the dispatch's order, 29.9 (5.1); fp32 throughout, as the experts here leave it,
// 12608 x 768 23.9 (4.9), 131072 x 1024 292 (5.5).
#include <type_traits>

#include "common.h"
#include "row_types.h"

namespace {

using namespace sa;

constexpr int kMaxE = kMaxExperts;

// exp(x), x <= 0, off by 2 units at most down to the smallest normal number, 0 below it and for -infinity (what a softmax loses by that is
// 1e-38), NaN for NaN: 2^t of the rounded product t = x / ln 2, and the product's rounding to first order.  Half of expf's instructions.
__device__ inline float exp_of(float x) {
    x = x < -104.0f ? -104.0f : x;
    const float t = x * 1.44269504f, r = __builtin_fmaf(x, 1.92596303e-8f, __builtin_fmaf(x, 1.44269504f, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e * 0.693147181f, r, e);
}
// exp(-z^2 / 2): the exponent's two roundings are z^2 of 2^-24 relative to the result, which is 0.74 of 2^-24 absolutely (at z^2 = 2); the
// instruction's own unit makes it 1.8 of 2^-24 at most.
__device__ inline float exp_minus_half_square(float z) { return __builtin_amdgcn_exp2f(z * z * -0.72134752f); }

// A token's routing: p, and for each expert the normal deviate of its distance to the best of the others.
template <int E>
struct TokenRouting {
    float p[E], z[E];
    int first, second;                   // largest and second largest logit, ties to the lowest index
};

template <int E>
__device__ inline TokenRouting<E> route_token(const float (&v)[E], float inv_noise_std) {
    TokenRouting<E> r;
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
    // of two experts, the largest one's exponential is 1; where it is infinite, l0 - l0 is the NaN that a softmax has there
    float den = E == 2 ? l0 - l0 : 0.0f;
    const float x1 = exp_of(l1 - l0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        r.p[e] = E == 2 ? (e == r.first ? 1.0f : x1) : exp_of(v[e] - l0);
        den += r.p[e];
    }
    const float p0 = __builtin_amdgcn_rcpf(den), p1 = x1 * p0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        r.p[e] *= p0;
        r.z[e] = (r.p[e] - (e == r.first ? p1 : p0)) * inv_noise_std;
    }
    return r;
}

// Phi(-|z|): exp(z^2 / 2) Phi(-z) is smooth and is t times a polynomial in t = 1 / (1 + 0.34 z), up to 2.7e-8 of itself for all z to 13.6
// (an exchange of extrema of the relative error against erfcx in fp64), behind which the result is no normal number.  A LOAD of distant
// tails alone is thus right relative to itself.  On the device, for all z to 13: off by (z^2 + 6.1) of 2^-24 relative to itself, by 1.7e-7 (2.9
// of 2^-24) at most; for z to 5 the mean error is -1.3e-9, the mean magnitude 6.5e-9.
// A library erfc takes five times the instructions, its two branches both, and was most of the sums' time.
__device__ inline float normal_tail(float z) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.34f, fabsf(z), 1.0f));
    float p = -0.0263198148f;
    p = __builtin_fmaf(p, t, 0.14043504f);
    p = __builtin_fmaf(p, t, -0.274990708f);
    p = __builtin_fmaf(p, t, 0.204215586f);
    p = __builtin_fmaf(p, t, -0.0460543782f);
    p = __builtin_fmaf(p, t, 0.115897283f);
    p = __builtin_fmaf(p, t, 0.115068316f);
    p = __builtin_fmaf(p, t, 0.136129111f);
    p = __builtin_fmaf(p, t, 0.135619581f);
    return exp_minus_half_square(z) * (p * t);
}

struct BalanceArgs {
    const float *logits;
    long T;
    const uint8_t *valid;
    const float *alpha;
    float inv_noise_std, peak;           // 1 / std, 1 / (sqrt(2 pi) std)
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

// Of two values: the upper half of a's lanes (rows) and the lower half of b's change places, and the sum is taken: sums of a in the
// lower half, of b in the upper one.
template <bool ROWS>
__device__ inline double swap_add_d(double a, double b) {
    const uint64_t u = __builtin_bit_cast(uint64_t, a), w = __builtin_bit_cast(uint64_t, b);
    const auto lo = ROWS ? __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)w, false, false)
                         : __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)w, false, false);
    const auto hi = ROWS ? __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(w >> 32), false, false)
                         : __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(w >> 32), false, false);
    return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}

// Sum over a row of 16 lanes in all of them.
__device__ inline double row_sum_d(double v) {
    v = dpp_add_d<0x128>(v);
    v = dpp_add_d<0x124>(v);
    v = dpp_add_d<0x122>(v);
    return dpp_add_d<0x121>(v);
}
__device__ inline double wave_sum_d(double v) { return row_sum_d(swap_add_d<true>(swap_add_d<false>(v, v), swap_add_d<false>(v, v))); }

// N sums over a wavefront at once, to out[k][wave]: four of them share the steps within rows of lanes, one to each.
template <int N, int WAVES>
__device__ inline void wave_sums_d(const double (&v)[N], double (*out)[WAVES], int lane, int wave) {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const double a = v[k], b = v[k + 1 < N ? k + 1 : k], c = v[k + 2 < N ? k + 2 : k], d = v[k + 3 < N ? k + 3 : k];
        // rows 0 and 1 of lanes: a and b; rows 2 and 3: c and d
        const double s = row_sum_d(swap_add_d<true>(swap_add_d<false>(a, c), swap_add_d<false>(b, d)));
        const int at = k + (lane >> 4);
        if ((lane & 15) == 0 && at < N) out[at][wave] = s;
    }
}

// A thread's share of the sums, tokens added one by one; counts are a wavefront's.
template <int E>
struct TokenSums {
    double v[2 * E];
    int cnt[E];
    __device__ inline TokenSums() {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = v[E + e] = 0.0, cnt[e] = 0;
    }
    __device__ inline void add(const TokenRouting<E> &r, bool in) {
        const float both = E == 2 ? normal_tail(r.z[0]) : 0.0f;          // of two experts, z has two signs
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float tail = E == 2 ? both : normal_tail(r.z[e]), q = e == r.first ? 1.0f - tail : tail;
            v[e] += in ? (double)r.p[e] : 0.0;
            v[E + e] += in ? (double)q : 0.0;
            cnt[e] += __popcll(__ballot(in && r.first == e));
        }
    }
};

// Workgroup's sums in LDS, a value to a wavefront.
template <int E, int WAVES>
struct GroupSums {
    double v[2 * E][WAVES];
    int32_t cnt[E][WAVES];
    __device__ inline void leave(const TokenSums<E> &s) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        wave_sums_d<2 * E, WAVES>(s.v, v, lane, wave);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane == 0) cnt[e][wave] = s.cnt[e];
        __syncthreads();
    }
    __device__ inline double sum(int i) const {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += v[i][w];
        return s;
    }
    __device__ inline int count(int e) const {
        int c = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c += cnt[e][w];
        return c;
    }
};

// A token as it is asked for: what of its logits and its place in the batch can be had before anything is known of the others.  No load
// waits for another one's outcome: tokens that are not there read the first one's.
template <int E>
struct Token {
    float l[E], old[E];                  // old: what the gradient is added to
    bool valid;
    __device__ inline void load(const BalanceArgs &a, long t, bool accumulate) {
        const bool there = t < a.T;
        const size_t at = there ? (size_t)t : 0;
        const uint8_t *mask = a.valid ? a.valid : reinterpret_cast<const uint8_t *>(a.logits);
        const uint8_t v = mask[at];
#pragma unroll
        for (int e = 0; e < E; ++e) l[e] = a.logits[at * E + e];
        if (accumulate) {
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] = a.dlogits[at * E + e];
        }
        valid = there && (!a.valid || v != 0);
    }
};

// What the losses are made of, in LDS; alpha and the losses' weights are asked for before the sums are there.
template <int E>
struct Losses {
    double sum[2 * E];                   // over tokens, of p and of q
    float alpha[E], weight[2], coeff[2 * E];     // coeff: gradients of the sums

    // asks; what came is put down by put, before a barrier
    struct Asked {
        float alpha, weight;
    };
    static __device__ inline Asked ask(const BalanceArgs &a) {
        const int i = threadIdx.x < E ? (int)threadIdx.x : 0;
        return {a.alpha[i], a.dlosses[i & 1]};
    }
    __device__ inline void put(const Asked &x) {
        if (threadIdx.x < E) alpha[threadIdx.x] = x.alpha;
        if (threadIdx.x < 2) weight[threadIdx.x] = x.weight;
    }
    // behind a barrier; another one before coeff is read
    __device__ inline void end(const BalanceArgs &a, bool write) {
        const int i = threadIdx.x, kind = i / E, e = i % E;
        if (i >= 2 * E) return;
        double u[E], total = 0.0, squares = 0.0, var = 0.0, mine = 0.0;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            u[k] = sum[kind * E + k] * (double)alpha[k];
            total += u[k], squares += u[k] * u[k];
            mine = k == e ? u[k] : mine;
        }
        const double m = total / E;
#pragma unroll
        for (int k = 0; k < E; ++k) var += (u[k] - m) * (u[k] - m);
        const double inv = 1.0 / (m * m * E);
        const bool none = m == 0.0;
        coeff[i] = none ? 0.0f : (float)(2.0 * inv * (mine - squares / total) * (double)alpha[e] * (double)weight[kind]);
        if (write) {
            if (e == 0) a.losses[kind] = none ? 0.0f : (float)(var * inv);
            if (a.sums) a.sums[i] = (float)mine;
        }
    }
};

template <int E>
__device__ inline void grad_token(const BalanceArgs &a, long t, const Token<E> &x, const TokenRouting<E> &r, const float (&density)[E],
                                  const float (&coeff)[2 * E]) {
    float *dl = a.dlogits + (size_t)t * E;
    float up[E], to_first = 0.0f, to_second = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float f = coeff[E + e] * density[e];
        up[e] = coeff[e] + f;
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
        const float d = r.p[e] * (up[e] - mean), none = a.accumulate ? x.old[e] : 0.0f;
        up[e] = !x.valid ? none : a.accumulate ? x.old[e] + d : d;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) dl[e] = up[e];
}

template <int E>
__device__ inline void densities(const TokenRouting<E> &r, float peak, float (&out)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = peak * exp_minus_half_square(r.z[e]);
}

static_assert(kMaxE <= 8, "an expert to a wavefront of the sums");
constexpr int kSumThreads = 512, kSumWaves = kSumThreads / 64, kMaxGradBlocks = 512;
// Two workgroups to a CU, but one for many experts: every workgroup of the gradient reads 2 E sums of each part.
constexpr int max_sum_parts(int E) { return E <= 4 ? 512 : 256; }
constexpr int kOneThreads = 1024;        // up to as many tokens, all of it in one workgroup

template <int E>
__global__ __launch_bounds__(kSumThreads) void balance_sums_kernel(BalanceArgs a) {
    __shared__ GroupSums<E, kSumWaves> group;
    TokenSums<E> s;
    const long step = (long)gridDim.x * kSumThreads;
    Token<E> nxt;
    long t0 = (long)blockIdx.x * kSumThreads;
    nxt.load(a, t0 + threadIdx.x, false);
    for (; t0 < a.T; t0 += step) {
        const Token<E> x = nxt;
        nxt.load(a, t0 + step + threadIdx.x, false);
        s.add(route_token<E>(x.l, a.inv_noise_std), x.valid);
    }
    group.leave(s);
    const int i = threadIdx.x;
    if (i < 2 * E) a.partial[(size_t)i * a.parts + blockIdx.x] = group.sum(i);
    else if (i < 3 * E) a.partial_counts[(size_t)(i - 2 * E) * a.parts + blockIdx.x] = group.count(i - 2 * E);
}

// Every workgroup adds up the parts (a few KB out of the caches) rather than wait for a launch that does; its first tokens' routing is
// computed while they are on the way.
template <int E>
__global__ __launch_bounds__(kSumThreads) void balance_grad_kernel(BalanceArgs a) {
    __shared__ Losses<E> losses;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kEach = max_sum_parts(E) / 64, kMine = (2 * E + kSumWaves - 1) / kSumWaves;
    const auto asked = Losses<E>::ask(a);
    double part[kMine][kEach];
#pragma unroll
    for (int m = 0; m < kMine; ++m)
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int v = wave + m * kSumWaves, at = lane + 64 * k;
            part[m][k] = a.partial[(size_t)(v < 2 * E ? v : 0) * a.parts + (at < a.parts ? at : 0)];
        }
    // the first workgroup adds up the counts, an expert to a wavefront
    const bool counting = blockIdx.x == 0 && a.counts && wave < E;
    int counted[kEach] = {};
    if (counting) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int at = lane + 64 * k;
            counted[k] = a.partial_counts[(size_t)wave * a.parts + (at < a.parts ? at : 0)];
        }
    }
    const long step = (long)gridDim.x * kSumThreads;
    long t = (long)blockIdx.x * kSumThreads + threadIdx.x;
    Token<E> x;
    x.load(a, t, a.accumulate);
    TokenRouting<E> r = route_token<E>(x.l, a.inv_noise_std);
    float density[E], coeff[2 * E];
    densities<E>(r, a.peak, density);
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        const int v = wave + m * kSumWaves;
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) s += lane + 64 * k < a.parts ? part[m][k] : 0.0;
        s = wave_sum_d(s);
        if (lane == 0 && v < 2 * E) losses.sum[v] = s;
    }
    losses.put(asked);
    if (counting) {
        int c = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) c += lane + 64 * k < a.parts ? counted[k] : 0;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
        if (lane == 0) a.counts[wave] = c;
    }
    __syncthreads();
    losses.end(a, blockIdx.x == 0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * E; ++i) coeff[i] = losses.coeff[i];
    while (t < a.T) {
        const Token<E> now = x;
        x.load(a, t + step, a.accumulate);
        grad_token<E>(a, t, now, r, density, coeff);
        t += step;
        if (t >= a.T) break;
        r = route_token<E>(x.l, a.inv_noise_std);
        densities<E>(r, a.peak, density);
    }
}

template <int E>
__global__ __launch_bounds__(kOneThreads) void balance_one_kernel(BalanceArgs a) {
    __shared__ GroupSums<E, kOneThreads / 64> group;
    __shared__ Losses<E> losses;
    const auto asked = Losses<E>::ask(a);
    Token<E> x;
    if (a.T > 0) x.load(a, threadIdx.x, a.accumulate);
    else x = Token<E>{};
    const TokenRouting<E> r = route_token<E>(x.l, a.inv_noise_std);
    TokenSums<E> s;
    s.add(r, x.valid);
    losses.put(asked);
    group.leave(s);
    const int i = threadIdx.x;
    if (i < 2 * E) losses.sum[i] = group.sum(i);
    else if (i < 3 * E && a.counts) a.counts[i - 2 * E] = group.count(i - 2 * E);
    __syncthreads();
    losses.end(a, true);
    __syncthreads();
    if (threadIdx.x >= a.T) return;
    float density[E], coeff[2 * E];
    densities<E>(r, a.peak, density);
#pragma unroll
    for (int k = 0; k < 2 * E; ++k) coeff[k] = losses.coeff[k];
    grad_token<E>(a, threadIdx.x, x, r, density, coeff);
}

int balance_parts(long T, int E) {
    const long parts = (T + kSumThreads - 1) / kSumThreads, most = max_sum_parts(E);
    return (int)(parts < most ? parts : most);
}
size_t balance_workspace(long T, int E) { return (size_t)balance_parts(T, E) * kMaxE * (2 * 8 + 4) + 256; }

template <int E>
int launch_balance(const BalanceArgs &a, hipStream_t st) {
    if (a.T <= kOneThreads) {
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

// 16 to 64 lanes to a row, which they walk over in blocks of columns; an expert of its routing to a lane.
template <class Y, class X, class S>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
    constexpr int VEC = S::VEC, CH = S::CH, GROUPS = 256 / S::LANES, COLUMNS = S::LANES * VEC * CH;
    const int32_t *rows;
    long n_rows;
    resolve_rows(a.sel, rows, n_rows);
    const int g = threadIdx.x / S::LANES, l = threadIdx.x % S::LANES;
    const bool dot = a.dgate || a.dlogits;
    const long stride = (long)gridDim.x * GROUPS;
    for (long i = (long)blockIdx.x * GROUPS + g; i < n_rows; i += stride) {
        const size_t r = rows ? (size_t)rows[i] : (size_t)i;
        const float gate = a.gate ? a.gate[r] : 1.0f;
        const Y *dy = static_cast<const Y *>(a.dy) + r * a.E;
        const X *src = static_cast<const X *>(a.src) + (size_t)i * a.E;
        X *dsrc = static_cast<X *>(a.dsrc) + (size_t)i * a.E;
        double blocks = 0.0;                 // a sum in fp32 loses what it is given once it has grown
        for (int j0 = 0; j0 < a.E; j0 += COLUMNS) {
            float s = 0.0f;
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
                if (a.dsrc) stream_piece<X, VEC>(dsrc + at[c], out);
            }
            blocks += (double)s;
        }
        if (!dot) continue;
        const float s = group_sum<S::LANES>((float)blocks);
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
            const long blocks = (a.sel.max_rows + 256 / S::LANES - 1) / (256 / S::LANES);
            combine_grad_kernel<Y, X, S><<<dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st>>>(a);
            return check_launch("sa_combine_rows_backward");
        };
        if (a.E < VEC) return rows(RowShape<1, 1, 16, 0>());
        // with 8 elements to a lane, half of the lanes or more would repeat what others do: 10^6 x 64 fp16 112 -> 109 us, 300000 x 17 28.7 -> 23.8
        if constexpr (VEC == 8)
            if (a.E <= 64) return rows(RowShape<4, 1, 16, 0>());
        if (a.E <= 16 * VEC) return rows(RowShape<VEC, 1, 16, 0>());
        if (a.E <= 32 * VEC) return rows(RowShape<VEC, 1, 32, 0>());
        if (a.E <= 64 * VEC) return rows(RowShape<VEC, 1, 64, 0>());
        return rows(RowShape<VEC, 8 / VEC, 64, 0>());
    }
};

}  // namespace

extern "C" size_t sa_moe_balance_loss_grad_workspace_bytes(long T, int E) {
    if (T < 0 || T >= (1L << 31) || E < 2 || E > kMaxE) return 0;
    return balance_workspace(T, E);
}

extern "C" int sa_moe_balance_loss_grad(const float *logits, long T, int E, const uint8_t *valid_or_null, const float *alpha,
                                        float noise_std, const float *dlosses, float *losses, float *sums_or_null,
                                        int32_t *counts_or_null, float *dlogits, int accumulate, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    sa::clear_error();
    SA_REQUIRE(T >= 0, SA_ERR_INVALID, "sa_moe_balance_loss_grad: T < 0");
    SA_REQUIRE(T < (1L << 31), SA_ERR_SHAPE, "sa_moe_balance_loss_grad: T >= 2^31");
    SA_REQUIRE(E >= 2 && E <= kMaxE, SA_ERR_SHAPE, "sa_moe_balance_loss_grad: 2 to 8 experts (got %d)", E);
    SA_REQUIRE(noise_std > 0.0f && __builtin_isfinite(noise_std) && __builtin_isfinite(1.0f / noise_std), SA_ERR_INVALID,
               "sa_moe_balance_loss_grad: noise_std must be positive and finite, and so must its reciprocal");
    SA_REQUIRE(alpha && dlosses && losses && (T == 0 || (logits && dlogits)), SA_ERR_INVALID, "sa_moe_balance_loss_grad: NULL buffer");
    SA_REQUIRE(sa::aligned16(logits) && sa::aligned16(valid_or_null) && sa::aligned16(alpha) && sa::aligned16(dlosses) &&
                   sa::aligned16(losses) && sa::aligned16(sums_or_null) && sa::aligned16(counts_or_null) && sa::aligned16(dlogits) &&
                   sa::aligned16(workspace),
               SA_ERR_ALIGN, "sa_moe_balance_loss_grad: pointers must be 16-byte aligned");
    const size_t need = balance_workspace(T, E);
    SA_REQUIRE(workspace != nullptr && workspace_bytes >= need, SA_ERR_WORKSPACE,
               "sa_moe_balance_loss_grad: workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    BalanceArgs a{logits, T, valid_or_null, alpha, 1.0f / noise_std, 0.39894228040143268f / noise_std, dlosses, losses, sums_or_null, counts_or_null, dlogits, accumulate};
    a.parts = balance_parts(T, E);
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
    SA_REQUIRE(E > 0 && E <= (1 << 30), SA_ERR_SHAPE, "sa_combine_rows_backward: E must be positive and at most 2^30");
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
