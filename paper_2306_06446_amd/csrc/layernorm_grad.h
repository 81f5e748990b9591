// The gradient of LayerNorm with the residual's and the router's (layernorm_train.hip has the formulas): one pass over the rows.
//
// A row's two sums need all of it, a column's sums all rows: lanes keep their columns' sums in registers while rows go by, a workgroup adds
// those of its wavefronts up in LDS, and what it leaves (a part: 2 + n rows of E sums) a second launch adds up in fp64.  One workgroup to a
// CU, or two of wide rows, so that parts are few: they are written and read again.  Where a lane would add up more than 512 rows, a sum in fp32
// loses what it is given once it has grown: launches of ranges of rows instead, each with its parts.  (More parts in one launch go over the
// rows in as many strides: 2^25 x 64 fp16 3.14 -> 3.68 ms, in ranges 2.98; 300000 x 2500 bf16
// with three experts, whose parts are twice as many, 2.03 -> 2.08.)
// What bounds it: memory once rows are many (x, dy, dres in, dx out: 131072 x 1024 bf16 189 us, 5.7 TB/s; 25000 x 4000 bf16 150, 5.3;
// 12608 x 768 fp16 under fp32 with the router of two 30.7 us, 4.4 TB/s over both launches).  Few rows: the two
// launches' latency, 197 x 192 4.6 + 3.6 us on the device.  Without statistics, which then are sums more over the row in hand, the same: 131072 x
// 1024 189 us, 12608 x 768 34.0 against 34.1 with others' rows in the caches; 10 % more behind many experts.
// Routers of 3 to 8 experts keep 8 elements to a lane (12608 x 768 54 us: no row ahead, and two wavefronts to a
// SIMD); beyond 2048 columns the weights come from the caches for every row (20000 x 8000 bf16 with eight 510 to 550 us,
// of which dx 420, bound by the 256 KB of weights a row, their sums 87, the parts 28).
#pragma once

#include "layernorm_train.h"

namespace sa {

// Rows of which more are read than half of the memory-side cache are not worth a place in the caches: they cannot all be there from the
// launches before, and this is their last use.  131072 x 1024 bf16 (805 MB read) 203 -> 189 us, 131072 x 200 bf16 (157 MB) 50.3 -> 49.4; but
// 12608 x 768 (97 MB, partly there) 30.8 -> 32.8 and 7000 x 300 fp32 (25 MB) 12.5 -> 14.5.
constexpr size_t kLargeRows = 128ull << 20;

// What a lane holds of a row that is to come: asked for while the row before it is worked on.
template <class X, class Y, class S, int ROUTE, bool LARGE>
struct GradRow {
    Piece<Y, S::VEC> dy[S::CH];
    Piece<X, S::VEC> x[S::CH], res[S::CH];
    float mean, rstd, dl[ROUTE ? ROUTE : 1];

    __device__ inline void load(const NormGradArgs &a, const RowPlace<S> &p, long t) {
        const size_t row = (size_t)t * a.E;
        auto fetch = [](auto &piece, const auto *from) {
            if constexpr (LARGE) piece.stream(from);
            else piece.load(from);
        };
#pragma unroll
        for (int c = 0; c < S::CH; ++c) {
            fetch(dy[c], static_cast<const Y *>(a.dy) + row + p.at[c]);
            fetch(x[c], static_cast<const X *>(a.x) + row + p.at[c]);
        }
        if (a.dres) {
#pragma unroll
            for (int c = 0; c < S::CH; ++c) fetch(res[c], static_cast<const X *>(a.dres) + row + p.at[c]);
        }
        if (a.mean) mean = a.mean[t], rstd = a.rstd[t];
        if constexpr (ROUTE > kStreamed) {
#pragma unroll
            for (int e = 0; e < ROUTE; ++e) {
                const bool in = ROUTE == 2 || e < a.n;
                const float v = a.dlogits[(size_t)t * a.n + (in ? e : 0)];
                dl[e] = in ? v : 0.0f;
            }
        }
    }
};

// A lane's registers, in all: the sums and parameters of its columns, and a row with its normalised values; with another row under way where
// that stays within two wavefronts to a SIMD (AHEAD).  Three wavefronts to a SIMD for rows that would fit were slower (131072 x 1024 bf16
// 205 -> 218 us), workgroups of four wavefronts and twice the parts for narrow rows too (12608 x 768 34.5 -> 35.3).
template <class X, class Y, class S, int ROUTE>
struct GradPlan {
    static constexpr int HELD = ROUTE > kStreamed ? ROUTE : 0;
    static constexpr int ELEMS = S::VEC * S::CH;
    static constexpr int ROW = ELEMS * (2 * sizeof(X) + sizeof(Y)) / 4;
    static constexpr int REGISTERS = ELEMS * (2 + HELD + 1 + HELD + 2) + 2 * (ROW + HELD) + 48;
    static constexpr bool AHEAD = REGISTERS < 256;
    // A workgroup to a CU, of the wavefronts that its registers have room for: the fewest parts that keep it busy.  Wavefronts that share
    // rows wait for each other at every row: there in workgroups of four, or a row's, of which a CU has two (25000 x 4000 fp16
    // 129 -> 122 us).
    static constexpr int WAVES = S::WIDE ? 4 : REGISTERS <= 136 ? 16 : 8;
    static constexpr int MOST = S::WIDE ? 8 : WAVES;         // of a workgroup
    static constexpr int SIDE = 64 * WAVES * ELEMS;          // a value to each of its elements, in LDS
    static constexpr int AT_ONCE = SIDE <= 8192 ? 4 : 2;
};

template <class X, class Y, class S, int ROUTE, bool LARGE>
__global__ __launch_bounds__((64 * GradPlan<X, Y, S, ROUTE>::MOST)) void norm_grad_kernel(NormGradArgs a) {
    using Plan = GradPlan<X, Y, S, ROUTE>;
    constexpr int VEC = S::VEC, CH = S::CH, HELD = Plan::HELD, Q = 2 + HELD;
    constexpr bool AHEAD = Plan::AHEAD;
    constexpr int PC = HELD ? CH : 1, PR = HELD ? HELD : 1;
    __shared__ __align__(16) float red[S::WIDE ? 2 : 1][2][8];
    constexpr int BATCH = Q < Plan::AT_ONCE ? Q : Plan::AT_ONCE;
    constexpr int SIDE = HELD == kMaxExperts && kRouterTileFloats > BATCH * Plan::SIDE ? kRouterTileFloats : BATCH * Plan::SIDE;
    __shared__ float side[SIDE], side_dl[64 * Plan::MOST / S::PERIOD][PR];
    const RowPlace<S> p(a.E);
    const int g = p.g, groups = p.groups;
    const float per = 1.0f / (float)a.E;
    RowSums<S, 2> sums(red, p);
    const long stride = (long)gridDim.x * groups;
    auto clamped = [&](long t) { return t < a.T ? t : a.T - 1; };
    GradRow<X, Y, S, ROUTE, LARGE> nxt;
    long t0 = (long)blockIdx.x * groups;
    float gm[CH][VEC], w[PR][PC][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_columns<VEC>(gm[c], a.gamma + p.at[c]);
        if constexpr (HELD == 2) load_router_pair<VEC, PC>(w, c, a.wg + 2 * (size_t)p.at[c]);
    }
    if constexpr (HELD == kMaxExperts) load_router<S, PR>(w, p, a.wg, a.E, a.n, side);
    float acc[Q][CH][VEC], dl_sum[PR];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[q][c][i] = 0.0f;
#pragma unroll
    for (int e = 0; e < PR; ++e) dl_sum[e] = 0.0f;

    auto work = [&](const GradRow<X, Y, S, ROUTE, LARGE> &r, long t, bool row_ok) {
        float mean = r.mean, rstd = r.rstd, s[2];
        if constexpr (S::WIDE) {
            // before the row's first barrier: dx may be in the place of any of them
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                arrived(r.dy[c]);
                arrived(r.x[c]);
                if (a.dres) arrived(r.res[c]);
            }
        }
        if (!a.mean) {
            s[0] = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[0] += p.own(c, i, r.x[c][i]);
            sums(s, 1);
            mean = s[0] * per;
            s[0] = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = p.own(c, i, r.x[c][i] - mean);
                    s[0] = __builtin_fmaf(d, d, s[0]);
                }
            sums(s, 1);
            rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(s[0], per, a.eps));
        }
        float xh[CH][VEC], h[CH][VEC];
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                xh[c][i] = (r.x[c][i] - mean) * rstd;
                h[c][i] = r.dy[c][i];
#pragma unroll
                for (int e = 0; e < HELD; ++e) h[c][i] = __builtin_fmaf(r.dl[e], w[e][HELD ? c : 0][i], h[c][i]);
            }
        if constexpr (ROUTE == kStreamed) {
            const float *dl = a.dlogits + (size_t)clamped(t) * a.n;
#pragma unroll 2
            for (int e = 0; e < a.n; ++e) {
                const float *row = a.weights + (size_t)e * padded_columns(a.E);
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    Piece<float, VEC> v;
                    v.load(row + p.at[c]);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) h[c][i] = __builtin_fmaf(dl[e], v[i], h[c][i]);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float gv = p.own(c, i, h[c][i] * gm[c][i]);
                s[0] += gv;
                s[1] = __builtin_fmaf(gv, xh[c][i], s[1]);
            }
        sums(s);
        if (!row_ok) return;
        const float c0 = s[0] * per, c1 = s[1] * per;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float d[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                acc[0][c][i] = __builtin_fmaf(h[c][i], xh[c][i], acc[0][c][i]);
                acc[1][c][i] += h[c][i];
#pragma unroll
                for (int e = 0; e < HELD; ++e) acc[2 + e][c][i] = __builtin_fmaf(xh[c][i], r.dl[e], acc[2 + e][c][i]);
                d[i] = rstd * (h[c][i] * gm[c][i] - c0 - xh[c][i] * c1);
                if (a.dres) d[i] += r.res[c][i];
            }
            stream_piece<X, VEC>(static_cast<X *>(a.dx) + (size_t)t * a.E + p.at[c], d);
        }
#pragma unroll
        for (int e = 0; e < HELD; ++e) dl_sum[e] += r.dl[e];
    };
    // Every step stores the same number of pieces: a wait for the next row then leaves the last row's stores in flight (loads and stores
    // are counted by one counter, in order).  Rows that are not there come in a last step of their own.
    if constexpr (AHEAD) nxt.load(a, p, clamped(t0 + g));
    for (; t0 + groups <= a.T; t0 += stride) {
        if constexpr (!AHEAD) nxt.load(a, p, t0 + g);
        const GradRow<X, Y, S, ROUTE, LARGE> r = nxt;
        if constexpr (AHEAD) nxt.load(a, p, clamped(t0 + g + stride));
        work(r, t0 + g, true);
    }
    if (t0 < a.T) {
        if constexpr (!AHEAD) nxt.load(a, p, clamped(t0 + g));
        work(nxt, t0 + g, t0 + g < a.T);
    }
    if (!a.partial) return;
    const int columns = padded_columns(a.E), n = ROUTE ? a.n : 0;
    if constexpr (HELD > 0) {
        // sum of y dlogits = gamma (sum of xh dlogits) + beta (sum of dlogits)
        if (a.dwg) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float beta = a.beta[p.at[c] + i];
#pragma unroll
                    for (int e = 0; e < HELD; ++e) acc[2 + e][c][i] = __builtin_fmaf(gm[c][i], acc[2 + e][c][i], beta * dl_sum[e]);
                }
        }
    }
    // the workgroup's part: its groups' sums in ascending order
    float *part = a.partial + (size_t)blockIdx.x * (2 + n) * columns;
    if (groups == 1) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (q >= 2 + n) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c) store_piece<float, VEC>(part + (size_t)q * columns + p.at[c], acc[q][c]);
        }
    } else {
        const int width = p.lanes * CH * VEC;
#pragma unroll
        for (int q0 = 0; q0 < Q; q0 += BATCH) {
            __syncthreads();
#pragma unroll
            for (int q = q0; q < q0 + BATCH && q < Q; ++q)
#pragma unroll
                for (int c = 0; c < CH; ++c) store_piece<float, VEC>(side + (q - q0) * Plan::SIDE + g * width + p.at[c], acc[q][c]);
            __syncthreads();
            const int have = 2 + n - q0 < BATCH ? 2 + n - q0 : BATCH;
            for (int k = threadIdx.x; k < have * columns; k += (int)blockDim.x) {
                const int q = k / columns, j = k - q * columns;
                if (j >= a.E) continue;
                const float *from = side + q * Plan::SIDE + j;
                float s = from[0];
#pragma unroll 4
                for (int r = 1; r < groups; ++r) s += from[r * width];
                part[(size_t)(q0 + q) * columns + j] = s;
            }
        }
    }
    if constexpr (HELD > 0) {
        __syncthreads();
        if (p.l == 0) {
#pragma unroll
            for (int e = 0; e < HELD; ++e) side_dl[g][e] = dl_sum[e];
        }
        __syncthreads();
        if ((int)threadIdx.x < HELD) {
            float s = 0.0f;
            for (int k = 0; k < groups; ++k) s += side_dl[k][threadIdx.x];
            a.partial_dbg[(size_t)blockIdx.x * kMaxExperts + threadIdx.x] = s;
        }
    }
}

// kStreamed: the sums of y dlogits over a part's rows, for a block of columns.
constexpr int kRouterColumns = 1024;         // of a workgroup
template <class X>
__global__ __launch_bounds__(256) void norm_grad_router_kernel(NormGradArgs a, long rows) {
    const int n = a.n, columns = padded_columns(a.E), part = blockIdx.y;
    const int j = (int)blockIdx.x * kRouterColumns + (int)threadIdx.x * 4, at = j + 4 <= a.E ? j : a.E - 4;
    const long t0 = part * rows, t1 = t0 + rows < a.T ? t0 + rows : a.T;
    float acc[kMaxExperts][4], dl_sum[kMaxExperts];
#pragma unroll
    for (int e = 0; e < kMaxExperts; ++e) {
        dl_sum[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[e][i] = 0.0f;
    }
    constexpr int kRows = 64;            // whose statistics and gradients of logits are fetched at a time
    __shared__ float mean[kRows], rstd[kRows], dl[kRows][kMaxExperts];
    for (long r0 = t0; r0 < t1; r0 += kRows) {
        const int count = (int)(t1 - r0 < kRows ? t1 - r0 : kRows);
        __syncthreads();
        for (int k = threadIdx.x; k < kRows * kMaxExperts; k += 256) {
            const int r = k / kMaxExperts, e = k % kMaxExperts;
            dl[r][e] = r < count && e < n ? a.dlogits[(size_t)(r0 + r) * n + e] : 0.0f;
            if (e == 0) {
                mean[r] = r < count ? a.mean[r0 + r] : 0.0f;
                rstd[r] = r < count ? a.rstd[r0 + r] : 0.0f;
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int r = 0; r < count; ++r) {
            Piece<X, 4> x;
            x.load(static_cast<const X *>(a.x) + (size_t)(r0 + r) * a.E + at);
            float xh[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) xh[i] = (x[i] - mean[r]) * rstd[r];
#pragma unroll
            for (int e = 0; e < kMaxExperts; ++e) {
                const float d = dl[r][e];
                dl_sum[e] += d;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[e][i] = __builtin_fmaf(xh[i], d, acc[e][i]);
            }
        }
    }
    float *out = a.partial + ((size_t)part * (2 + n) + 2) * columns + at;
#pragma unroll
    for (int e = 0; e < kMaxExperts; ++e) {
        if (e >= n || j >= a.E) continue;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(a.gamma[at + i], acc[e][i], a.beta[at + i] * dl_sum[e]);
        store_piece<float, 4>(out + (size_t)e * columns, v);
    }
    if (blockIdx.x == 0 && threadIdx.x < 1) {
#pragma unroll
        for (int e = 0; e < kMaxExperts; ++e) a.partial_dbg[(size_t)part * kMaxExperts + e] = dl_sum[e];
    }
}

// The rows of a from `first` on, `count` of them, whose parts go behind `parts` others.
template <class X, class Y>
NormGradArgs some_rows(const NormGradArgs &a, long first, long count, int parts) {
    NormGradArgs b = a;
    const size_t at = (size_t)first * a.E;
    b.T = count;
    b.dy = static_cast<const Y *>(a.dy) + at, b.x = static_cast<const X *>(a.x) + at, b.dx = static_cast<X *>(a.dx) + at;
    if (a.dres) b.dres = static_cast<const X *>(a.dres) + at;
    if (a.mean) b.mean = a.mean + first, b.rstd = a.rstd + first;
    if (a.dlogits) b.dlogits = a.dlogits + (size_t)first * a.n;
    if (a.partial) {
        b.partial = a.partial + (size_t)parts * (2 + a.n) * padded_columns(a.E);
        b.partial_dbg = a.partial_dbg + (size_t)parts * kMaxExperts;
    }
    return b;
}

template <class X, class Y>
int launch_norm_grad_rows(const NormGradArgs &a, int *parts, hipStream_t st) {
    constexpr int VEC = row_vec<X, Y>();
    const bool large = (size_t)a.T * a.E * (sizeof(Y) + (a.dres ? 2 : 1) * sizeof(X)) > kLargeRows;
    auto range = [&](auto shape, auto route, const NormGradArgs &a, int waves, int *parts) {
        using S = decltype(shape);
        const int threads = S::threads(a.E, waves);
        // two parts to a CU of workgroups of four, but 16 rows to a part or one to a CU; the same number of steps in each (12608 x 768 in
        // 226 workgroups 35.9 us, in 256 of which some have a step less 36.9)
        const long cap = !S::WIDE || threads > 256 || a.T < 256 * 16 ? 256 : a.T >= 512 * 16 ? 512 : a.T / 16;
        const long groups = S::groups(a.E, waves), steps = (a.T + groups * cap - 1) / (groups * cap);
        *parts = (int)((a.T + groups * steps - 1) / (groups * steps));
        if constexpr (decltype(route)::value == kStreamed) {
            if (a.dwg) {
                // before dx, which may take the place of x
                const long per = (a.T + *parts - 1) / *parts;
                norm_grad_router_kernel<X><<<dim3((unsigned)((a.E + kRouterColumns - 1) / kRouterColumns), (unsigned)*parts), dim3(256), 0, st>>>(a, per);
                const int rc = check_launch("sa_layernorm_backward(router)");
                if (rc != SA_OK) return rc;
            }
        }
        const dim3 grid((unsigned)*parts), block((unsigned)threads);
        if (large)
            norm_grad_kernel<X, Y, S, decltype(route)::value, true><<<grid, block, 0, st>>>(a);
        else
            norm_grad_kernel<X, Y, S, decltype(route)::value, false><<<grid, block, 0, st>>>(a);
        return check_launch("sa_layernorm_backward(rows)");
    };
    auto rows = [&](auto shape, auto route) {
        using S = decltype(shape);
        using Plan = GradPlan<X, Y, S, decltype(route)::value>;
        int waves = Plan::WAVES;                             // fewer where rows are, down to 4: more CUs have some
        while (waves > 4 && (long)S::groups(a.E, waves) * 256 >= 2 * a.T) waves /= 2;
        // ranges of which a lane adds up kMaxGradSteps rows at most; as a range is long wherever there are two, its parts are those of `most` here
        const long most = (long)S::groups(a.E, waves) * (S::WIDE && S::threads(a.E, waves) <= 256 ? 512 : 256) * kMaxGradSteps;
        const long ranges = (a.T + most - 1) / most, each = (a.T + ranges - 1) / ranges;
        *parts = 0;
        for (long first = 0; first < a.T; first += each) {
            int more = 0;
            const int rc = range(shape, route, some_rows<X, Y>(a, first, a.T - first < each ? a.T - first : each, *parts), waves, &more);
            if (rc != SA_OK) return rc;
            *parts += more;
        }
        return (int)SA_OK;
    };
    auto with = [&](auto route) { return [&rows, route](auto shape) { return rows(shape, route); }; };
    if (!a.dlogits) return by_shape<VEC, VEC == 4>(a.E, with(std::integral_constant<int, 0>()));
    if (a.n == 2) return by_shape<VEC, VEC == 4>(a.E, with(std::integral_constant<int, 2>()));
    if (a.E > kMaxRoute8Columns) return by_wide_shape<VEC, VEC == 4>(a.E, with(std::integral_constant<int, kStreamed>()));
    return by_shape_route8<VEC>(a.E, with(std::integral_constant<int, kMaxExperts>()));
}

}  // namespace sa
