// LayerNorm of training: what its entry points (layernorm_train.hip) and the kernels of either direction share.
#pragma once

#include <type_traits>

#include "row_types.h"

namespace sa {

constexpr int kMaxNormColumns = 8192;
constexpr int kMaxGradParts = 512;           // workgroups whose sums over rows are added up by a second launch

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
    float eps;
    const float *mean, *rstd;        // null: from x
    const void *dres;        // or null
    const float *dlogits, *wg;       // null: no router
    int n;
    const float *weights;    // kStreamed: of expert e, column j at weights[e * by_expert + j * by_column]
    long by_expert;
    int by_column;
    void *dx;
    float *partial;          // [parts][2 + n][columns, a multiple of 4]: dgamma, dbeta, dwg by expert; null: none wanted
    float *partial_dbg;      // [parts][kMaxExperts]
    float *dgamma, *dbeta, *dwg, *dbg;
    int accumulate;
};

__host__ __device__ inline int padded_columns(int E) { return (E + 3) / 4 * 4; }

// ROUTE: experts whose weights a kernel of the gradient holds in registers, with their sums (0, 2 or kMaxExperts), or
// kStreamed: weights from memory row by row, sums elsewhere.
constexpr int kStreamed = 1;

// The shape of a row of E elements.  Up to 16 elements to a lane (with a gradient's sums, as many registers as leave two wavefronts to a
// SIMD), fewer lanes for narrow rows, so that a wavefront works on several; wider rows take several wavefronts.
template <int VEC, class F>
int by_wide_shape(F &&f) { return f(RowShape<VEC, 16 / VEC, kWide, 8 / VEC>()); }
template <int VEC, class F>
int by_shape(int E, F &&f) {
    if (E < VEC) return f(RowShape<1, 1, 16, 0>());
    if (E <= 16 * VEC) return f(RowShape<VEC, 1, 16, 0>());
    if (E <= 32 * VEC) return f(RowShape<VEC, 1, 32, 0>());
    if (E <= 64 * VEC) return f(RowShape<VEC, 1, 64, 0>());
    if (E <= 128 * VEC) return f(RowShape<VEC, 2, 64, 1>());
    if constexpr (VEC == 4) {
        if (E <= 192 * VEC) return f(RowShape<VEC, 3, 64, 2>());
        if (E <= 256 * VEC) return f(RowShape<VEC, 4, 64, 3>());
    }
    return by_wide_shape<VEC>(f);
}
// With a router of up to 8 experts: 8 elements to a lane, whose 64 weights and 64 sums are registers too.  Wider rows would want more
// of them than there are.
constexpr int kMaxRoute8Columns = 2048;
template <int VEC, class F>
int by_shape_route8(int E, F &&f) {
    if (E < VEC) return f(RowShape<1, 1, 16, 0>());
    if (E <= 512) return f(RowShape<VEC, 8 / VEC, 64, 0>());
    return f(RowShape<VEC, 8 / VEC, kWide, 0>());
}

// A piece of a parameter row, and of the router's weights [E, n]: N experts, zeros behind the n there are.
template <int VEC>
__device__ inline void load_columns(float (&out)[VEC], const float *p) {
    Piece<float, VEC> v;
    v.load(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] = v[i];
}
template <int VEC, int N, int CH>
__device__ inline void load_router(float (&out)[N][CH][VEC], int c, const float *p, int n) {
    if constexpr (N == 2) {
        Piece<float, 2 * VEC> v;
        v.load(p);
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[0][c][i] = v[2 * i], out[1][c][i] = v[2 * i + 1];
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float v = p[i * n + (e < n ? e : 0)];
                out[e][c][i] = e < n ? v : 0.0f;
            }
    }
}

template <class X, class Y>
int launch_norm_rows(const NormArgs &a, hipStream_t st);
// Leaves sums over rows in a.partial, in *parts parts.
template <class X, class Y>
int launch_norm_grad_rows(const NormGradArgs &a, int *parts, hipStream_t st);

}  // namespace sa
