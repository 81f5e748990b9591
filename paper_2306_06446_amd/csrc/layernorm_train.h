// LayerNorm of training: what its entry points (layernorm_train.hip) and the kernels of either direction share.
#pragma once

#include <type_traits>

#include "row_types.h"

namespace sa {

constexpr int kMaxNormColumns = 8192;
constexpr int kGradParts = 512;              // workgroups of a range of rows, whose sums a last launch adds up
constexpr int kMaxGradSteps = 512;           // rows of a range that a lane adds up in fp32 (16384 of 0.1 would be off by 1.5e-4)

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
    const float *weights;    // kStreamed: wg as [n][columns, a multiple of 4]
    void *dx;
    float *partial;          // [parts][2 + n][columns, a multiple of 4]: dgamma, dbeta, dwg by expert; null: none wanted
    float *partial_dbg;      // [parts][kMaxExperts]
    float *dgamma, *dbeta, *dwg, *dbg;
    int accumulate;
};

__host__ __device__ inline int padded_columns(int E) { return (E + 3) / 4 * 4; }

// The gradient's parts at most, of any types: a workgroup has 8 rows side by side at least where rows are narrow and this many, else one, and a
// range has 512 parts of 512 times as many rows, or 256 of half of them.
inline long max_grad_parts(long T, int E) {
    const long rows = (long)kGradParts * kMaxGradSteps * (E <= 512 ? 8 : 1);
    return T < kGradParts ? T : (T + rows - 1) / rows * kGradParts;
}

// ROUTE: experts whose weights a kernel holds in registers, the gradient with their sums (0, 2 or kMaxExperts); kStreamed: the gradient
// has the weights from memory row by row, and the sums come of a launch of their own.
constexpr int kStreamed = 1;

// The shape of a row of E elements.  Up to 16 elements to a lane (with a gradient's sums, as many registers as leave two wavefronts to a
// SIMD), fewer lanes for narrow rows, so that a wavefront works on several; wider rows take several wavefronts.
// Wide rows: 12 elements to a lane of 2, 4 or 8 wavefronts where that is enough (FEW), else 16.
// 16-bit rows of up to 64 elements: 4 to a lane, as with 8 half of a row's 16 lanes or more would repeat what others do.  Forward
// 10^6 x 64 fp16 67 -> 59 us, with a router of two 91 -> 75; backward 131072 x 64 bf16 20.5 -> 18.8, 27.5 -> 21.9.
constexpr int kMaxRoute8Columns = 2048;
template <int VEC, bool FEW, class F>
int by_wide_shape(int E, F &&f) {
    if constexpr (FEW)
        if (E <= 12 * 128 || (E > 2048 && E <= 12 * 256) || (E > 4096 && E <= 12 * 512)) return f(RowShape<4, 3, kWide, 2>());
    return f(RowShape<VEC, 16 / VEC, kWide, FEW ? 12 / VEC : 8 / VEC>());
}
template <int VEC, bool FEW, class F>
int by_shape(int E, F &&f) {
    if (E < VEC) return f(RowShape<1, 1, 16, 0>());
    if constexpr (VEC == 8)
        if (E <= 64) return f(RowShape<4, 1, 16, 0>());
    if (E <= 16 * VEC) return f(RowShape<VEC, 1, 16, 0>());
    if (E <= 32 * VEC) return f(RowShape<VEC, 1, 32, 0>());
    if (E <= 64 * VEC) return f(RowShape<VEC, 1, 64, 0>());
    if (E <= 128 * VEC) return f(RowShape<VEC, 2, 64, 1>());
    if constexpr (VEC == 4) {
        if (E <= 192 * VEC) return f(RowShape<VEC, 3, 64, 2>());
        if (E <= 256 * VEC) return f(RowShape<VEC, 4, 64, 3>());
    }
    return by_wide_shape<VEC, FEW>(E, f);
}
// The gradient with a router of up to 8 experts: 8 elements to a lane, whose 64 weights and 64 sums are registers too.  Wider rows would
// want more of them than there are.  Up to 64 elements 4 to a lane, all sixteen at work: 131072 x 64 bf16 with eight 39.6 -> 32.9 us, fp32
// 41.1 -> 36.5; 131072 x 33 fp16 with three 35.6 -> 25.6.
template <int VEC, class F>
int by_shape_route8(int E, F &&f) {
    if (E < VEC) return f(RowShape<1, 1, 16, 0>());
    if (E <= 64) return f(RowShape<4, 1, 16, 0>());
    if (E <= 128) return f(RowShape<VEC, 8 / VEC, 16, 0>());
    if (E <= 256) return f(RowShape<VEC, 8 / VEC, 32, 0>());
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
template <int VEC, int CH>
__device__ inline void load_router_pair(float (&out)[2][CH][VEC], int c, const float *p) {
    Piece<float, 2 * VEC> v;
    v.load(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[0][c][i] = v[2 * i], out[1][c][i] = v[2 * i + 1];
}
// Of up to N experts, zeros behind the n there are: in tiles of columns through LDS (a lane's own weights are 4 n VEC bytes from the next
// lane's in memory, a line to a lane and load: 12608 x 768 with eight experts took 75 us, 45 of them for this).  Tiles overlap by a
// piece, so that one of them has the whole of it.
constexpr int kRouterTile = 2048;
constexpr int kRouterTileFloats = (kRouterTile * kMaxExperts) / 32 * 33 + 1;
template <class S, int N>
__device__ inline void load_router(float (&out)[N][S::CH][S::VEC], const RowPlace<S> &p, const float *wg, int E, int n, float *tile) {
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
        for (int c = 0; c < S::CH; ++c)
#pragma unroll
            for (int i = 0; i < S::VEC; ++i) out[e][c][i] = 0.0f;
    for (int j0 = 0; j0 < E; j0 += kRouterTile - S::VEC) {
        const int columns = E - j0 < kRouterTile ? E - j0 : kRouterTile;
        __syncthreads();
        for (int k = threadIdx.x; k < columns * n; k += (int)blockDim.x) tile[k + k / 32] = wg[(size_t)j0 * n + k];
        __syncthreads();
#pragma unroll
        for (int c = 0; c < S::CH; ++c) {
            const int at = p.at[c] - j0;
            if (at < 0 || at + S::VEC > columns) continue;
#pragma unroll
            for (int i = 0; i < S::VEC; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int k = (at + i) * n + e;
                    if (e < n) out[e][c][i] = tile[k + k / 32];
                }
        }
    }
}

template <class X, class Y>
int launch_norm_rows(const NormArgs &a, hipStream_t st);
// Leaves sums over rows in a.partial, in *parts parts.
template <class X, class Y>
int launch_norm_grad_rows(const NormGradArgs &a, int *parts, hipStream_t st);

}  // namespace sa
