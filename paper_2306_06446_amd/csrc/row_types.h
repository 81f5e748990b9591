// Rows of the training operators: fp32, fp16 or bf16 in memory, fp32 in registers; which lanes hold which part of a row.
#pragma once

#include "common.h"
#include "layernorm.h"

namespace sa {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// V elements as they are in memory.  Only an element's own alignment is promised: rows of a width that V does not divide begin
// anywhere, and the vector memory unit takes any address.
template <class T, int V>
struct Piece {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    vec v;
    __device__ inline void load(const T *p) { v = *reinterpret_cast<const vec *>(p); }
    __device__ inline float operator[](int i) const { return (float)v[i]; }
};
template <class T>
struct Piece<T, 1> {
    T v;
    __device__ inline void load(const T *p) { v = *p; }
    __device__ inline float operator[](int) const { return (float)v; }
};

// A result in 32 bits to T by one rounding to nearest even.  For fp16 the compiler would fuse the conversion with the operation before it
// where nothing else reads that, which rounds otherwise on a tie: the same rows would differ between calls with other outputs.
template <class T>
__device__ inline T rounded(float f) {
    if constexpr (sizeof(T) == 2) asm("" : "+v"(f));
    return (T)f;
}

template <class T, int V>
__device__ inline void store_piece(T *p, const float (&f)[V]) {
    if constexpr (V == 1) {
        *p = rounded<T>(f[0]);
    } else {
        typename Piece<T, V>::vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = rounded<T>(f[i]);
        *reinterpret_cast<typename Piece<T, V>::vec *>(p) = v;
    }
}

// Elements of one load: 16 bytes of the wider type.
template <class X, class Y>
constexpr int row_vec() { return sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4; }

// A row of E elements on LANES lanes, CH pieces of VEC elements each; lane l's piece c begins at VEC (c LANES + l).  A piece that
// would reach past the row's end (the last one of a row that VEC does not divide, and those behind it) begins VEC before the end
// instead: no load or store needs a choice, elements that two lanes hold are computed and written by both, the same bits.  Only sums
// over the row ask whether an element is a lane's own.  The first FULL pieces of a lane are whole in every row that comes here.
template <int VEC_, int CH_, int LANES_, int FULL_>
struct RowShape {
    static constexpr int VEC = VEC_, CH = CH_, LANES = LANES_, FULL = FULL_;
    static constexpr int THREADS = LANES <= 256 ? 256 : LANES;
    static constexpr int GROUPS = THREADS / LANES;           // rows side by side in a workgroup
    static constexpr int WAVES = THREADS / 64;
    static constexpr int COLUMNS = VEC * CH * LANES;
};

template <class S>
struct RowPlace {
    int at[S::CH], skip[S::CH];
    __device__ inline RowPlace(int l, int E) {
#pragma unroll
        for (int c = 0; c < S::CH; ++c) {
            const int j = (c * S::LANES + l) * S::VEC;
            at[c] = c < S::FULL || j + S::VEC <= E ? j : E - S::VEC;
            skip[c] = j - at[c];
        }
    }
    __device__ inline float own(int c, int i, float v) const { return c < S::FULL || i >= skip[c] ? v : 0.0f; }
};

// Sums of a row over its lanes, N at a time, in all of them.  Rows of several wavefronts exchange theirs in LDS; two buffers in turn, so that
// one barrier per exchange is enough (a wavefront that writes a buffer again has passed the barrier behind its last reads).
template <class S, int N>
struct RowSums {
    float (*red)[2][S::WAVES];           // [N][2][WAVES] in LDS, where a row has several wavefronts
    int turn = 0;
    __device__ inline void operator()(float (&v)[N], int used = N) {
        constexpr int L = S::LANES < 64 ? S::LANES : 64;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < used) v[k] = group_sum<L>(v[k]);
        if constexpr (S::LANES > 64) {
            constexpr int W = S::LANES / 64;
            const int wave = threadIdx.x >> 6, first = wave / W * W;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (k < used) red[k][turn][wave] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k >= used) continue;
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) s += red[k][turn][first + w];
                v[k] = s;
            }
            turn ^= 1;
        }
    }
};

// What a launch does with the type of a residual stream (X) and of the rows it meets (Y).
template <template <class, class> class F, class... A>
int for_row_types(int x_type, int y_type, A &&...a) {
    if (x_type == SA_F32 && y_type == SA_F32) return F<float, float>::run(a...);
    if (x_type == SA_F32 && y_type == SA_F16) return F<float, f16_t>::run(a...);
    if (x_type == SA_F32 && y_type == SA_BF16) return F<float, bf16_t>::run(a...);
    if (x_type == SA_F16) return F<f16_t, f16_t>::run(a...);
    return F<bf16_t, bf16_t>::run(a...);
}

inline int check_row_types(const char *what, int x_type, int y_type) {
    SA_REQUIRE(x_type >= SA_F32 && x_type <= SA_BF16 && y_type >= SA_F32 && y_type <= SA_BF16, SA_ERR_INVALID,
               "%s: unknown element type (%d, %d)", what, x_type, y_type);
    SA_REQUIRE(x_type == y_type || x_type == SA_F32, SA_ERR_UNSUPPORTED,
               "%s: element types %d and %d do not go together (the same, or a residual stream of SA_F32)", what, x_type, y_type);
    return SA_OK;
}

}  // namespace sa
