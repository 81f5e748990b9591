// Rows of the training operators: fp32, fp16 or bf16 in memory, fp32 in registers; which lanes hold which part of a row.
#pragma once

#include <type_traits>

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
    __device__ inline void stream(const T *p) { v = __builtin_nontemporal_load(reinterpret_cast<const vec *>(p)); }      // not for the caches to keep
    __device__ inline float operator[](int i) const { return (float)v[i]; }
};
template <class T>
struct Piece<T, 1> {
    T v;
    __device__ inline void load(const T *p) { v = *p; }
    __device__ inline void stream(const T *p) { v = *p; }
    __device__ inline float operator[](int) const { return (float)v; }
};

// Has the loads of a piece behind it: values that two wavefronts read are there in both before a barrier, behind which one of them may store
// over them (a result in its operand's place).
template <class P>
__device__ inline void arrived(const P &p) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(p.v) / 4)));
    asm volatile("" : : "v"(__builtin_bit_cast(words, p.v)) : "memory");
}

// A result in 32 bits to T by one rounding to nearest even.  For fp16 the compiler would fuse the conversion with the operation before it
// where nothing else reads that, which rounds otherwise on a tie: the same rows would differ between calls with other outputs.
template <class T>
__device__ inline T rounded(float f) {
    if constexpr (sizeof(T) == 2) asm("" : "+v"(f));
    return (T)f;
}

template <class T, int V>
__device__ inline typename Piece<T, V>::vec rounded_piece(const float (&f)[V]) {
    typename Piece<T, V>::vec v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = rounded<T>(f[i]);
    return v;
}
template <class T, int V>
__device__ inline void store_piece(T *p, const float (&f)[V]) {
    if constexpr (V == 1) *p = rounded<T>(f[0]);
    else *reinterpret_cast<typename Piece<T, V>::vec *>(p) = rounded_piece<T, V>(f);
}
// Rows of results, past the caches' reuse order: written once and large, they would push out the rows that are being read.  LayerNorm of
// 12608 x 768 with router 13.6 -> 10.8 us, 100000 x 1024 bf16 78.5 -> 73.0, its gradient of 131072 x 1024 206 -> 200, the combine's of
// 50021 x 500 34.5 -> 31.6; nothing where all of it fits a cache (197 x 192).
template <class T, int V>
__device__ inline void stream_piece(T *p, const float (&f)[V]) {
    if constexpr (V == 1) *p = rounded<T>(f[0]);
    else __builtin_nontemporal_store(rounded_piece<T, V>(f), reinterpret_cast<typename Piece<T, V>::vec *>(p));
}

// Elements of one load: 16 bytes of the wider type.
template <class X, class Y>
constexpr int row_vec() { return sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4; }

// A row of E elements on LANES lanes, CH pieces of VEC elements each; lane l's piece c begins at VEC (c LANES + l).  A piece that
// would reach past the row's end (the last one of a row that VEC does not divide, and those behind it) begins VEC before the end
// instead: no load or store needs a choice, elements that two lanes hold are computed and written by both, the same bits.  Only sums
// over the row ask whether an element is a lane's own.  The first FULL pieces of a lane are whole in every row that comes here.
// LANES is 16, 32 or 64, rows side by side in a wavefront, or kWide: the lanes of 2, 4 or 8 wavefronts, as many as the row takes.  (Of 3, 5, 6
// or 7 the SIMDs of a CU get unequal shares, and all wait for the largest: 43859 x 4560 fp16 on 5 wavefronts 209 us, on 8 165.)
constexpr int kWide = 512;
template <int VEC_, int CH_, int LANES_, int FULL_>
struct RowShape {
    static constexpr int VEC = VEC_, CH = CH_, LANES = LANES_, FULL = FULL_;
    static constexpr bool WIDE = LANES > 64;
    static constexpr int PERIOD = WIDE ? 64 : LANES;         // rows whose statistics the lanes of one wavefront can keep
    static __host__ __device__ inline int waves(int E) { return !WIDE ? 1 : E <= 128 * VEC * CH ? 2 : E <= 256 * VEC * CH ? 4 : 8; }
    // rows side by side in a workgroup of up to max_waves wavefronts
    static int groups(int E, int max_waves) { return WIDE ? (waves(E) < max_waves ? max_waves / waves(E) : 1) : max_waves * 64 / LANES; }
    static int threads(int E, int max_waves) { return WIDE ? 64 * waves(E) * groups(E, max_waves) : 64 * max_waves; }
};

template <class S>
struct RowPlace {
    int g, l, lanes, groups;             // this lane's row among the workgroup's, and its place in it
    int at[S::CH], skip[S::CH];
    __device__ inline RowPlace(int E) {
        const int waves = S::waves(E);
        lanes = S::WIDE ? 64 * waves : S::LANES;
        groups = S::WIDE ? (int)(blockDim.x >> 6) / waves : (int)blockDim.x / S::LANES;
        g = S::WIDE ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6) / waves) : (int)threadIdx.x / S::LANES;
        l = (int)threadIdx.x - g * lanes;
#pragma unroll
        for (int c = 0; c < S::CH; ++c) {
            const int j = (c * lanes + l) * S::VEC;
            at[c] = c < S::FULL || j + S::VEC <= E ? j : E - S::VEC;
            skip[c] = j - at[c];
        }
    }
    __device__ inline float own(int c, int i, float v) const { return c < S::FULL || i >= skip[c] ? v : 0.0f; }
};

// Eight sums over a wavefront, the one of value lane / 8 in each lane: every step adds two values at once, each in half of the lanes.
__device__ inline float eight_sums(const float (&v)[8]) {
    auto swap_add = [](float a, float b, auto rows) {
        const uint32_t u = __builtin_bit_cast(uint32_t, a), w = __builtin_bit_cast(uint32_t, b);
        const auto r = decltype(rows)::value ? __builtin_amdgcn_permlane16_swap(u, w, false, false) : __builtin_amdgcn_permlane32_swap(u, w, false, false);
        const uint32_t r0 = r[0], r1 = r[1];
        return __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
    };
    float h[4], q[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) h[k] = swap_add(v[k], v[k + 4], std::false_type());
#pragma unroll
    for (int k = 0; k < 2; ++k) q[k] = swap_add(h[k], h[k + 2], std::true_type());
    const bool upper = threadIdx.x & 8;
    const float mine = upper ? q[1] : q[0], other = upper ? q[0] : q[1];
    const int moved = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, other), 0x128, 0xF, 0xF, true);      // row_ror:8
    float s = mine + __builtin_bit_cast(float, moved);
    s = dpp_add<0x141>(s);                // row_half_mirror
    s = dpp_add<0x4E>(s);                 // quad_perm: lanes 2 apart
    return dpp_add<0xB1>(s);              // lanes 1 apart
}

// Sums of a row over its lanes, N at a time, in all of them.  Rows of several wavefronts exchange theirs in LDS; two buffers in turn, so that
// one barrier per exchange is enough (a wavefront that writes a buffer again has passed the barrier behind its last reads).
template <class S, int N>
struct RowSums {
    float (*red)[2][8];                  // [N][2][wavefronts] in LDS, where a row has several wavefronts
    int first, waves, turn = 0;
    __device__ inline RowSums(float (*red_)[2][8], const RowPlace<S> &p) : red(red_), first(p.g * (p.lanes / 64)), waves(p.lanes / 64) {}
    // what the row's wavefronts have left of value k: 2, 4 or 8, in loads as wide as that
    __device__ inline float of(int k) const {
        const float *from = red[k][turn] + first;
        if (waves == 2) return from[0] + from[1];
        const float4 a = *reinterpret_cast<const float4 *>(from);
        float s = (a.x + a.y) + (a.z + a.w);
        if (waves == 8) {
            const float4 b = *reinterpret_cast<const float4 *>(from + 4);
            s += (b.x + b.y) + (b.z + b.w);
        }
        return s;
    }
    template <int M>
    __device__ inline void operator()(float (&v)[M], int used = M) {
        static_assert(M <= N, "room in LDS");
        constexpr int L = S::LANES < 64 ? S::LANES : 64;
#pragma unroll
        for (int k = 0; k < M; ++k)
            if (k < used) v[k] = group_sum<L>(v[k]);
        if constexpr (S::WIDE) {
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < M; ++k)
                    if (k < used) red[k][turn][threadIdx.x >> 6] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < M; ++k) {
                if (k >= used) continue;
                v[k] = of(k);
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
