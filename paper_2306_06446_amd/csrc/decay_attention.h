// Linear attention with a decay for each head: what its kernels share (chunks of tokens in LDS as bf16 terms, products of such terms,
// sequences and their segments).
#pragma once

#include "common.h"
#include "row_types.h"

namespace sa {
namespace decay {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;               // tokens of a chunk
constexpr int kSlice = 64;               // columns of the result (and of the state) that a workgroup has
constexpr int kThreads = 256;

// Values as sums of bf16 terms, each the rounding of what the ones before it leave: of an operand in memory as many as hold it exactly (a
// bf16 value is one, an fp16 value two, an fp32 value three), whatever its magnitude: an fp16 product may be far outside of fp16.
// What is computed on the way (probabilities, the state) is 2 terms where the result is rounded to 16 bits (off by 2^-18 of itself at most, the result's
// own rounding is 2^-9 or 2^-12), else 3 (2^-27).  What is added to the fp32 state is 3 terms always.  `ORDER`: products of term i and term j are
// left out where i + j is above it: 2^-9 (i + j) of the operands' product.
template <class T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int RAW = 1, MADE = 2, ORDER_RAW = 0, ORDER = 1; };
template <> struct Terms<f16_t> { static constexpr int RAW = 2, MADE = 2, ORDER_RAW = 1, ORDER = 1; };
template <> struct Terms<float> { static constexpr int RAW = 3, MADE = 3, ORDER_RAW = 2, ORDER = 2; };
constexpr int kUpdateTerms = 3, kUpdateOrder = 2;

template <int N, class V, int W>
__device__ inline void split(const float (&x)[W], V (&t)[N]) {
    float r[W];
#pragma unroll
    for (int i = 0; i < W; ++i) r[i] = x[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            t[n][i] = (__bf16)r[i];
            if (n + 1 < N) r[i] -= (float)t[n][i];
        }
    }
}

// c += A B, 16 x 16 x 32, of operands in NA and NB terms.  Lane l has row (column) l % 16 of A (B) and 8 of the 32 places of the
// sum, those of l / 16; of c it has rows 4 (l / 16) + r of column l % 16.
template <int ORDER, int NA, int NB>
__device__ inline void product(f4 &c, const b8 (&a)[NA], const b8 (&b)[NB]) {
#pragma unroll
    for (int o = (ORDER < NA + NB - 2 ? ORDER : NA + NB - 2); o >= 0; --o) {
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            if (o - i >= 0 && o - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[o - i], c, 0, 0, 0);
        }
    }
}

// Four tokens of one column: the 16 lanes of a group point at 4 rows (lane / 4 % 4) and 4 blocks of 4 columns (lane % 4), lane l
// gets column l % 16 of the 4 rows.
__device__ inline b4 read_transposed(const __bf16 *p) {
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)p);
    return __builtin_bit_cast(b4, v);
}
__device__ inline b8 join(const b4 &a, const b4 &b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// 8 elements on their way from memory to LDS.
template <class T>
struct Eight {
    T v[8];
    __device__ inline void load(const T *p) {
        typedef uint32_t u4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u4 *>(v)[i] = reinterpret_cast<const u4 *>(p)[i];
    }
    __device__ inline void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)0.0f;
    }
    template <int N>
    __device__ inline void terms(b8 (&t)[N]) const {
        if constexpr (sizeof(T) == 2 && N == 1) {
            t[0] = __builtin_bit_cast(b8, *this);
        } else {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
            split(x, t);
        }
    }
};

// Rows of several heads in memory: [tokens][heads][width], tokens `stride` elements apart.
struct HeadRows {
    const void *p;
    long stride;
    int width;
};

// Tokens [begin, end) of one sequence, or a segment of it: position i of the recurrence is token first + i (or first - i, where time is reversed).
struct Span {
    int seq, unit, seg;      // (unit: the segment's place in the workspace)
    long begin, length;      // of the whole sequence
};

// Sequences side by side: T tokens, B sequences of the same length or those between offsets[b] and offsets[b + 1]; segments of `seg`
// tokens, a multiple of kChunk.  Sequence b's first segment is unit first_unit(b): segments of equal sequences follow each other, in a ragged
// batch there is a place for each full segment of all tokens and one more for each sequence, which is enough: a sequence from a seg + r
// to c seg + s has at most c - a + 1 segments.
struct Sequences {
    const int32_t *offsets;  // or null
    long T;
    int B;
    long seg;
    int per_sequence;        // units of a sequence of an equal batch
    __host__ __device__ inline long units() const { return offsets != nullptr ? T / seg + B : (long)per_sequence * B; }
    __device__ inline long offset(int b) const {
        if (offsets == nullptr) return T / B * b;
        const long at = offsets[b];
        return at < 0 ? 0 : at > T ? T : at;
    }
    __device__ inline long first_unit(int b) const { return offsets == nullptr ? (long)per_sequence * b : offset(b) / seg + b; }
    __device__ inline Span of_sequence(int b) const {
        Span s;
        s.seq = b, s.seg = 0;
        s.begin = offset(b);
        const long end = offset(b + 1);
        s.length = end > s.begin ? end - s.begin : 0;
        s.unit = (int)first_unit(b);
        return s;
    }
    // The sequence that has unit u: the last one whose first unit is not behind u, 64 sequences at a time.
    __device__ inline Span of_unit(long u) const {
        int b = 0;
        if (offsets == nullptr) {
            b = (int)(u / per_sequence);
        } else {
            int n = B;
            while (n > 1) {
                const int step = (n + 63) >> 6, lane = (int)(threadIdx.x & 63), at = lane * step;
                const uint64_t there = __ballot(at < n && first_unit(b + (at < n ? at : 0)) <= u);
                const int last = there == 0 ? 0 : 63 - __builtin_clzll(there);
                b += last * step;
                n = n - last * step < step ? n - last * step : step;
            }
            b = __builtin_amdgcn_readfirstlane(b);
        }
        Span s = of_sequence(b);
        s.seg = (int)(u - s.unit);
        s.unit = (int)u;
        return s;
    }
};

// exp(n g): 1 for n = 0 also where g is -infinity (a head without memory).  The exponent is rounded once, relative to itself: a result of 2^-20 is off
// by 20 units, one near 1 by one or two.
__device__ inline float decay_pow(float g, int n) { return n <= 0 ? 1.0f : expf(g * (float)n); }

// A workgroup's share of the launch: workgroups go to the 8 XCDs in turn, neighbours of one list of work belong on one XCD (they read the
// same keys and values).
__device__ inline long xcd_place(long total) {
    const long each = (total + 7) / 8, i = blockIdx.x;
    return (i & 7) * each + (i >> 3);
}
inline long xcd_blocks(long total) { return (total + 7) / 8 * 8; }

template <class F>
int by_type(int type, F f) {
    if (type == SA_F32) return f(float());
    if (type == SA_F16) return f(f16_t());
    return f(bf16_t());
}

inline int check_heads(const char *what, int type, long T, int H, int Hk, int d, int dv) {
    SA_REQUIRE(type >= SA_F32 && type <= SA_BF16, SA_ERR_INVALID, "%s: unknown element type %d", what, type);
    SA_REQUIRE(T >= 0, SA_ERR_INVALID, "%s: a negative number of tokens", what);
    SA_REQUIRE(T < (1L << 31), SA_ERR_SHAPE, "%s: 2^31 tokens or more", what);
    SA_REQUIRE(H > 0 && Hk > 0 && H % Hk == 0, SA_ERR_SHAPE, "%s: %d heads do not share %d key/value heads evenly", what, H, Hk);
    SA_REQUIRE(d > 0 && dv > 0 && d % 8 == 0 && dv % 8 == 0, SA_ERR_SHAPE, "%s: head widths must be multiples of 8 (got %d, %d)", what, d, dv);
    SA_REQUIRE(d <= 128 && dv <= 128, SA_ERR_UNSUPPORTED, "%s: head widths up to 128 (got %d, %d)", what, d, dv);
    SA_REQUIRE(H <= 4096, SA_ERR_UNSUPPORTED, "%s: up to 4096 heads (got %d)", what, H);
    return SA_OK;
}

inline int check_rows(const char *what, const char *name, const void *p, long stride, int heads, int width, int type) {
    SA_REQUIRE(p != nullptr, SA_ERR_INVALID, "%s: %s is NULL", what, name);
    SA_REQUIRE(stride >= (long)heads * width, SA_ERR_SHAPE, "%s: the rows of %s overlap (stride %ld, %d heads of %d)", what, name, stride, heads, width);
    SA_REQUIRE(aligned16(p) && stride % (type == SA_F32 ? 4 : 8) == 0, SA_ERR_ALIGN, "%s: the rows of %s must be 16-byte aligned", what, name);
    return SA_OK;
}

#define SA_TRY(call) \
    do {             \
        if (const int rc_ = (call); rc_ != SA_OK) return rc_; \
    } while (0)

}  // namespace decay
}  // namespace sa
