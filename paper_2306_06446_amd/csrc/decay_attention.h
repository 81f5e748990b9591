// Linear attention with a decay for each head: what its kernels share (chunks of tokens in LDS as 16-bit terms, bf16 or fp16, products of such terms,
// sequences and their segments).
#pragma once

#include <type_traits>
#include <utility>

#include "common.h"
#include "row_types.h"

namespace sa {
namespace decay {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
template <class E, int N>
using Vec = E __attribute__((ext_vector_type(N)));

constexpr int kChunk = 64;               // tokens of a chunk
constexpr int kHalf = 64;                // columns of the result (and of the state) to four wavefronts

// Operands of the matrix cores as sums of 16-bit terms, each the rounding of what the ones before it leave.  What is in memory enters exactly: a
// bf16 or fp16 value is one term of its own type, an fp32 value three of bf16.  What is computed on the way (products q k, the state) is 2 terms where
// the result is rounded to 16 bits, else 3; what is added to the fp32 state 2 of fp16 or 3 of bf16.  `ORDER`: products of term i and
// term j are left out where i + j is above it, of fp32 2^-24 of a product.  A value in two terms of bf16 is off by 2^-17 of itself at most (1 + 2^-8 - 2^-17
// is), in three by 2^-26, in two of fp16 by 2^-23, where the result's own rounding is 2^-8, 2^-24 and 2^-11.  (bf16 rows from three terms: 8 x 16384 tokens, 4 heads of 64,
// 92 -> 100 us, their gradient 193 -> 231, and no closer to 64 bits once they are rounded.)  What meets fp16 operands is scaled by a power of two (Scale),
// one for each sum, that puts its largest term between 2^14 and 2^15.  Terms of 2^-17 of that and more keep their 22 bits, smaller ones are off by 2^-39 of
// the largest; where that is not enough, in states in memory, they are added by themselves.
template <class T> struct Terms;
template <> struct Terms<bf16_t> { typedef bf16_t E; static constexpr int RAW = 1, MADE = 2, ADDED = 3, ORDER_RAW = 0, ORDER = 1, ORDER_ADDED = 2; static constexpr bool SCALED = false; };
template <> struct Terms<f16_t> { typedef f16_t E; static constexpr int RAW = 1, MADE = 2, ADDED = 2, ORDER_RAW = 0, ORDER = 1, ORDER_ADDED = 1; static constexpr bool SCALED = true; };
template <> struct Terms<float> { typedef bf16_t E; static constexpr int RAW = 3, MADE = 3, ADDED = 3, ORDER_RAW = 2, ORDER = 2, ORDER_ADDED = 2; static constexpr bool SCALED = false; };

// f(0), f(1), ... with constants.
template <class F, int... I>
__device__ inline void each_of(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F>
__device__ inline void each(F f) { each_of(std::make_integer_sequence<int, N>(), f); }

// Zeros that the compiler does not know as such.  An array that is cleared with known ones is one piece of memory to it, then one vector of 16
// registers, which moves, and leaves the registers, as a whole: 20 KB of moves to scratch memory a wavefront.
__device__ inline f4 zeros() {
    float z = 0.0f;
    asm("" : "+v"(z));
    return f4{z, z, z, z};
}

template <class E, int N, int W>
__device__ inline void split(const float (&x)[W], Vec<E, W> (&t)[N], float up = 1.0f) {
    each<W / 2>([&](auto pair) {
        constexpr int i = 2 * pair;
        f2 r = {x[i] * up, x[i + 1] * up};
        each<N>([&](auto term) {
            constexpr int n = term;
            const Vec<E, 2> h = __builtin_convertvector(r, Vec<E, 2>);     // one instruction for two values
            t[n][i] = h[0], t[n][i + 1] = h[1];
            if (n + 1 < N) r[0] -= (float)h[0], r[1] -= (float)h[1];
        });
    });
}

// Powers of two that bring values of magnitude m and less below 2^15, and back.  (Below 2^-112 and for infinities as far as there are such powers.)
struct Scale {
    float up, down;
    __device__ inline explicit Scale(float m) {
        int e = (int)(__builtin_bit_cast(uint32_t, m) >> 23);
        e = e < 15 ? 15 : e > 254 ? 254 : e;
        up = __builtin_bit_cast(float, (uint32_t)(268 - e) << 23);
        down = __builtin_bit_cast(float, (uint32_t)(e - 14) << 23);
    }
};
template <int W>
__device__ inline float largest(const float (&x)[W], float m = 0.0f) {
    each<W>([&](auto i) { m = fmaxf(m, fabsf(x[i])); });
    return m;
}
// The smallest magnitude that is not zero, as twice its bits less one, which puts zeros above all others.
template <int W>
__device__ inline uint32_t least(const float (&x)[W], uint32_t m = ~0u) {
    each<W>([&](auto i) {
        const uint32_t u = (__builtin_bit_cast(uint32_t, x[i]) << 1) - 1u;
        m = u < m ? u : m;
    });
    return m;
}
// The largest of the four lanes of a column of the matrix cores' results.
__device__ inline float column_max(float m) {
    const uint32_t u = __builtin_bit_cast(uint32_t, m);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    const uint32_t h = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)));
    const auto s = __builtin_amdgcn_permlane16_swap(h, h, false, false);
    const uint32_t s0 = s[0], s1 = s[1];
    return fmaxf(__builtin_bit_cast(float, s0), __builtin_bit_cast(float, s1));
}

// (A sum of products is aligned to the largest one's exponent and cut 24 bits below it, and to that a subnormal fp16 operand counts as one of exponent -14:
// 2^-24 times 2^14 beside a sum of 2^-25 leaves nothing of the latter.  A subnormal number so takes part to 2^-38.)
// c += A B, 16 x 16 x 32, of operands in NA and NB terms.  Lane l has row (column) l % 16 of A (B) and 8 of the 32 places of the
// sum, those of l / 16; of c it has rows 4 (l / 16) + r of column l % 16.
__device__ inline f4 matrix(const Vec<bf16_t, 8> &a, const Vec<bf16_t, 8> &b, const f4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f4 matrix(const Vec<f16_t, 8> &a, const Vec<f16_t, 8> &b, const f4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
template <int ORDER, class E, int NA, int NB>
__device__ inline void product(f4 &c, const Vec<E, 8> (&a)[NA], const Vec<E, 8> (&b)[NB]) {
#pragma unroll
    for (int o = (ORDER < NA + NB - 2 ? ORDER : NA + NB - 2); o >= 0; --o) {
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            if (o - i >= 0 && o - i < NB) c = matrix(a[i], b[o - i], c);
        }
    }
}

// Results of the matrix cores at the end of a way through the code that others join.  What reads them has to come 8 wait states later, and the compiler, which
// sees to that, does not where it can also come to the place by a longer way: of 32 keys in fp16, the results of one of four wavefronts were read 2 wait
// states behind their product, and wrong.
template <int N>
__device__ inline void settled(f4 (&x)[N]) {
    each<N>([&](auto i) {
        f4 y = x[i];
        if constexpr (i + 1 < N) asm volatile("" : "+v"(y));
        else asm volatile("s_nop 7" : "+v"(y));
        x[i] = y;
    });
}

// Four tokens of one column: the 16 lanes of a group point at 4 rows (lane / 4 % 4) and 4 blocks of 4 columns (lane % 4), lane l
// gets column l % 16 of the 4 rows.
template <class E>
__device__ inline Vec<E, 4> read_transposed(const E *p) {
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)const_cast<E *>(p));
    return __builtin_bit_cast(Vec<E, 4>, v);
}
template <class E>
__device__ inline Vec<E, 8> join(const Vec<E, 4> &a, const Vec<E, 4> &b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// The thread's number once more, for what is seldom done and not worth registers for what could be made of it ahead.
__device__ inline int thread_of(int wave) {
    int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    return 64 * wave + lane;
}

// What all lanes have the same, in a scalar register.
// (The builtin's result is signed: as the low half of an address it would set all of the high one.)
__device__ inline uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ inline float uniform(float x) { return __builtin_bit_cast(float, uniform(__builtin_bit_cast(uint32_t, x))); }

// Rows of one head, from memory: a base and a size in bytes that all lanes share and a 32-bit offset each.  What begins behind the size, as kNowhere
// and up to 2^30 less do, reads as zeros and is not written, without a branch.
constexpr uint32_t kNowhere = 0xc0000000u;
__device__ inline __amdgpu_buffer_rsrc_t buffer(uint64_t p, uint32_t bytes) {
    const uint64_t at = (uint64_t)uniform((uint32_t)(p >> 32)) << 32 | uniform((uint32_t)p);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(at), 0, (int)uniform(bytes), 0x00027000);
}

// 8 elements on their way from memory to LDS.
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
template <class T>
struct Eight {
    typedef T vec __attribute__((ext_vector_type(8)));
    vec v;
    __device__ inline void load(__amdgpu_buffer_rsrc_t from, uint32_t at) {
        if constexpr (sizeof(T) == 2) {
            v = __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, 0));
        } else {
            struct { u4 a, b; } x = {__builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, 0), __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 16, 0)};
            v = __builtin_bit_cast(vec, x);
        }
    }
    template <class E, int N>
    __device__ inline void terms(Vec<E, 8> (&t)[N]) const {
        if constexpr (N == 1) {
            t[0] = v;
        } else {
            float x[8];
            each<8>([&](auto i) { x[i] = (float)v[(int)i]; });
            split(x, t);
        }
    }
};
// What is not finite as an operand of the matrix cores (the first term of an fp32 value, too, that is rounded to infinity): one by one, and two at a time,
// whose products with zero are added to a sum of zeros.
__device__ inline bool not_finite(bf16_t x) { return (__builtin_bit_cast(uint16_t, x) & 0x7fffu) >= 0x7f80u; }
__device__ inline bool not_finite(f16_t x) { return (__builtin_bit_cast(uint16_t, x) & 0x7fffu) >= 0x7c00u; }
__device__ inline float times_zero(const Vec<f16_t, 2> &x, float sum) { return __builtin_amdgcn_fdot2(x, Vec<f16_t, 2>{(f16_t)0.0f, (f16_t)0.0f}, sum, false); }
__device__ inline float times_zero(const Vec<bf16_t, 2> &x, float sum) {
    return __builtin_amdgcn_fdot2_f32_bf16(x, Vec<bf16_t, 2>{(bf16_t)0.0f, (bf16_t)0.0f}, sum, false);
}
// STREAM: past the caches' reuse order, for results that fill whole lines of 128 bytes (gradient of 64 x 197 tokens, 12 heads of 64, bf16: 58 -> 50 us; rows
// of 144 bytes, which do not, lost 6 %).
template <class T, bool STREAM>
__device__ inline void store_eight(__amdgpu_buffer_rsrc_t to, uint32_t at, const float (&x)[8]) {
    typename Eight<T>::vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = rounded<T>(x[i]);
    struct Words { u4 a[sizeof(T) / 2]; };
    const Words w = __builtin_bit_cast(Words, v);
    each<sizeof(T) / 2>([&](auto i) {
        __builtin_amdgcn_raw_buffer_store_b128(w.a[i], to, (int)at, 16 * i, STREAM ? 2 : 0);
    });
}

// Rows of several heads in memory: [tokens][heads][width], tokens `stride` elements apart.
struct HeadRows {
    const void *p;
    long stride;
    int width;
};

// One segment of a sequence: position i of the recurrence is token begin + i (or begin + length - 1 - i, where time is reversed), the segment has
// those from seg segments on.
struct Span {
    int seq, seg;
    int place;               // the segment's state in the workspace
    int begin, length;       // of the whole sequence
};

// Sequences side by side: T tokens, B sequences of `each` tokens or those between offsets[b] and offsets[b + 1]; segments of `seg` tokens, a
// multiple of kChunk.  Sequence b's first segment is unit first_unit(b): segments of equal sequences follow each other, in a ragged batch
// (whose segments are powers of two) there is a place for each full segment of all tokens and one more for each sequence, which is enough: a
// sequence from a seg + r to c seg + s has at most c - a + 1 segments.
// The states of segments are at their units; where segments are longer than most sequences (`whole`), only sequences of several segments have any, and the
// first place is 2 a, which is enough, too: c is a + 1 at least, and the last place a + c below 2 c, the next such sequence's first.
struct Sequences {
    const int32_t *offsets;  // or null
    int T, B, each;
    int seg, log_seg;
    int per_sequence;        // units of a sequence of an equal batch
    bool whole;
    __device__ inline bool cut(int length) const { return !whole || length > seg; }
    __host__ __device__ inline long units() const { return offsets != nullptr ? (long)(T >> log_seg) + B : (long)per_sequence * B; }
    __device__ inline int offset(int b) const {
        const int at = offsets[b];
        return at < 0 ? 0 : at > T ? T : at;
    }
    __device__ inline Span of_sequence(int b) const {
        Span s;
        s.seq = b, s.seg = 0;
        if (offsets == nullptr) {
            s.begin = each * b, s.length = each, s.place = per_sequence * b;
        } else {
            s.begin = __builtin_amdgcn_readfirstlane(offset(b));
            const int end = __builtin_amdgcn_readfirstlane(offset(b + 1));
            s.length = end > s.begin ? end - s.begin : 0;
            s.place = whole ? 2 * (s.begin >> log_seg) : (s.begin >> log_seg) + b;
        }
        return s;
    }
    // The sequence that has unit u: the last one whose first unit is not behind u, 64 sequences at a time.
    __device__ inline Span of_unit(uint32_t u) const {
        if (offsets == nullptr) {
            Span s = of_sequence(per_sequence == 1 ? (int)u : (int)(u / (uint32_t)per_sequence));
            s.seg = (int)u - s.place;
            s.place = (int)u;
            return s;
        }
        int b = 0, n = B, at, last;
        do {
            const int step = (n + 63) >> 6, lane = (int)(threadIdx.x & 63) * step, place = b + (lane < n ? lane : n);
            at = offset(place);          // (there are B + 1 of them)
            const uint64_t there = __ballot(lane < n && (uint32_t)((at >> log_seg) + place) <= u);
            last = there == 0 ? 0 : 63 - __builtin_clzll(there);
            b += last * step;
            n = n - last * step < step ? n - last * step : step;
        } while (n > 1);
        // the last round's lanes have the sequence's first token and, but for the last lane, the one behind its last
        Span s;
        s.seq = __builtin_amdgcn_readfirstlane(b);
        s.begin = __builtin_amdgcn_readlane(at, last);
        const int end = last < 63 ? __builtin_amdgcn_readlane(at, last + 1) : __builtin_amdgcn_readfirstlane(offset(s.seq + 1));
        s.length = end > s.begin ? end - s.begin : 0;
        s.seg = (int)u - ((s.begin >> log_seg) + s.seq);
        s.place = whole ? 2 * (s.begin >> log_seg) + s.seg : (int)u;
        return s;
    }
};

// exp(n g), n >= 0, as 2^(n g / ln 2): the exponent is rounded twice, relative to itself, so a result of 2^-20 is off by some 30 units and one near 1 by
// one or two.  A head without memory (g = -infinity) has 1 for n = 0 and 0 for all others: so has one of -2000.
__device__ inline float decay_rate(float g) { return (g < -2000.0f ? -2000.0f : g) * 1.44269504f; }
__device__ inline float decay_pow(float rate, int n) { return __builtin_amdgcn_exp2f(rate * (float)n); }

// Workgroups go to the 8 XCDs in turn.  Those of one segment (`per` of them, which read the same rows) belong on one XCD.  Equal segments that follow each
// other do, too (8 x 16384 tokens, 4 heads of 64: 98 -> 94 us); those of a ragged batch are dealt one at a time, so that no XCD has the long
// sequences (50021 tokens in 37 sequences, 12 heads of 96 over 4 of 72, fp16: 180 -> 162).  The segment, and the workgroup's place in it.
__device__ inline uint32_t xcd_unit(uint32_t units, uint32_t per, bool equal, uint32_t &place) {
    const uint32_t i = blockIdx.x, k = i >> 3, round = per == 1 ? k : k / per;
    place = k - round * per;
    return equal ? (i & 7) * ((units + 7) / 8) + round : round * 8 + (i & 7);
}
inline long xcd_blocks(long groups, long per) { return (groups + 7) / 8 * 8 * per; }

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
    SA_REQUIRE(stride < (1L << 22), SA_ERR_UNSUPPORTED, "%s: the tokens of %s are too far apart (stride %ld)", what, name, stride);
    SA_REQUIRE(aligned16(p) && stride % (type == SA_F32 ? 4 : 8) == 0, SA_ERR_ALIGN, "%s: the rows of %s must be 16-byte aligned", what, name);
    return SA_OK;
}

#define SA_TRY(call) \
    do {             \
        if (const int rc_ = (call); rc_ != SA_OK) return rc_; \
    } while (0)

}  // namespace decay
}  // namespace sa
