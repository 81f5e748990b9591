// Linear attention with a decay for each head over whole sequences, and its gradient.
//
//   S_t = l S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t,  l = exp(g) of the key/value head
// over chunks of 64 tokens, S the state before the chunk, i and j places in it:
//   o_i = scale (sum_{j <= i} l^(i - j) (q_i k_j) v_j + l^(i + 1) q_i S),  S' = l^n S + sum_j l^(n - 1 - j) k_j v_j^T
// The gradient is the same operator three times, in the order of time or against it, with other rows in the places of q, k and v:
//   dq = (do, v, k) on S^T;  dv = (k, q, do) reversed, dk = (v, do, q) reversed, on R_t = l R_{t+1} + scale q_t do_t^T (dk: R^T)
// R begins with the gradient of the last state, which meets the last token undecayed, so in reversed time a state is read as it is and decays on
// its way on: l^i instead of l^(i + 1), l^(n - j) instead of l^(n - 1 - j) (`shift`).
//
// A chunk of 64 tokens: 32 have twice the state's ways to LDS, 128 twice the pairs of tokens.  Four wavefronts have 16 queries each, and 16 columns of the
// state each, which stays in their registers; what a chunk adds to it and what the next one reads of it go through LDS.
// Where sequences and states are too few to fill the GPU, sequences are cut into segments: what each adds to the state (decay_states_kernel), the states
// before them (decay_scan_kernel), the rows from there (decay_rows_kernel).  Keys and values are then read twice.  Few short sequences need
// no state (decay_short_kernel).
//
// What bounds it, with keys of up to 64 in 16 bits: memory.  8 x 16384 tokens, 4 heads of 64, bf16 (medians of launches one after the other): rows 54 us (268 MB,
// 5 TB/s), sums of the segments 34 (134 MB), their scan 7.6; 64 x 197 tokens, 12 heads of 64, one pass: 21 us (77 MB, 15 at a copy's rate).  Its gradient at 8 x 16384:
// rows 140 to 172 us, 805 MB through the memory-side cache of which 430 come from memory.  With keys of 128, latency: 16384 tokens, 16 heads of 128, bf16: rows 82 us (268 MB;
// vector ALU 31 %, LDS 37 %, matrix cores 21 % of the time), as the terms of the state take 70 KB of LDS and 187 registers leave two wavefronts to a SIMD.  The same of
// fp32, whose operands are three terms: 8 x 16384 tokens, 4 heads of 64: 238 us in all (537 MB, 107 us).
#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "common.h"
#include "decay_attention.h"

namespace {

using namespace sa;
using namespace sa::decay;

// One operator: rows of q meet the keys k and values v of their key/value head.
struct Role {
    HeadRows q, k, v, out;   // out.width = v.width, k.width = q.width
    int outs;                // heads of q (and out) to a key/value head
    int sums;                // heads of k and v to one, which are added up
    int shift, reverse;
    int transposed;          // a state in memory has v's column for its row
    float inside, into, update;          // factors of (q k) v, of q S, of what is added to the state
    const float *first;      // [places][Hk][d][dv] or null: the state before the sequence
    float *last;             // or null: the state behind it
    const float *starts;     // or null: [places of the workspace][Hk][d][dv], the state before each segment
    float *sums_out;         // (states kernel) the same: what a segment adds to the state
};

struct Args {
    Role role[3];
    uint32_t shares[3];      // of a segment and key/value head: workgroups of the roles up to this one
    int roles;
    uint32_t units;          // segments
    Sequences seq;
    const float *g;
    int Hk, dv;              // (dv: columns of a state in memory)
    int state;               // elements of a state: d dv
    const int32_t *slots;
    int places;
    __device__ inline const float *place(const float *states, int p, int hk) const { return states + ((long)p * Hk + hk) * state; }
    __device__ inline float *place(float *states, int p, int hk) const { return states + ((long)p * Hk + hk) * state; }
};

// A kernel for keys of up to DK elements and HALVES * 64 columns of the result: 4 wavefronts to 64 columns.
template <class T_, int DK_, int HALVES_>
struct Shape {
    typedef T_ T;
    typedef typename Terms<T>::E E;
    static constexpr int DK = DK_, HALVES = HALVES_, RAW = Terms<T>::RAW, MADE = Terms<T>::MADE, ADDED = Terms<T>::ADDED;
    static constexpr bool SCALED = Terms<T>::SCALED;
    static constexpr int THREADS = 256 * HALVES, COLS = kHalf * HALVES;
    // Pitch of rows in LDS: 16 rows by 16 bytes (4.6 cycles of a CU a read; 8 with 16 bytes less, 16 without any) and transposed reads of 16 rows by
    // 32 bytes (4.3) meet each bank evenly.
    static constexpr int KP = DK + 16, VP = COLS + 16;
    // Columns of the values, and of the state, are in LDS in the order in which the product with them takes them: tile t's row 4 a + b is column
    // 16 a + 4 t + b of 64, so that a lane's results are 16 columns side by side while a tile's columns are side by side in LDS.
    // (fp16) The columns' scales are behind the values' rows, 8 to a row: 256 bytes more would be a workgroup less of keys of 96 on a CU.
    static __device__ inline float *down(E (*vl)[kChunk][VP], int at) { return reinterpret_cast<float *>(&vl[0][at >> 3][COLS]) + (at & 7); }
    // Values that are not finite: a zero takes their place in the products, as zero products of earlier rows with them would be NaN, and what comes behind them
    // is NaN in memory.  Behind the keys' rows in LDS, 8 to a row: each column's first place in the segment that has one, and whether any has.  (Looking for them
    // takes 0 to 3 % of a call, 7 of fp16 with keys of 128: 16384 tokens, 16 heads, 144 -> 154 us.)
    static constexpr int kNone = 0x7fffffff;
    static __device__ inline int *spoilt(E (*kl)[kChunk][KP], int at) { return reinterpret_cast<int *>(&kl[0][at >> 3][DK]) + (at & 7); }
    static __device__ inline int *any_spoilt(E (*kl)[kChunk][KP]) { return spoilt(kl, 128); }
    static __device__ inline void none_spoilt(E (*kl)[kChunk][KP]) {
        if ((int)threadIdx.x < COLS) *spoilt(kl, (int)threadIdx.x) = kNone;
        if ((int)threadIdx.x == COLS) *any_spoilt(kl) = 0;
    }
    static __device__ inline int column(int at) { return (at & ~63) + 16 * ((at & 15) >> 2) + 4 * ((at & 63) >> 4) + (at & 3); }
    static constexpr int KPIECES = kChunk * DK / 8 / THREADS, VPIECES = kChunk * COLS / 8 / THREADS;
    static constexpr int TILES = DK / 16;
    static_assert(kChunk * DK / 8 % THREADS == 0, "a thread has whole pieces of the keys");
};

// Where a workgroup's tokens are in one tensor: row i of chunk c is token first + c kChunk + i, or first - c kChunk - i.
struct Tokens {
    uint64_t base;           // of row 0 of the current chunk, or of row 63 where time is reversed
    int64_t next;            // bytes to the next chunk
    uint32_t pitch;          // bytes from token to token (of 64 tokens: 2^30 at most)
    bool reverse;
    template <class T>
    __device__ inline void set(const HeadRows &r, const Span &sp, int p0, bool reverse_, int head, int col) {
        reverse = reverse_;
        pitch = (uint32_t)r.stride * (uint32_t)sizeof(T);
        const long first = reverse ? (long)sp.begin + sp.length - p0 - kChunk : (long)sp.begin + p0;
        base = reinterpret_cast<uint64_t>(r.p) + (uint64_t)(first * (long)pitch) + (uint64_t)(head * r.width + col) * sizeof(T);
        next = (reverse ? -(int64_t)kChunk : (int64_t)kChunk) * (int64_t)pitch;
    }
    // The first n rows of the chunk: their memory alone is in the buffer, at row(i) - skipped(n) for row i.  All others' offsets are beyond it.
    __device__ inline uint32_t row(int i) const { return (uint32_t)(reverse ? kChunk - 1 - i : i) * pitch; }
    __device__ inline uint32_t skipped(int n) const { return reverse ? (uint32_t)(kChunk - n) * pitch : 0u; }
    __device__ inline __amdgpu_buffer_rsrc_t rows(int n, uint64_t more = 0) const { return buffer(base + more + skipped(n), (uint32_t)n * pitch); }
};

// The keys and values of one chunk: from memory to registers, from there to LDS.
template <class P>
struct Rows {
    typedef typename P::T T;
    typedef typename P::E E;
    static constexpr int KN = P::KPIECES, VN = P::VPIECES;
    Eight<T> k[KN], v[VN];
    uint32_t kat[KN], vat[VN];
    __device__ inline static int krow(int j) { return ((int)threadIdx.x + P::THREADS * j) / (P::DK / 8); }
    __device__ inline static int kcol(int j) { return ((int)threadIdx.x + P::THREADS * j) % (P::DK / 8) * 8; }
    __device__ inline static int vrow(int j) { return ((int)threadIdx.x + P::THREADS * j) / (P::COLS / 8); }
    __device__ inline static int vcol(int j) { return ((int)threadIdx.x + P::THREADS * j) % (P::COLS / 8) * 8; }
    __device__ inline void places(const Tokens &kt, int kwidth, const Tokens &vt, int vwidth) {
        each<KN>([&](auto j) { kat[j] = kcol(j) < kwidth ? kt.row(krow(j)) + kcol(j) * (uint32_t)sizeof(T) : kNowhere; });
        each<VN>([&](auto j) { vat[j] = vcol(j) < vwidth ? vt.row(vrow(j)) + vcol(j) * (uint32_t)sizeof(T) : kNowhere; });
    }
    __device__ inline void load(const Tokens &kt, const Tokens &vt, int n) {
        const __amdgpu_buffer_rsrc_t kp = kt.rows(n), vp = vt.rows(n);
        each<KN>([&](auto j) { k[j].load(kp, kat[j] - kt.skipped(n)); });
        each<VN>([&](auto j) { v[j].load(vp, vat[j] - vt.skipped(n)); });
    }
    // 8 columns are 4 of each of two tiles
    __device__ inline static int vplace(int col) { return (col & ~63) + 16 * ((col & 8) >> 2) + 4 * ((col & 63) >> 4); }
    // (the chunk begins at place c of the segment)
    __device__ inline static void remove(E (*kl)[kChunk][P::KP], E (*vl)[kChunk][P::VP], int c, int wave) {
        const int thread = thread_of(wave);
#pragma unroll 1
        for (int i = 0; i < 8 * VN; ++i) {
            const int piece = thread + P::THREADS * (i >> 3), row = piece / (P::COLS / 8), at = vplace(piece % (P::COLS / 8) * 8) + (i & 3) + 4 * (i & 4);
            if (!not_finite(vl[0][row][at])) continue;
            each<P::RAW>([&](auto p) { vl[p][row][at] = (E)0.0f; });
            atomicMin(P::spoilt(kl, at), c + row);
            *P::any_spoilt(kl) = 1;
        }
    }
    // Whether all values are finite as operands.
    __device__ inline bool stage(E (*kl)[kChunk][P::KP], E (*vl)[kChunk][P::VP]) const {
        each<KN>([&](auto j_) {
            constexpr int j = j_;
            Vec<E, 8> t[P::RAW];
            k[j].terms(t);
            each<P::RAW>([&](auto p) { *reinterpret_cast<Vec<E, 8> *>(&kl[p][krow(j)][kcol(j)]) = t[p]; });
        });
        float nothing = 0.0f;        // NaN else
        each<VN>([&](auto j_) {
            constexpr int j = j_;
            Vec<E, 8> t[P::RAW];
            v[j].terms(t);
            each<4>([&](auto i) { nothing = times_zero(Vec<E, 2>{t[0][2 * i], t[0][2 * i + 1]}, nothing); });
            each<P::RAW>([&](auto p_) {
                constexpr int p = p_;
                E *to = &vl[p][vrow(j)][vplace(vcol(j))];
                *reinterpret_cast<Vec<E, 4> *>(to) = __builtin_shufflevector(t[p], t[p], 0, 1, 2, 3);
                *reinterpret_cast<Vec<E, 4> *>(to + 16) = __builtin_shufflevector(t[p], t[p], 4, 5, 6, 7);
            });
        });
        return nothing == 0.0f;
    }
};

// The state of a slice, in registers: wavefront w has the columns that LDS has at 16 w to 16 w + 15, lane l rows 16 t + 4 (l / 16) + r of the one at l % 16.
template <class P>
struct State {
    typedef typename P::E E;
    f4 s[P::TILES];
    __device__ inline void clear() {
        each<P::TILES>([&](auto t) { s[t] = zeros(); });
    }
    // Four rows of a lane are side by side in memory where the state lies there transposed.
    __device__ inline void load(const float *p, bool transposed, int rows, int cols, int dv, int c0) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, col = c0 + P::column(16 * ((int)threadIdx.x >> 6) + (lane & 15));
        clear();
        if (col >= cols) return;
        each<P::TILES>([&](auto t_) {
            constexpr int t = t_;
            const int row = 16 * t + 4 * g;
            if (row >= rows) return;
            if (transposed) {
                s[t] = *reinterpret_cast<const f4 *>(p + col * dv + row);
            } else {
                each<4>([&](auto i_) {
                    constexpr int i = i_;
                    s[t][i] = p[(row + i) * dv + col];
                });
            }
        });
    }
    __device__ inline void store(float *p, bool transposed, int rows, int cols, int dv, int c0, int thread) const {
        const int lane = thread & 63, g = lane >> 4, col = c0 + P::column(16 * (thread >> 6) + (lane & 15));
        if (col >= cols) return;
        each<P::TILES>([&](auto t_) {
            constexpr int t = t_;
            const int row = 16 * t + 4 * g;
            if (row >= rows) return;
            if (transposed) {
                *reinterpret_cast<f4 *>(p + col * dv + row) = s[t];
            } else {
                each<4>([&](auto i_) {
                    constexpr int i = i_;
                    p[(row + i) * dv + col] = s[t][i];
                });
            }
        });
    }
    __device__ inline void spoil(E (*kl)[kChunk][P::KP], int thread) {
        if (*P::spoilt(kl, 16 * (thread >> 6) + (thread & 15)) == P::kNone) return;
        each<P::TILES>([&](auto t) { s[t] = f4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")}; });
    }
    // To LDS as terms, for the product with q: [column][row].
    __device__ inline void stage(E (*sl)[P::COLS][P::KP], E (*vl)[kChunk][P::VP]) const {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, at = 16 * ((int)threadIdx.x >> 6) + (lane & 15);
        float up = 1.0f;
        if constexpr (P::SCALED) {
            float m = 0.0f;
            each<P::TILES>([&](auto t_) {
                constexpr int t = t_;
                const float x[4] = {s[t][0], s[t][1], s[t][2], s[t][3]};
                m = largest(x, m);
            });
            const Scale scale(column_max(m));
            up = scale.up;
            if (g == 0) *P::down(vl, at) = scale.down;
        }
        each<P::TILES>([&](auto t_) {
            constexpr int t = t_;
            const float x[4] = {s[t][0], s[t][1], s[t][2], s[t][3]};
            Vec<E, 4> p[P::MADE];
            split(x, p, up);
            each<P::MADE>([&](auto n_) {
                constexpr int n = n_;
                *reinterpret_cast<Vec<E, 4> *>(&sl[n][at][16 * t + 4 * g]) = p[n];
            });
        });
    }
    // S = carry S + sum_j weight[j] k_j v_j^T over the chunk in LDS.  Both operands have tokens for the places of the sum: transposed
    // reads, in the order 32 s + 16 (e / 4) + 4 (l / 16) + e % 4 for element e.
    // TERMS: of what is added to the state.  WHOLE (fp16): for a state in memory, whose elements have fp32's precision of what they are made of, small values
    // alone where the large ones' keys are zero.  Two terms behind one power of two hold 22 bits of what is above 2^-18 of the column's largest; what is
    // below is looked at, and has turns of its own if it matters (50021 tokens in 37 sequences, 4 of 96 x 72: sums 33 -> 38 us; heads of fast decay look).
    template <int TERMS, bool WHOLE>
    __device__ inline void update(const E (*kl)[kChunk][P::KP], const E (*vl)[kChunk][P::VP], const float *weight, float carry) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, w = (int)threadIdx.x >> 6, row = 4 * g + (i >> 2), col = 4 * (i & 3);
        auto decayed = [&](auto ks, float (&x)[8]) {
            const f4 w0 = *reinterpret_cast<const f4 *>(&weight[32 * ks + 4 * g]), w1 = *reinterpret_cast<const f4 *>(&weight[32 * ks + 16 + 4 * g]);
            Vec<E, 8> raw[P::RAW];
            each<P::RAW>([&](auto p) {
                raw[p] = join<E>(read_transposed(&vl[p][32 * ks + row][16 * w + col]), read_transposed(&vl[p][32 * ks + 16 + row][16 * w + col]));
            });
            each<8>([&](auto e) {
                float y = (float)raw[P::RAW - 1][(int)e];
                each<P::RAW - 1>([&](auto p) { y += (float)raw[P::RAW - 2 - p][(int)e]; });
                x[e] = y * (e < 4 ? w0[e & 3] : w1[e & 3]);
            });
        };
        auto keys = [&](auto ks, auto t, Vec<E, 8> (&a)[P::RAW]) {
            each<P::RAW>([&](auto p) {
                a[p] = join<E>(read_transposed(&kl[p][32 * ks + row][16 * t + col]), read_transposed(&kl[p][32 * ks + 16 + row][16 * t + col]));
            });
        };
        if constexpr (P::SCALED) {
            float below = __builtin_inff();
            bool more = false;       // turns, each of the values that hold their bits behind its power of two
            do {
                float x0[8], x1[8];
                decayed(std::integral_constant<int, 0>(), x0);
                decayed(std::integral_constant<int, 1>(), x1);
                // (the first turn has what is not finite, too)
                if (more) each<8>([&](auto e) { x0[e] = fabsf(x0[e]) >= below ? 0.0f : x0[e], x1[e] = fabsf(x1[e]) >= below ? 0.0f : x1[e]; });
                const float top = column_max(largest(x1, largest(x0)));
                const Scale scale(top);
                const float kept = more ? 1.0f : carry;
                below = scale.down > 0x1p-126f ? 0.125f * scale.down : 0.0f;          // (behind the last power of two nothing is left)
                const bool some = WHOLE && __any(least(x1, least(x0)) < __builtin_bit_cast(uint32_t, below) << 1);
                // What is below 2^-18 of the largest would be off by 2^-25 scale.down.  That matters where this, times the keys' magnitudes, is above 2^-19 of
                // what all is together: where sum |k| (1 - 64 |x| scale.up) is positive, the large values' keys (next to) zero.
                if (some && !more) {
                    float most = 0.0f;
                    Vec<E, 8> sign[2];
                    each<8>([&](auto e) {
                        sign[0][(int)e] = (E)(1.0f - fminf(fabsf(x0[e]) * scale.up * 64.0f, 0x1p14f));
                        sign[1][(int)e] = (E)(1.0f - fminf(fabsf(x1[e]) * scale.up * 64.0f, 0x1p14f));
                    });
                    each<P::TILES>([&](auto t) {
                        __builtin_amdgcn_sched_barrier(0);
                        f4 sum = zeros();
                        each<2>([&](auto ks) {
                            Vec<E, 8> a[P::RAW];
                            keys(ks, t, a);
                            const u4 size = __builtin_bit_cast(u4, a[0]) & 0x7fff7fffu;
                            sum = matrix(__builtin_bit_cast(Vec<E, 8>, size), sign[ks], sum);
                        });
                        each<4>([&](auto e) { most = fmaxf(most, sum[(int)e] < __builtin_inff() ? sum[(int)e] : 0.0f); });       // (a row that is not finite has no say)
                    });
                    __builtin_amdgcn_sched_barrier(0);
                    more = __any(top > 0.0f && most > 0.0f);          // (not in a column of zeros, as those behind the last are)
                } else {
                    more = some;
                }
                if (more) each<8>([&](auto e) { x0[e] = fabsf(x0[e]) < below ? 0.0f : x0[e], x1[e] = fabsf(x1[e]) < below ? 0.0f : x1[e]; });
                Vec<E, 8> b[2][TERMS];
                split(x0, b[0], scale.up);
                split(x1, b[1], scale.up);
                each<P::TILES>([&](auto t) {
                    f4 add = zeros();
                    each<2>([&](auto ks) {
                        Vec<E, 8> a[P::RAW];
                        keys(ks, t, a);
                        product<Terms<typename P::T>::ORDER_ADDED>(add, a, b[ks]);
                    });
                    each<4>([&](auto e) { s[t][(int)e] = __builtin_fmaf(add[(int)e], scale.down, s[t][(int)e] * kept); });
                });
            } while (more);
        } else {
            each<P::TILES>([&](auto t) { s[t] *= carry; });
            each<2>([&](auto ks) {
                float x[8];
                decayed(ks, x);
                Vec<E, 8> b[TERMS];
                split(x, b);
                each<P::TILES>([&](auto t) {
                    Vec<E, 8> a[P::RAW];
                    keys(ks, t, a);
                    product<Terms<typename P::T>::ORDER_ADDED>(s[t], a, b);
                });
            });
            settled(s);
        }
    }
};

// Decays of a chunk's n tokens on their way into the state, into LDS: exp(g (n - shift - j)) for token j.
__device__ inline void stage_weights(float *weight, float rate, int n, int shift, float factor) {
    const int j = (int)threadIdx.x;
    if (j < kChunk) weight[j] = n - shift - j >= 0 ? factor * decay_pow(rate, n - shift - j) : 0.0f;
}

// A sequence's place among the states; -1: none, it begins with zeros and leaves no state.
__device__ inline int state_place(const Args &a, int seq) {
    if (a.slots == nullptr) return seq;
    const int p = a.slots[seq];
    return p >= 0 && p < a.places ? p : -1;
}

// A workgroup's role, segment and key/value head and, of the role, its slice of columns (and head).
__device__ inline const Role &role_of(const Args &a, uint32_t &unit, int &hk, uint32_t &item) {
    const uint32_t per = a.shares[a.roles - 1];
    unit = uniform(xcd_unit(a.units, per * (uint32_t)a.Hk, a.seq.offsets == nullptr, item));
    hk = (int)uniform(per == 1 ? item : item / per);
    item = uniform(item - (uint32_t)hk * per);
    int r = 0;
    while (r + 1 < a.roles && item >= a.shares[r]) ++r;
    if (r > 0) item -= a.shares[r - 1];
    return a.role[r];
}

// The queries of a wavefront, as operands of the products with the keys and with the state.  Those in memory as one term are loaded into the operand's place.
template <class P>
struct Queries {
    typedef typename P::T T;
    typedef typename P::E E;
    Vec<E, 8> t[P::DK / 32][P::RAW];
    Eight<T> raw[P::RAW > 1 ? P::DK / 32 : 1];
    __device__ inline void load(const Tokens &qt, uint32_t at, int n, int width) {
        const __amdgpu_buffer_rsrc_t from = qt.rows(n);
        const int g = ((int)threadIdx.x & 63) >> 4;
        at -= qt.skipped(n);
        each<P::DK / 32>([&](auto s) {
            const uint32_t place = 32 * s + 8 * g < width ? at + 32 * s * (uint32_t)sizeof(T) : kNowhere;
            if constexpr (P::RAW > 1) {
                raw[s].load(from, place);
            } else {
                Eight<T> x;
                x.load(from, place);
                t[s][0] = x.v;
            }
        });
    }
    // Has them there: what is asked for behind this is not waited for with them.
    __device__ inline void arrived() {
        each<P::DK / 32>([&](auto s) {
            if constexpr (P::RAW > 1) {
                raw[s].terms(t[s]);
            } else {
                u4 words = __builtin_bit_cast(u4, t[s][0]);
                asm volatile("" : "+v"(words));
                t[s][0] = __builtin_bit_cast(Vec<E, 8>, words);
            }
        });
    }
};

// o += sum_j exp(g (i - j)) (q_i k_j) v_j for the keys in LDS: those of the queries' own chunk, of which wavefront W has queries 16 W to 16 W + 15, or
// all 64 of an earlier one (W = 4).  (k_j q_i) comes out in the registers of the lanes that have it as the right operand of the product
// with v.  Decays: `inside` within a tile of 16 x 16; of earlier tiles `from_first`, which counts from the tile's (the chunk's) first
// query, and `behind`, which counts to it from the keys of 64 places before.
template <class P, int W, class F>
__device__ inline void add_values(f4 (&o)[4], const Vec<typename P::E, 8> (&q)[P::DK / 32][P::RAW], const typename P::E (*kl)[kChunk][P::KP],
                                  const typename P::E (*vl)[kChunk][P::VP], int half, const f4 &inside, float from_first, const float *behind, F keys_done) {
    typedef typename P::E E;
    typedef Terms<typename P::T> N;
    constexpr int TILES = W < 4 ? W + 1 : 4, STEPS = (TILES + 1) / 2;        // of 16 keys; of 32
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    float x[STEPS][8];
    each<2 * STEPS>([&](auto tile) {
        constexpr int t = tile;
        if constexpr (t < TILES) {
            f4 s = f4{0.0f, 0.0f, 0.0f, 0.0f};
            each<P::DK / 32>([&](auto d) {
                Vec<E, 8> kterms[P::RAW];
                each<P::RAW>([&](auto p) { kterms[p] = *reinterpret_cast<const Vec<E, 8> *>(&kl[p][16 * t + i][32 * d + 8 * g]); });
                product<N::ORDER_RAW>(s, kterms, q[d]);
            });
            if constexpr (t == W) {      // (a product that is not in the sum may be infinite)
                each<4>([&](auto e) { x[t / 2][4 * (t % 2) + e] = i >= 4 * g + e ? s[(int)e] * inside[(int)e] : 0.0f; });
            } else {
                const f4 far = *reinterpret_cast<const f4 *>(&behind[kChunk - 16 * (W - t) + 4 * g]);
                each<4>([&](auto e) { x[t / 2][4 * (t % 2) + e] = s[(int)e] * from_first * far[(int)e]; });
            }
        } else {
            each<4>([&](auto e) { x[t / 2][4 * (t % 2) + e] = 0.0f; });
        }
    });
    keys_done();
    float up = 1.0f, back = 1.0f;
    if constexpr (P::SCALED) {
        float m = 0.0f;
        each<STEPS>([&](auto ks) { m = largest(x[ks], m); });
        const Scale scale(column_max(m));
        up = scale.up, back = scale.down;
    }
    Vec<E, 8> pt[STEPS][P::MADE];
    each<STEPS>([&](auto ks) { split(x[ks], pt[ks], up); });
    each<4>([&](auto t) {
        const int row = 4 * g + (i >> 2), col = half + 16 * t + 4 * (i & 3);
        f4 sum = P::SCALED ? zeros() : o[t];
        each<STEPS>([&](auto ks) {
            Vec<E, 8> vterms[P::RAW];
            each<P::RAW>([&](auto p) {
                vterms[p] = join<E>(read_transposed(&vl[p][32 * ks + row][col]), read_transposed(&vl[p][32 * ks + row + 16][col]));
            });
            product<N::ORDER>(sum, vterms, pt[ks]);
        });
        if constexpr (P::SCALED) {
            each<4>([&](auto e) { o[t][(int)e] = __builtin_fmaf(sum[(int)e], back, o[t][(int)e]); });
        } else {
            o[t] = sum;
        }
    });
    settled(o);
}

// The same for a wavefront's own chunk: each wavefront has code of its own, without a branch in it, so that loads and products of its tiles overlap.
template <class P, class F>
__device__ inline void add_own_values(f4 (&o)[4], const Vec<typename P::E, 8> (&q)[P::DK / 32][P::RAW], const typename P::E (*kl)[kChunk][P::KP],
                                      const typename P::E (*vl)[kChunk][P::VP], int w, int half, const f4 &inside, float from_first, const float *behind,
                                      F keys_done) {
    if (w == 0) add_values<P, 0>(o, q, kl, vl, half, inside, from_first, behind, keys_done);
    else if (w == 1) add_values<P, 1>(o, q, kl, vl, half, inside, from_first, behind, keys_done);
    else if (w == 2) add_values<P, 2>(o, q, kl, vl, half, inside, from_first, behind, keys_done);
    else add_values<P, 3>(o, q, kl, vl, half, inside, from_first, behind, keys_done);
}

// Results of the chunk at place c of the segment behind values that are not finite.
template <class P>
__device__ inline void spoil_rows(f4 (&o)[4], typename P::E (*kl)[kChunk][P::KP], int c, int wave) {
    typedef int i4 __attribute__((ext_vector_type(4)));
    const int thread = thread_of(wave), g = (thread & 63) >> 4, half = kHalf * (thread >> 8), query = c + 16 * (thread >> 6 & 3) + (thread & 15);
    each<4>([&](auto t) {
        const i4 first = *reinterpret_cast<const i4 *>(P::spoilt(kl, half + 16 * t + 4 * g));
        each<4>([&](auto e) { o[t][(int)e] = query >= first[(int)e] ? __builtin_nanf("") : o[t][(int)e]; });
    });
}

// Wavefronts on a SIMD: as many workgroups as have room for their rows in a CU's LDS, unless registers would go to scratch memory, whose loads wait for
// the rows that are under way (8 x 16384 tokens, 4 heads of 64, bf16: 65 us with 165 registers, 93 with 168 and 22 in memory).
template <class P>
constexpr int rows_waves() {
    return P::RAW == 3 ? (P::DK <= 32 || P::HALVES == 2 ? 2 : 1) : P::DK <= 96 ? 3 : 2;
}

// Rows of the result.  A workgroup has one segment, the heads of one state (their keys, values and state are in LDS once for all of them: 12 heads of 96
// over 4 of 72 250 -> 203 us) and a slice of the columns and goes through the chunks one after the other;
// of each half of the slice, wavefront w has queries 16 w to 16 w + 15 of a chunk, and columns 16 w to 16 w + 15 of the state.
// LAST: a role leaves its last state (of fp16 another kernel: a loop in it keeps loads from their places, rows of the ragged batch's gradient 114 -> 128 us).
template <class P, bool STREAM, bool LAST>
__global__ __launch_bounds__(P::THREADS, (rows_waves<P>())) void decay_rows_kernel(const Args a) {
    typedef typename P::T T;
    typedef typename P::E E;
    constexpr int DK = P::DK;
    __shared__ __attribute__((aligned(16))) E kl[P::RAW][kChunk][P::KP];
    __shared__ __attribute__((aligned(16))) E vl[P::RAW][kChunk][P::VP];
    __shared__ __attribute__((aligned(16))) E sl[P::MADE][P::COLS][P::KP];
    __shared__ __attribute__((aligned(16))) float weight[kChunk], behind[kChunk];      // exp(g (64 - j)) in the latter
    P::none_spoilt(kl);
    uint32_t unit, item;
    int hk;
    const Role &r = role_of(a, unit, hk, item);
    if (unit >= a.units) return;
    const int kwidth = r.k.width, vwidth = r.v.width, sums = r.sums, outs = r.outs, shift = r.shift;
    const float update = r.update;
    const bool transposed = r.transposed, reverse = r.reverse;
    const int c0 = (int)item * P::COLS;
    State<P> state;
    const bool early = r.starts != nullptr && !a.seq.whole;       // (asked for first: it takes nothing but the segment's number to find it)
    if (early) state.load(a.place(r.starts, (int)unit, hk), transposed, kwidth, vwidth, a.dv, c0);
    else state.clear();
    const Span sp = a.seq.of_unit(unit);
    const int p0 = sp.seg * a.seq.seg, left = sp.length - p0;
    if (sp.seg < 0 || (left <= 0 && (sp.seg > 0 || r.last == nullptr))) return;
    const bool segments = r.starts != nullptr && a.seq.cut(sp.length);
    const int tokens = left < a.seq.seg ? left : a.seq.seg;

    const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int w = wave & 3, half = kHalf * (wave >> 2), query = 16 * w + i;
    const float rate = uniform(decay_rate(a.g[hk]));
    const int chunks = (tokens + kChunk - 1) / kChunk;
    auto in_chunk = [&](int c) { return tokens - c * kChunk < kChunk ? tokens - c * kChunk : kChunk; };

    Tokens qt, kt, vt, ot;
    qt.set<T>(r.q, sp, p0, reverse, hk * outs, 0);
    ot.set<T>(r.out, sp, p0, reverse, hk * outs, c0);
    kt.set<T>(r.k, sp, p0, reverse, hk * sums, 0);
    vt.set<T>(r.v, sp, p0, reverse, hk * sums, c0);
    const uint32_t kmore = (uint32_t)kwidth * (uint32_t)sizeof(T), vmore = (uint32_t)vwidth * (uint32_t)sizeof(T);     // to the next head
    const uint32_t qat = qt.row(query) + 8 * g * (uint32_t)sizeof(T), oat = ot.row(query) + (half + 16 * g) * (uint32_t)sizeof(T);
    Rows<P> rows;
    rows.places(kt, kwidth, vt, vwidth - c0);
    Queries<P> q;

    const int place = r.first != nullptr || r.last != nullptr ? state_place(a, sp.seq) : -1;
    float *const last = r.last != nullptr && !segments && place >= 0 ? a.place(r.last, place, hk) : nullptr;
    bool live = segments || (r.first != nullptr && place >= 0);      // a state that is not zero
    if (live && !early) state.load(segments ? a.place(r.starts, sp.place, hk) : a.place(r.first, place, hk), transposed, kwidth, vwidth, a.dv, c0);

    // Loads and stores come back in the order in which they left, and the compiler counts those behind the one it waits for, the fewest that may be there
    // on any way to that place.  So every turn of the loop asks for as many rows and queries and stores as many, and what is
    // not needed goes nowhere; and the loop is entered as it is entered again, keys and values before queries before stores.  (With branches around
    // them each chunk waited for the rows of the next one and for the stores of the last.)
    rows.load(kt, vt, chunks > 0 ? in_chunk(0) : 0);
    q.load(qt, qat, chunks > 0 ? in_chunk(0) : 0, kwidth);
    auto store = [&](int n, uint64_t more, const f4 (&o)[4]) {
        const __amdgpu_buffer_rsrc_t to = ot.rows(n, more);
        each<2>([&](auto p) {
            float x[8];
            each<8>([&](auto e) { x[e] = o[2 * p + e / 4][e % 4]; });
            store_eight<T, STREAM>(to, c0 + half + 16 * g + 8 * p < vwidth ? oat - ot.skipped(n) + 8 * p * (uint32_t)sizeof(T) : kNowhere, x);
        });
    };
    stage_weights(weight, rate, kChunk < tokens ? kChunk : tokens, shift, update);
    stage_weights(behind, rate, kChunk, 0, 1.0f);
    const float from_first = decay_pow(rate, i), scale = r.inside, into = uniform(r.into * decay_pow(rate, 16 * w + shift));
    f4 inside;
    each<4>([&](auto e) { inside[(int)e] = i >= 4 * g + e ? scale * decay_pow(rate, i - 4 * g - e) : 0.0f; });
    float carry = uniform(decay_pow(rate, kChunk));

    f4 o[4];
    each<4>([&](auto t) { o[t] = zeros(); });
    store(0, 0, o);
    // h: of several heads of keys and values that are added up; u: of several heads of queries.  One of the two has more than one.
    for (int c = 0; c < chunks; ++c) {
        const int n = in_chunk(c), next = c + 1 < chunks ? in_chunk(c + 1) : 0;
        const bool add = next > 0 || last != nullptr;
        if (n < kChunk) carry = uniform(decay_pow(rate, n));
        int h = 0;
        do {
            __syncthreads();
            if (__builtin_expect(!rows.stage(kl, vl), 0)) rows.remove(kl, vl, c * kChunk, wave);
            if (h == 0) {
                if (n < kChunk && c > 0) stage_weights(weight, rate, n, shift, update);
                if (live) state.stage(sl, vl);
            }
            if (h == 0 || P::RAW == 1) q.arrived();          // (ahead of the next rows, which they would be waited for with)
            const bool end = h + 1 == sums;
            kt.base += end ? (uint64_t)kt.next - (uint64_t)(sums - 1) * kmore : kmore;
            vt.base += end ? (uint64_t)vt.next - (uint64_t)(sums - 1) * vmore : vmore;
            rows.load(kt, vt, end ? next : n);
            __syncthreads();
            const int spoilt = *P::any_spoilt(kl);
            int u = 0;
            do {
                // (where they are is settled here: a branch between products and what reads them is one too many)
                const bool turn = u + 1 == outs;
                if (end) qt.base += turn ? (uint64_t)qt.next - (uint64_t)(outs - 1) * kmore : kmore;
                const int next_n = turn && end ? next : n;
                auto next_q = [&] { q.load(qt, qat, next_n, kwidth); };      // (the same again for the next head of the keys)
                if (u > 0) q.arrived();
                if (h == 0) each<4>([&](auto t) { o[t] = zeros(); });
                float decayed = from_first;
                if constexpr (P::SCALED) asm("" : "+v"(decayed));        // (its products are made here again: with them kept, keys of 64 are a register short)
                if (h == 0 && live) {
                    each<DK / 32>([&](auto s) {
                        each<4>([&](auto t) {
                            Vec<E, 8> st[P::MADE];
                            each<P::MADE>([&](auto p) { st[p] = *reinterpret_cast<const Vec<E, 8> *>(&sl[p][half + 16 * t + i][32 * s + 8 * g]); });
                            product<Terms<T>::ORDER>(o[t], st, q.t[s]);
                        });
                    });
                    each<4>([&](auto t) {
                        if constexpr (P::SCALED) {
                            o[t] *= *reinterpret_cast<const f4 *>(P::down(vl, half + 16 * t + 4 * g)) * (decayed * into);
                        } else {
                            o[t] *= decayed * into;
                        }
                    });
                }
                add_own_values<P>(o, q.t, kl, vl, w, half, inside, scale * decayed, behind, next_q);
                if (uniform((uint32_t)spoilt) != 0) spoil_rows<P>(o, kl, c * kChunk, wave);
                store(end ? n : 0, (uint64_t)u * vmore, o);
            } while (++u < outs);
            // (a state that only rows in 16 bits are made of takes the terms that these do)
            if (add) {
                if (P::MADE == P::ADDED || last != nullptr) state.template update<P::ADDED, P::SCALED && LAST>(kl, vl, weight, h == 0 ? carry : 1.0f);
                else state.template update<P::MADE, false>(kl, vl, weight, h == 0 ? carry : 1.0f);
            }
        } while (++h < sums);
        ot.base += (uint64_t)ot.next;
        live = live || add;
    }
    if (last != nullptr) {
        const int thread = thread_of(wave);
        if (chunks > 0) state.spoil(kl, thread);
        state.store(last, transposed, kwidth, vwidth, a.dv, c0, thread);
    }
}

// Few short sequences without a state before or behind them (197 tokens, 3 heads of 64, fp32: 21 -> 12 us on the device; with 768 sequences and heads of 197
// tokens one pass is faster, 20.5 us to 24.6): a workgroup has 64 queries of one head and a slice of the columns, and adds the values of
// all keys up to them, chunk by chunk, without a state: all queries at once instead of one chunk after the other.
template <class P>
__global__ __launch_bounds__(P::THREADS, (rows_waves<P>())) void decay_short_kernel(const Args a) {
    typedef typename P::T T;
    typedef typename P::E E;
    __shared__ __attribute__((aligned(16))) E kl[P::RAW][kChunk][P::KP];
    __shared__ __attribute__((aligned(16))) E vl[P::RAW][kChunk][P::VP];
    __shared__ __attribute__((aligned(16))) float behind[kChunk];
    P::none_spoilt(kl);
    uint32_t unit, item;
    int hk;
    const Role &r = role_of(a, unit, hk, item);
    if (unit >= a.units) return;
    const int kwidth = r.k.width, vwidth = r.v.width, sums = r.sums;
    const bool reverse = r.reverse;
    const uint32_t slices = vwidth > P::COLS ? 2 : 1;
    const int sub = (int)(slices == 2 ? item >> 1 : item), c0 = (int)(slices == 2 ? item & 1 : 0) * P::COLS;
    const Span sp = a.seq.of_unit(unit);
    const int left = sp.length - sp.seg * kChunk;
    if (sp.seg < 0 || left <= 0) return;
    const int mine = left < kChunk ? left : kChunk;

    const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int w = wave & 3, half = kHalf * (wave >> 2), query = 16 * w + i;
    const float rate = uniform(decay_rate(a.g[hk]));
    Tokens qt, kt, vt, ot;
    qt.set<T>(r.q, sp, sp.seg * kChunk, reverse, hk * r.outs + sub, 0);
    ot.set<T>(r.out, sp, sp.seg * kChunk, reverse, hk * r.outs + sub, c0);
    kt.set<T>(r.k, sp, 0, reverse, hk * sums, 0);
    vt.set<T>(r.v, sp, 0, reverse, hk * sums, c0);
    const uint32_t kmore = (uint32_t)kwidth * (uint32_t)sizeof(T), vmore = (uint32_t)vwidth * (uint32_t)sizeof(T);
    const uint32_t qat = qt.row(query) + 8 * g * (uint32_t)sizeof(T), oat = ot.row(query) + (half + 16 * g) * (uint32_t)sizeof(T);
    Rows<P> rows;
    rows.places(kt, kwidth, vt, vwidth - c0);
    Queries<P> q;
    q.load(qt, qat, mine, kwidth);
    rows.load(kt, vt, sp.seg > 0 ? kChunk : mine);
    stage_weights(behind, rate, kChunk, 0, 1.0f);
    const float from_first = r.inside * decay_pow(rate, i);
    f4 inside;
    each<4>([&](auto e) { inside[(int)e] = i >= 4 * g + e ? r.inside * decay_pow(rate, i - 4 * g - e) : 0.0f; });
    f4 o[4];
    each<4>([&](auto t) { o[t] = zeros(); });
    q.arrived();
    for (int c = 0; c <= sp.seg; ++c) {
        for (int h = 0; h < sums; ++h) {
            __syncthreads();
            if (__builtin_expect(!rows.stage(kl, vl), 0)) rows.remove(kl, vl, c * kChunk, wave);
            const bool end = h + 1 == sums;
            kt.base += end ? (uint64_t)kt.next - (uint64_t)(sums - 1) * kmore : kmore;
            vt.base += end ? (uint64_t)vt.next - (uint64_t)(sums - 1) * vmore : vmore;
            rows.load(kt, vt, c + end < sp.seg ? kChunk : c + end == sp.seg ? mine : 0);
            __syncthreads();
            if (c < sp.seg) add_values<P, 4>(o, q.t, kl, vl, half, inside, r.inside * decay_pow(rate, query + kChunk * (sp.seg - c - 1)), behind, [] {});
            else add_own_values<P>(o, q.t, kl, vl, w, half, inside, from_first, behind, [] {});
        }
    }
    if (*P::any_spoilt(kl) != 0) spoil_rows<P>(o, kl, sp.seg * kChunk, wave);
    const __amdgpu_buffer_rsrc_t to = ot.rows(mine);
    each<2>([&](auto p) {
        float x[8];
        each<8>([&](auto e) { x[e] = o[2 * p + e / 4][e % 4]; });
        store_eight<T, false>(to, c0 + half + 16 * g + 8 * p < vwidth ? oat - ot.skipped(mine) + 8 * p * (uint32_t)sizeof(T) : kNowhere, x);
    });
}

// What each segment adds to the state, from a state of zeros.  The chunks' keys and values pass through LDS for the transposed reads alone.
template <class P, bool LAST>
__global__ __launch_bounds__(P::THREADS) void decay_states_kernel(const Args a) {
    typedef typename P::T T;
    typedef typename P::E E;
    __shared__ __attribute__((aligned(16))) E kl[P::RAW][kChunk][P::KP];
    __shared__ __attribute__((aligned(16))) E vl[P::RAW][kChunk][P::VP];
    uint32_t unit, item;
    int hk;
    const Role &r = role_of(a, unit, hk, item);
    if (unit >= a.units) return;
    const int kwidth = r.k.width, vwidth = r.v.width, sums = r.sums, shift = r.shift;
    const float update = r.update;
    const bool reverse = r.reverse;
    const int c0 = (int)item * P::COLS;
    const Span sp = a.seq.of_unit(unit);
    const int p0 = sp.seg * a.seq.seg, left = sp.length - p0;
    // the last segment's sum is for the state behind the sequence only
    if (sp.seg < 0 || left <= 0 || (left <= a.seq.seg && r.last == nullptr) || !a.seq.cut(sp.length)) return;
    const int tokens = left < a.seq.seg ? left : a.seq.seg, chunks = (tokens + kChunk - 1) / kChunk;
    const float rate = uniform(decay_rate(a.g[hk]));
    State<P> state;
    state.clear();
    auto in_chunk = [&](int c) { return tokens - c * kChunk < kChunk ? tokens - c * kChunk : kChunk; };
    Tokens kt, vt;
    kt.set<T>(r.k, sp, p0, reverse, hk * sums, 0);
    vt.set<T>(r.v, sp, p0, reverse, hk * sums, c0);
    const uint32_t kmore = (uint32_t)kwidth * (uint32_t)sizeof(T), vmore = (uint32_t)vwidth * (uint32_t)sizeof(T);
    Rows<P> rows;
    rows.places(kt, kwidth, vt, vwidth - c0);
    rows.load(kt, vt, in_chunk(0));
    __shared__ __attribute__((aligned(16))) float weight[kChunk];
    stage_weights(weight, rate, kChunk < tokens ? kChunk : tokens, shift, update);
    float carry = decay_pow(rate, kChunk);
    for (int c = 0; c < chunks; ++c) {
        const int n = in_chunk(c);
        if (n < kChunk) carry = uniform(decay_pow(rate, n));
        for (int h = 0; h < sums; ++h) {
            if (c + h > 0) __syncthreads();
            rows.stage(kl, vl);
            if (n < kChunk && c > 0 && h == 0) stage_weights(weight, rate, n, shift, update);
            const bool end = h + 1 == sums;
            kt.base += end ? (uint64_t)kt.next - (uint64_t)(sums - 1) * kmore : kmore;
            vt.base += end ? (uint64_t)vt.next - (uint64_t)(sums - 1) * vmore : vmore;
            rows.load(kt, vt, !end ? n : c + 1 < chunks ? in_chunk(c + 1) : 0);
            __syncthreads();
            if (P::MADE == P::ADDED || r.last != nullptr) state.template update<P::ADDED, P::SCALED && LAST>(kl, vl, weight, h == 0 ? carry : 1.0f);
            else state.template update<P::MADE, false>(kl, vl, weight, h == 0 ? carry : 1.0f);
        }
    }
    state.store(a.place(r.sums_out, sp.place, hk), r.transposed, kwidth, vwidth, a.dv, c0, (int)threadIdx.x);
}

// From the segments' sums to the states before them, in their place, and to the state behind the sequence.  A thread has 4 elements, 16 segments of them
// under way at a time (one at a time: 16384 tokens, 16 states of 128 x 128, 16 segments 13 -> 9 us).
constexpr int kScanThreads = 256;
__global__ __launch_bounds__(kScanThreads) void decay_scan_kernel(const Args a) {
    const Role &r = a.role[blockIdx.z];
    const int hk = (int)(blockIdx.y % (unsigned)a.Hk), b = (int)(blockIdx.y / (unsigned)a.Hk);
    const Span sp = a.seq.of_sequence(b);
    if (!a.seq.cut(sp.length)) return;
    const int place = r.first != nullptr || r.last != nullptr ? state_place(a, b) : -1;
    const int segs = (sp.length + a.seq.seg - 1) / a.seq.seg;
    const float rate = uniform(decay_rate(a.g[hk]));
    const long next = (long)a.Hk * a.state;
    const float whole = decay_pow(rate, a.seq.seg);
    const int sums = r.last != nullptr ? segs : segs - 1;    // (of the last segment only where the state behind it is asked for)
    constexpr int kAhead = 16;
    for (int at = (int)(blockIdx.x * kScanThreads + threadIdx.x) * 4; at < a.state; at += (int)gridDim.x * kScanThreads * 4) {
        f4 x = f4{0.0f, 0.0f, 0.0f, 0.0f};
        if (r.first != nullptr && place >= 0) x = *reinterpret_cast<const f4 *>(a.place(r.first, place, hk) + at);
        float *p = a.place(r.sums_out, sp.place, hk) + at;
        for (int s = 0; s < segs; s += kAhead) {
            f4 add[kAhead];
            each<kAhead>([&](auto k) { add[k] = s + k < sums ? *reinterpret_cast<const f4 *>(p + (s + k) * next) : f4{0.0f, 0.0f, 0.0f, 0.0f}; });
            each<kAhead>([&](auto k) {
                if (s + k >= segs) return;
                *reinterpret_cast<f4 *>(p + (s + k) * next) = x;
                x = x * (s + k + 1 == segs ? decay_pow(rate, sp.length - (s + k) * a.seq.seg) : whole) + add[k];
            });
        }
        if (r.last != nullptr && place >= 0) *reinterpret_cast<f4 *>(a.place(r.last, place, hk) + at) = x;
    }
}

// ------------------------------------------------------------------------------------------- plan --

// The kernel of a role: by the widths of its keys and of its result.  128 columns are eight wavefronts of one workgroup, which read the keys
// once, where two workgroups of four would not have room in a CU together (keys of 65 to 128 in 16 bits, of 33 to 64 in fp32); of fp32 with more than 64
// not even eight wavefronts' state has.
struct Form {
    int keys, halves;
    bool operator==(const Form &o) const { return keys == o.keys && halves == o.halves; }
};
Form form_of(int keys, int columns, int type) {
    Form f;
    f.keys = keys <= 32 ? 32 : keys <= 64 ? 64 : keys <= 96 ? 96 : 128;
    f.halves = columns > kHalf && f.keys == (type == SA_F32 ? 64 : 128) ? 2 : 1;
    return f;
}
Form form_of(const Role &r, int type) { return form_of(r.k.width, r.v.width, type); }
int slices_of(int columns, const Form &f) { return columns > kHalf * f.halves ? 2 : 1; }
// Workgroups of decay_rows_kernel that a CU has at once, by registers and LDS.
int resident(const Form &f, int type) { return type == SA_F32 ? (f.keys == 32 ? 2 : 1) : f.keys <= 96 ? 3 : f.halves == 2 ? 1 : 2; }

struct Plan {
    int seg = 0;             // 0: one pass
    int per_sequence = 1;
    bool shorts = false;     // decay_short_kernel, segments of 64 queries
    bool whole = false;      // sequences of one segment are rows from their own first state to their own last
};

// What a call's rows take: workgroups of a segment and key/value head, and how many of them fill the GPU.
struct Load {
    int workgroups, fill;
};
Load load_of(int type, std::initializer_list<std::pair<int, int>> roles) {       // keys' and results' widths
    Load l{0, 1 << 30};
    for (const auto &r : roles) {
        const Form f = form_of(r.first, r.second, type);
        l.workgroups += slices_of(r.second, f);
        l.fill = std::min(l.fill, 256 * resident(f, type));
    }
    return l;
}

constexpr long kThreads = 1L << 32;      // a launch has less

// Segments where sequences and states alone leave CUs without work, as many as fill them once, or where one long sequence among short ones would go on
// alone.
Plan make_plan(long T, int B, int H, int Hk, const Load &l, bool ragged, bool states) {
    Plan p;
    if (T == 0 || B == 0) return p;
    const long mean = (T + B - 1) / B, groups = (long)B * Hk * l.workgroups, longest = ragged ? T : T / B;
    const long kLeast = ragged ? 256 : 128;
    constexpr long kRagged = 4, kShort = 512;
    long seg = 0;
    if (!states && longest <= kShort && groups < l.fill && (T / kChunk + B + 8) * H * l.workgroups * 512 < kThreads) {
        p.shorts = true;
        seg = kChunk;
    } else if ((2 * groups <= l.fill || ragged) && longest > kLeast) {
        // (of a ragged batch four times as many: the GPU is busy as long as there are segments left, and its longest sequence may be many times the mean; no
        // more of them where there are more sequences and states than that)
        const long most = ragged ? kRagged * l.fill : l.fill;
        if (groups <= most) seg = (mean + most / groups - 1) / (most / groups);
        else seg = (long)((double)mean * (double)groups / (double)most);
        if (seg < kLeast) seg = kLeast;
        if (ragged && seg >= T) seg = 0;
    }
    if (!ragged && !p.shorts && seg >= T / B) seg = 0;
    if (seg > 0) {
        if (ragged) {
            long power = kChunk;
            while (2 * power <= seg) power *= 2;
            seg = power;
            // Of most sequences one segment: their states stay out of the workspace and their keys and values are read once
            p.whole = !p.shorts && seg >= mean;
        } else {
            seg = (seg + kChunk - 1) / kChunk * kChunk;
            p.per_sequence = (int)((T / B + seg - 1) / seg);
        }
    }
    p.seg = (int)seg;
    return p;
}

Sequences sequences(const int32_t *offsets, long T, int B, const Plan &p) {
    // one pass: one segment to a sequence, unit b is sequence b
    Sequences s{offsets, (int)T, B, offsets == nullptr ? (int)(T / B) : 0, p.seg > 0 ? p.seg : 1 << 30, 30, p.per_sequence, p.whole};
    while (s.log_seg > 0 && 1 << s.log_seg > s.seg) --s.log_seg;
    return s;
}

size_t plan_bytes(const Plan &p, long T, int B, bool ragged, int Hk, int d, int dv) {
    if (p.seg == 0 || p.shorts) return 0;
    const long places = p.whole ? 2 * (T / p.seg) : ragged ? T / p.seg + B : (long)p.per_sequence * B;
    return (size_t)places * Hk * d * dv * sizeof(float);
}

template <class F>
int by_form(int type, const Form &f, F run) {
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        if (f.halves == 2) return run(Shape<T, sizeof(T) == 4 ? 64 : 128, 2>());
        if (f.keys == 32) return run(Shape<T, 32, 1>());
        if (f.keys == 64) return run(Shape<T, 64, 1>());
        if (f.keys == 96) return run(Shape<T, 96, 1>());
        return run(Shape<T, 128, 1>());
    });
}

// Roles of one form are one launch.
template <class F>
int by_forms(const char *what, int type, const Args &a, int roles, bool shorts, F run) {
    bool done[3] = {false, false, false};
    for (int r = 0; r < roles; ++r) {
        if (done[r]) continue;
        const Form f = form_of(a.role[r], type);
        Args some = a;
        some.roles = 0;
        uint32_t shares = 0;
        for (int s = r; s < roles; ++s) {
            if (done[s] || !(form_of(a.role[s], type) == f)) continue;
            done[s] = true;
            shares += (uint32_t)((shorts ? a.role[s].outs : 1) * slices_of(a.role[s].v.width, f));
            some.role[some.roles] = a.role[s];
            some.shares[some.roles++] = shares;
        }
        const long total = xcd_blocks(a.seq.units(), (long)shares * a.Hk);
        some.units = (uint32_t)a.seq.units();
        SA_REQUIRE(total * 256 * f.halves < kThreads, SA_ERR_UNSUPPORTED, "%s: too many heads and tokens for one launch", what);
        SA_TRY(by_form(type, f, [&](auto shape) {
            run(shape, dim3((unsigned)total), some);
            return check_launch(what);
        }));
    }
    return SA_OK;
}

bool leaves_states(const Args &a) {
    for (int r = 0; r < a.roles; ++r)
        if (a.role[r].last != nullptr) return true;
    return false;
}

// f with the flag as a constant, where there are two kernels for it.
template <bool TWO, class F>
void by_flag(bool flag, F f) {
    if (TWO && !flag) f(std::integral_constant<bool, !TWO>());
    else f(std::true_type());
}

// The rows of all roles; before them, where there are segments, the sums of the first `states` roles and their scan.
int launch(const char *what, int type, Args a, const Plan &p, int states, hipStream_t st) {
    if (a.seq.units() == 0) return SA_OK;
    if (p.shorts) {
        return by_forms(what, type, a, a.roles, true, [&](auto shape, dim3 grid, const Args &some) {
            decay_short_kernel<decltype(shape)><<<grid, dim3(decltype(shape)::THREADS), 0, st>>>(some);
        });
    }
    if (p.seg > 0) {
        SA_TRY(by_forms(what, type, a, states, false, [&](auto shape, dim3 grid, const Args &some) {
            typedef decltype(shape) S;
            by_flag<S::SCALED>(leaves_states(some), [&](auto last) { decay_states_kernel<S, last><<<grid, dim3(S::THREADS), 0, st>>>(some); });
        }));
        // (where most sequences have nothing to scan, a quarter of the workgroups: 512 sequences of 100 tokens, 32 heads of 128, 95 -> 31 us)
        const int parts = (a.state / 4 + kScanThreads - 1) / kScanThreads;
        const dim3 grid((unsigned)(p.whole ? (parts + 3) / 4 : parts), (unsigned)(a.Hk * a.seq.B), (unsigned)states);
        decay_scan_kernel<<<grid, dim3(kScanThreads), 0, st>>>(a);
        SA_TRY(check_launch(what));
        for (int r = 0; r < a.roles && !p.whole; ++r) a.role[r].first = nullptr, a.role[r].last = nullptr;
    }
    return by_forms(what, type, a, a.roles, false, [&](auto shape, dim3 grid, const Args &some) {
        typedef decltype(shape) S;
        bool lines = true;
        for (int r = 0; r < some.roles; ++r) lines = lines && some.role[r].out.width * sizeof(typename S::T) % 128 == 0;
        by_flag<S::SCALED>(leaves_states(some), [&](auto last) {
            if (lines) decay_rows_kernel<S, true, last><<<grid, dim3(S::THREADS), 0, st>>>(some);
            else decay_rows_kernel<S, false, last><<<grid, dim3(S::THREADS), 0, st>>>(some);
        });
    });
}

int check_sequences(const char *what, int type, long T, int B, bool ragged, int H, int Hk, int d, int dv) {
    SA_TRY(check_heads(what, type, T, H, Hk, d, dv));
    SA_REQUIRE(B >= 0, SA_ERR_INVALID, "%s: B < 0", what);
    SA_REQUIRE(ragged || (B > 0 ? T % B == 0 : T == 0), SA_ERR_SHAPE, "%s: %ld tokens are no %d sequences of the same length", what, T, B);
    SA_REQUIRE(T < (1L << 30), SA_ERR_UNSUPPORTED, "%s: up to 2^30 tokens a call (got %ld)", what, T);
    SA_REQUIRE((long)B * Hk <= 65535, SA_ERR_UNSUPPORTED, "%s: up to 65535 states a call (got %d x %d)", what, B, Hk);
    return SA_OK;
}

}  // namespace

extern "C" size_t sa_decay_attention_workspace_bytes(long T, int B, int H, int Hk, int d, int dv, int ragged) {
    if (check_sequences("", SA_F32, T, B, ragged != 0, H, Hk, d, dv) != SA_OK) return 0;
    size_t most = 0;
    for (const int type : {SA_F32, SA_F16, SA_BF16})
        most = std::max(most, plan_bytes(make_plan(T, B, H, Hk, load_of(type, {{d, dv}}), ragged != 0, true), T, B, ragged != 0, Hk, d, dv));
    return most;
}

extern "C" int sa_decay_attention(const void *q, long q_stride, const void *k, long k_stride, const void *v, long v_stride, int type,
                                  const float *log_decay, long T, int B, const int32_t *offsets_or_null, int H, int Hk, int d, int dv, float scale,
                                  const float *state_in_or_null, float *state_out_or_null, const int32_t *slots_or_null, int n_slots, void *out,
                                  long out_stride, void *workspace, size_t workspace_bytes, void *stream) {
    const char *what = "sa_decay_attention";
    sa::clear_error();
    const bool ragged = offsets_or_null != nullptr;
    SA_TRY(check_sequences(what, type, T, B, ragged, H, Hk, d, dv));
    SA_REQUIRE(log_decay != nullptr, SA_ERR_INVALID, "%s: log_decay is NULL", what);
    SA_REQUIRE(slots_or_null == nullptr || n_slots >= 0, SA_ERR_INVALID, "%s: n_slots < 0", what);
    if (T > 0) {
        SA_TRY(check_rows(what, "q", q, q_stride, H, d, type));
        SA_TRY(check_rows(what, "k", k, k_stride, Hk, d, type));
        SA_TRY(check_rows(what, "v", v, v_stride, Hk, dv, type));
        SA_TRY(check_rows(what, "out", out, out_stride, H, dv, type));
        SA_REQUIRE(out != q && out != k && out != v, SA_ERR_INVALID, "%s: out must not be an input", what);
    }
    SA_REQUIRE(sa::aligned4(log_decay) && sa::aligned16(state_in_or_null) && sa::aligned16(state_out_or_null) && sa::aligned16(workspace) &&
                   sa::aligned4(offsets_or_null) && sa::aligned4(slots_or_null),
               SA_ERR_ALIGN, "%s: pointers must be 16-byte aligned", what);
    if (B == 0 || (T == 0 && state_out_or_null == nullptr)) return SA_OK;
    const Plan p = make_plan(T, B, H, Hk, load_of(type, {{d, dv}}), ragged, state_in_or_null != nullptr || state_out_or_null != nullptr);
    const size_t need = plan_bytes(p, T, B, ragged, Hk, d, dv);
    SA_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), SA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what,
               need, workspace_bytes);
    Args a{};
    a.roles = 1;
    a.seq = sequences(offsets_or_null, T, B, p);
    a.g = log_decay, a.Hk = Hk, a.dv = dv, a.state = d * dv, a.slots = slots_or_null, a.places = n_slots;
    Role &r = a.role[0];
    r.q = {q, q_stride, d}, r.k = {k, k_stride, d}, r.v = {v, v_stride, dv}, r.out = {out, out_stride, dv};
    r.outs = H / Hk, r.sums = 1, r.shift = 1;
    r.inside = scale, r.into = scale, r.update = 1.0f;
    r.first = state_in_or_null, r.last = state_out_or_null;
    if (p.seg > 0 && !p.shorts) r.starts = r.sums_out = static_cast<float *>(workspace);
    return launch(what, type, a, p, 1, sa::as_stream(stream));
}

extern "C" size_t sa_decay_attention_backward_workspace_bytes(long T, int B, int H, int Hk, int d, int dv, int ragged) {
    if (check_sequences("", SA_F32, T, B, ragged != 0, H, Hk, d, dv) != SA_OK) return 0;
    size_t most = 0;
    for (const int type : {SA_F32, SA_F16, SA_BF16})
        most = std::max(most, plan_bytes(make_plan(T, B, H, Hk, load_of(type, {{d, dv}, {dv, d}, {dv, d}}), ragged != 0, true), T, B, ragged != 0, Hk, d, dv));
    return 2 * most;
}

extern "C" int sa_decay_attention_backward(const void *dout, long dout_stride, const void *q, long q_stride, const void *k, long k_stride,
                                           const void *v, long v_stride, int type, const float *log_decay, long T, int B,
                                           const int32_t *offsets_or_null, int H, int Hk, int d, int dv, float scale, const float *state_in_or_null,
                                           const float *dstate_out_or_null, void *dq, long dq_stride, void *dk, long dk_stride, void *dv_rows,
                                           long dv_stride, float *dstate_in_or_null, void *workspace, size_t workspace_bytes, void *stream) {
    const char *what = "sa_decay_attention_backward";
    sa::clear_error();
    const bool ragged = offsets_or_null != nullptr;
    SA_TRY(check_sequences(what, type, T, B, ragged, H, Hk, d, dv));
    SA_REQUIRE(log_decay != nullptr, SA_ERR_INVALID, "%s: log_decay is NULL", what);
    if (T > 0) {
        SA_TRY(check_rows(what, "dout", dout, dout_stride, H, dv, type));
        SA_TRY(check_rows(what, "q", q, q_stride, H, d, type));
        SA_TRY(check_rows(what, "k", k, k_stride, Hk, d, type));
        SA_TRY(check_rows(what, "v", v, v_stride, Hk, dv, type));
        SA_TRY(check_rows(what, "dq", dq, dq_stride, H, d, type));
        SA_TRY(check_rows(what, "dk", dk, dk_stride, Hk, d, type));
        SA_TRY(check_rows(what, "dv", dv_rows, dv_stride, Hk, dv, type));
        const void *outs[] = {dq, dk, dv_rows}, *ins[] = {dout, q, k, v};
        for (int i = 0; i < 3; ++i) {
            for (const void *in : ins) SA_REQUIRE(outs[i] != in, SA_ERR_INVALID, "%s: a gradient must not be an input", what);
            SA_REQUIRE(outs[i] != outs[(i + 1) % 3], SA_ERR_INVALID, "%s: two gradients in one place", what);
        }
    }
    SA_REQUIRE(dstate_in_or_null == nullptr || (dstate_in_or_null != dstate_out_or_null && dstate_in_or_null != state_in_or_null), SA_ERR_INVALID,
               "%s: dstate_in must not be an input", what);
    SA_REQUIRE(sa::aligned4(log_decay) && sa::aligned16(state_in_or_null) && sa::aligned16(dstate_out_or_null) && sa::aligned16(dstate_in_or_null) &&
                   sa::aligned16(workspace) && sa::aligned4(offsets_or_null),
               SA_ERR_ALIGN, "%s: pointers must be 16-byte aligned", what);
    if (B == 0 || (T == 0 && dstate_in_or_null == nullptr)) return SA_OK;
    const Plan p = make_plan(T, B, H, Hk, load_of(type, {{d, dv}, {dv, d}, {dv, d}}), ragged, state_in_or_null != nullptr || dstate_out_or_null != nullptr || dstate_in_or_null != nullptr);
    const size_t each = plan_bytes(p, T, B, ragged, Hk, d, dv);
    SA_REQUIRE(each == 0 || (workspace != nullptr && workspace_bytes >= 2 * each), SA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given",
               what, 2 * each, workspace_bytes);
    Args a{};
    a.roles = 3;
    a.seq = sequences(offsets_or_null, T, B, p);
    a.g = log_decay, a.Hk = Hk, a.dv = dv, a.state = d * dv;
    const HeadRows rq{q, q_stride, d}, rk{k, k_stride, d}, rv{v, v_stride, dv}, ro{dout, dout_stride, dv};
    const int G = H / Hk;
    // dv and dq first: with segments, their roles are also those whose states are summed, R and (transposed) S
    Role &gv = a.role[0], &gq = a.role[1], &gk = a.role[2];
    gv.q = rk, gv.k = rq, gv.v = ro, gv.out = {dv_rows, dv_stride, dv};
    gq.q = ro, gq.k = rv, gq.v = rk, gq.out = {dq, dq_stride, d};
    gk.q = rv, gk.k = ro, gk.v = rq, gk.out = {dk, dk_stride, d};
    gv.outs = gk.outs = 1, gv.sums = gk.sums = G, gv.shift = gk.shift = 0, gv.reverse = gk.reverse = 1;
    gq.outs = G, gq.sums = 1, gq.shift = 1, gq.reverse = 0;
    gq.transposed = gk.transposed = 1;
    gv.inside = gk.inside = scale, gv.into = gk.into = 1.0f, gv.update = gk.update = scale;
    gq.inside = gq.into = scale, gq.update = 1.0f;
    gv.first = gk.first = dstate_out_or_null, gv.last = dstate_in_or_null;
    gq.first = state_in_or_null;
    if (p.seg > 0 && !p.shorts) {
        float *ws = static_cast<float *>(workspace);
        gv.starts = gv.sums_out = ws;
        gk.starts = ws;
        gq.starts = gq.sums_out = ws + each / sizeof(float);
    }
    return launch(what, type, a, p, 2, sa::as_stream(stream));
}
