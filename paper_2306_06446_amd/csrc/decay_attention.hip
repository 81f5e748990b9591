// Linear attention with a decay for each head over whole sequences, and its gradient.
//
//   S_t = l S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t,  l = exp(g) of the key/value head
// over chunks of 64 tokens, S the state before the chunk, i and j places in it:
//   o_i = scale (sum_{j <= i} l^(i - j) (q_i k_j) v_j + l^(i + 1) q_i S),  S' = l^n S + sum_j l^(n - 1 - j) k_j v_j^T
// The gradient is the same operator three times, in the order of time or against it, with other rows in the places of q, k and v:
//   dq = (do, v, k) on S^T;  dv = (k, q, do) reversed, dk = (v, do, q) reversed, on R_t = l R_{t+1} + scale q_t do_t^T (dk: R^T)
// R begins with the gradient of the last state, which meets the last token undecayed, so in reversed time a state is read as it is and decays on
// its way on: l^i instead of l^(i + 1), l^(n - j) instead of l^(n - 1 - j) (`shift`).
#include <type_traits>

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
    const float *starts;     // or null: [units][Hk][d][dv], the state before each segment
    float *sums_out;         // (states kernel) [units][Hk][d][dv]: what a segment adds to the state
};

struct Args {
    Role role[3];
    long items[3];           // of the roles before and with this one
    int roles;
    Sequences seq;
    const float *g;
    int Hk, dv;              // (dv: columns of a state in memory)
    long state;              // elements of a state: d dv
    const int32_t *slots;
    int places;
};

template <class T, int DK>
struct Shape {
    static constexpr int RAW = Terms<T>::RAW, MADE = Terms<T>::MADE;
    static constexpr int KP = DK + 8, VP = kSlice + 8;       // pitch: rows begin 4 banks apart
    static constexpr int KPIECES = DK / 32, VPIECES = kSlice / 32;
    static constexpr int TILES = DK / 16;
};

// The rows of one chunk: from memory to registers, from there to LDS.
template <class T, int DK>
struct Rows {
    using P = Shape<T, DK>;
    Eight<T> k[P::KPIECES], v[P::VPIECES];
    __device__ inline void load(const Role &r, long begin, long length, long pos, int n, int head, int c0) {
        const long dir = r.reverse ? -1 : 1, t0 = r.reverse ? begin + length - 1 - pos : begin + pos;
        const T *kp = static_cast<const T *>(r.k.p) + (long)head * r.k.width, *vp = static_cast<const T *>(r.v.p) + (long)head * r.v.width + c0;
#pragma unroll
        for (int j = 0; j < P::KPIECES; ++j) {
            const int at = (int)threadIdx.x + kThreads * j, row = at / (DK / 8), col = at % (DK / 8) * 8;
            if (row < n && col < r.k.width) k[j].load(kp + (t0 + dir * row) * r.k.stride + col);
            else k[j].zero();
        }
#pragma unroll
        for (int j = 0; j < P::VPIECES; ++j) {
            const int at = (int)threadIdx.x + kThreads * j, row = at / (kSlice / 8), col = at % (kSlice / 8) * 8;
            if (row < n && c0 + col < r.v.width) v[j].load(vp + (t0 + dir * row) * r.v.stride + col);
            else v[j].zero();
        }
    }
    __device__ inline void stage(__bf16 (*kl)[kChunk][P::KP], __bf16 (*vl)[kChunk][P::VP]) const {
#pragma unroll
        for (int j = 0; j < P::KPIECES; ++j) {
            const int at = (int)threadIdx.x + kThreads * j, row = at / (DK / 8), col = at % (DK / 8) * 8;
            b8 t[P::RAW];
            k[j].terms(t);
#pragma unroll
            for (int p = 0; p < P::RAW; ++p) *reinterpret_cast<b8 *>(&kl[p][row][col]) = t[p];
        }
#pragma unroll
        for (int j = 0; j < P::VPIECES; ++j) {
            const int at = (int)threadIdx.x + kThreads * j, row = at / (kSlice / 8), col = at % (kSlice / 8) * 8;
            b8 t[P::RAW];
            v[j].terms(t);
#pragma unroll
            for (int p = 0; p < P::RAW; ++p) *reinterpret_cast<b8 *>(&vl[p][row][col]) = t[p];
        }
    }
};

// The state of a slice, in registers: wavefront w has columns 16 w to 16 w + 15, lane l rows 16 t + 4 (l / 16) + r of column l % 16.
template <class T, int DK>
struct State {
    using P = Shape<T, DK>;
    f4 s[P::TILES];
    __device__ inline void clear() {
#pragma unroll
        for (int t = 0; t < P::TILES; ++t) s[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    template <class F>
    __device__ inline void each(const Role &r, int dv, int c0, F f) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, col = c0 + 16 * ((int)threadIdx.x >> 6) + (lane & 15);
#pragma unroll
        for (int t = 0; t < P::TILES; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * t + 4 * g + i;
                float x = s[t][i];
                if (row < r.k.width && col < r.v.width) f(r.transposed ? col * dv + row : row * dv + col, x);
                s[t][i] = x;
            }
        }
    }
    __device__ inline void load(const Role &r, const float *p, int dv, int c0) {
        each(r, dv, c0, [&](int at, float &x) { x = p[at]; });
    }
    __device__ inline void store(const Role &r, float *p, int dv, int c0) {
        each(r, dv, c0, [&](int at, float &x) { p[at] = x; });
    }
    // To LDS as terms, for the product with q: [column of the slice][row].  Columns are in the order in which the product's tiles take them: tile
    // t, row 4 a + b is column 16 a + 4 t + b, so that a lane's results are 16 columns side by side.
    __device__ inline void stage(__bf16 (*sl)[kSlice][P::KP]) const {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, place = 16 * (i >> 2) + 4 * ((int)threadIdx.x >> 6) + (i & 3);
#pragma unroll
        for (int t = 0; t < P::TILES; ++t) {
            const float x[4] = {s[t][0], s[t][1], s[t][2], s[t][3]};
            b4 p[P::MADE];
            split(x, p);
#pragma unroll
            for (int n = 0; n < P::MADE; ++n) *reinterpret_cast<b4 *>(&sl[n][place][16 * t + 4 * g]) = p[n];
        }
    }
    // S = carry S + sum_j weight[j] k_j v_j^T over the chunk in LDS.  Both operands have tokens for the places of the sum:
    // transposed reads, in the order 32 s + 16 (e / 4) + 4 (l / 16) + e % 4 for element e.
    __device__ inline void update(const __bf16 (*kl)[kChunk][P::KP], const __bf16 (*vl)[kChunk][P::VP], const float (&weight)[2][2][4]) {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, w = (int)threadIdx.x >> 6, row = 4 * g + (i >> 2), col = 4 * (i & 3);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            float x[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                b4 raw[P::RAW];
#pragma unroll
                for (int p = 0; p < P::RAW; ++p) raw[p] = read_transposed(&vl[p][32 * ks + 16 * h + row][16 * w + col]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y = 0.0f;
#pragma unroll
                    for (int p = P::RAW - 1; p >= 0; --p) y = p == P::RAW - 1 ? (float)raw[p][e] : y + (float)raw[p][e];
                    x[4 * h + e] = y * weight[ks][h][e];
                }
            }
            b8 b[kUpdateTerms];
            split(x, b);
#pragma unroll
            for (int t = 0; t < P::TILES; ++t) {
                b8 a[P::RAW];
#pragma unroll
                for (int p = 0; p < P::RAW; ++p)
                    a[p] = join(read_transposed(&kl[p][32 * ks + row][16 * t + col]), read_transposed(&kl[p][32 * ks + 16 + row][16 * t + col]));
                product<kUpdateOrder>(s[t], a, b);
            }
        }
    }
};

// Decays of a chunk of n tokens on their way into the state, for the tokens that a lane has in State::update.
__device__ inline void update_weights(float (&weight)[2][2][4], const float *pw, int n, int shift, float factor) {
    const int g = ((int)threadIdx.x & 63) >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int left = n - shift - (32 * ks + 16 * h + 4 * g + e);
                weight[ks][h][e] = left >= 0 ? factor * pw[left] : 0.0f;
            }
}

// A sequence's place among the states; -1: none, it begins with zeros and leaves no state.
__device__ inline int state_place(const Args &a, int seq) {
    if (a.slots == nullptr) return seq;
    const int p = a.slots[seq];
    return p >= 0 && p < a.places ? p : -1;
}

__device__ inline const Role &role_of(const Args &a, long &item) {
    int r = 0;
    while (r + 1 < a.roles && item >= a.items[r]) ++r;
    if (r > 0) item -= a.items[r - 1];
    return a.role[r];
}

// Rows of the result.  A workgroup has one segment, one head and a slice of 64 columns and goes through the chunks one after the other; wavefront w has
// queries 16 w to 16 w + 15 of a chunk, and columns 16 w to 16 w + 15 of the state.
template <class T, int DK>
__global__ __launch_bounds__(kThreads) void decay_rows_kernel(const Args a) {
    using P = Shape<T, DK>;
    __shared__ __attribute__((aligned(16))) __bf16 kl[P::RAW][kChunk][P::KP];
    __shared__ __attribute__((aligned(16))) __bf16 vl[P::RAW][kChunk][P::VP];
    __shared__ __attribute__((aligned(16))) __bf16 sl[P::MADE][kSlice][P::KP];
    __shared__ float pw[kChunk + 1];
    long item = xcd_place(a.items[a.roles - 1]);
    if (item >= a.items[a.roles - 1]) return;
    const Role &r = role_of(a, item);
    const int slices = (r.out.width + kSlice - 1) / kSlice;
    const int c0 = (int)(item % slices) * kSlice;
    item /= slices;
    const int sub = (int)(item % r.outs);
    item /= r.outs;
    const int hk = (int)(item % a.Hk);
    const Span sp = a.seq.of_unit(item / a.Hk);
    const long p0 = sp.seg * a.seq.seg;
    const long left = sp.length - p0;
    if (sp.seg < 0 || (left <= 0 && (sp.seg > 0 || r.last == nullptr))) return;
    const int tokens = (int)(left < a.seq.seg ? left : a.seq.seg);
    const int out_head = hk * r.outs + sub;

    const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const float log_decay = a.g[hk];
    if ((int)threadIdx.x <= kChunk) pw[threadIdx.x] = decay_pow(log_decay, (int)threadIdx.x);
    State<T, DK> state;
    state.clear();
    bool live = false;                   // a state that is not zero
    const int place = r.first != nullptr || r.last != nullptr ? state_place(a, sp.seq) : -1;
    if (r.starts != nullptr) {
        state.load(r, r.starts + ((long)sp.unit * a.Hk + hk) * a.state, a.dv, c0);
        live = true;
    } else if (r.first != nullptr && place >= 0) {
        state.load(r, r.first + ((long)place * a.Hk + hk) * a.state, a.dv, c0);
        live = true;
    }
    const bool keep = r.last != nullptr && place >= 0;

    const int chunks = (tokens + kChunk - 1) / kChunk;
    Rows<T, DK> rows;
    Eight<T> q[DK / 32];
    auto in_chunk = [&](int c) { return tokens - c * kChunk < kChunk ? tokens - c * kChunk : kChunk; };
    auto token = [&](int pos) { return r.reverse ? sp.begin + sp.length - 1 - p0 - pos : sp.begin + p0 + pos; };
    auto load_q = [&](int c) {
        const int pos = c * kChunk + 16 * w + i;
        const T *p = static_cast<const T *>(r.q.p) + token(pos) * r.q.stride + (long)out_head * r.q.width;
#pragma unroll
        for (int s = 0; s < DK / 32; ++s) {
            const int col = 32 * s + 8 * g;
            if (pos < tokens && col < r.q.width) q[s].load(p + col);
            else q[s].zero();
        }
    };
    if (chunks > 0) {
        load_q(0);
        rows.load(r, sp.begin, sp.length, p0, in_chunk(0), hk * r.sums, c0);
    }
    __syncthreads();

    float inside[4][4], weight[2][2][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int far = 16 * (w - t) + i - 4 * g - e;
            inside[t][e] = far >= 0 ? r.inside * pw[far] : 0.0f;
        }
    const float into = r.into * pw[16 * w + i + r.shift];
    update_weights(weight, pw, kChunk, r.shift, r.update);

    f4 o[4];
    b8 qt[DK / 32][P::RAW];
    for (int c = 0; c < chunks; ++c) {
        const int n = in_chunk(c);
        const bool add = c + 1 < chunks || keep;
        if (n < kChunk && add) update_weights(weight, pw, n, r.shift, r.update);
        for (int h = 0; h < r.sums; ++h) {
            if (c + h > 0) __syncthreads();
            rows.stage(kl, vl);
            if (h == 0) {
                if (live) state.stage(sl);
#pragma unroll
                for (int s = 0; s < DK / 32; ++s) q[s].terms(qt[s]);
                if (c + 1 < chunks) load_q(c + 1);
            }
            if (h + 1 < r.sums) rows.load(r, sp.begin, sp.length, p0 + (long)c * kChunk, n, hk * r.sums + h + 1, c0);
            else if (c + 1 < chunks) rows.load(r, sp.begin, sp.length, p0 + (long)(c + 1) * kChunk, in_chunk(c + 1), hk * r.sums, c0);
            __syncthreads();
            if (h == 0) {
#pragma unroll
                for (int t = 0; t < 4; ++t) o[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
                if (live) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
#pragma unroll
                        for (int s = 0; s < DK / 32; ++s) {
                            b8 st[P::MADE];
#pragma unroll
                            for (int p = 0; p < P::MADE; ++p) st[p] = *reinterpret_cast<const b8 *>(&sl[p][16 * t + i][32 * s + 8 * g]);
                            product<Terms<T>::ORDER>(o[t], st, qt[s]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][e] *= into;
                    }
                }
            }
            // (k_j q_i) for 32 keys at a time, which are in the registers of the lanes that have them as the right operand of the product with v
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if (2 * ks > w) continue;
                float x[8];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int t = 2 * ks + half;
                    f4 s = f4{0.0f, 0.0f, 0.0f, 0.0f};
                    if (t <= w) {
#pragma unroll
                        for (int d = 0; d < DK / 32; ++d) {
                            b8 kt[P::RAW];
#pragma unroll
                            for (int p = 0; p < P::RAW; ++p) kt[p] = *reinterpret_cast<const b8 *>(&kl[p][16 * t + i][32 * d + 8 * g]);
                            product<Terms<T>::ORDER_RAW>(s, kt, qt[d]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * half + e] = t < w || (t == w && i >= 4 * g + e) ? s[e] * inside[t][e] : 0.0f;
                }
                b8 pt[P::MADE];
                split(x, pt);
                const int row = 32 * ks + 4 * g + (i >> 2);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int col = 16 * (i & 3) + 4 * t;
                    b8 vt[P::RAW];
#pragma unroll
                    for (int p = 0; p < P::RAW; ++p) vt[p] = join(read_transposed(&vl[p][row][col]), read_transposed(&vl[p][row + 16][col]));
                    product<Terms<T>::ORDER>(o[t], vt, pt);
                }
            }
            if (add) {
                if (h == 0 && live) {
                    const float carry = pw[n];
#pragma unroll
                    for (int t = 0; t < P::TILES; ++t) state.s[t] *= carry;
                }
                state.update(kl, vl, weight);
            }
        }
        if (add) live = true;
        const int pos = c * kChunk + 16 * w + i;
        if (pos < tokens) {
            T *p = static_cast<T *>(const_cast<void *>(r.out.p)) + token(pos) * r.out.stride + (long)out_head * r.out.width;
            const int col = c0 + 16 * g;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = o[2 * half + e / 4][e % 4];
                if (col + 8 * half < r.out.width) store_piece<T, 8>(p + col + 8 * half, x);
            }
        }
    }
    if (keep) state.store(r, r.last + ((long)place * a.Hk + hk) * a.state, a.dv, c0);
}

// What each segment adds to the state, from a state of zeros.
template <class T, int DK>
__global__ __launch_bounds__(kThreads) void decay_states_kernel(const Args a) {
    using P = Shape<T, DK>;
    __shared__ __attribute__((aligned(16))) __bf16 kl[P::RAW][kChunk][P::KP];
    __shared__ __attribute__((aligned(16))) __bf16 vl[P::RAW][kChunk][P::VP];
    __shared__ float pw[kChunk + 1];
    long item = xcd_place(a.items[a.roles - 1]);
    if (item >= a.items[a.roles - 1]) return;
    const Role &r = role_of(a, item);
    const int slices = (r.v.width + kSlice - 1) / kSlice;
    const int c0 = (int)(item % slices) * kSlice;
    item /= slices;
    const int hk = (int)(item % a.Hk);
    const Span sp = a.seq.of_unit(item / a.Hk);
    const long p0 = sp.seg * a.seq.seg, left = sp.length - p0;
    // the last segment's sum is for the state behind the sequence only
    if (sp.seg < 0 || left <= 0 || (left <= a.seq.seg && r.last == nullptr)) return;
    const int tokens = (int)(left < a.seq.seg ? left : a.seq.seg), chunks = (tokens + kChunk - 1) / kChunk;
    const float log_decay = a.g[hk];
    if ((int)threadIdx.x <= kChunk) pw[threadIdx.x] = decay_pow(log_decay, (int)threadIdx.x);
    State<T, DK> state;
    state.clear();
    Rows<T, DK> rows;
    auto in_chunk = [&](int c) { return tokens - c * kChunk < kChunk ? tokens - c * kChunk : kChunk; };
    rows.load(r, sp.begin, sp.length, p0, in_chunk(0), hk * r.sums, c0);
    __syncthreads();
    float weight[2][2][4];
    update_weights(weight, pw, kChunk, r.shift, r.update);
    for (int c = 0; c < chunks; ++c) {
        const int n = in_chunk(c);
        if (n < kChunk) update_weights(weight, pw, n, r.shift, r.update);
        for (int h = 0; h < r.sums; ++h) {
            if (c + h > 0) __syncthreads();
            rows.stage(kl, vl);
            if (h + 1 < r.sums) rows.load(r, sp.begin, sp.length, p0 + (long)c * kChunk, n, hk * r.sums + h + 1, c0);
            else if (c + 1 < chunks) rows.load(r, sp.begin, sp.length, p0 + (long)(c + 1) * kChunk, in_chunk(c + 1), hk * r.sums, c0);
            __syncthreads();
            if (h == 0) {
                const float carry = pw[n];
#pragma unroll
                for (int t = 0; t < P::TILES; ++t) state.s[t] *= carry;
            }
            state.update(kl, vl, weight);
        }
    }
    state.store(r, r.sums_out + ((long)sp.unit * a.Hk + hk) * a.state, a.dv, c0);
}

// From the segments' sums to the states before them, in their place, and to the state behind the sequence.  A thread has 4 elements.
__global__ __launch_bounds__(kThreads) void decay_scan_kernel(const Args a) {
    const Role &r = a.role[blockIdx.z];
    const int hk = (int)(blockIdx.y % (unsigned)a.Hk), b = (int)(blockIdx.y / (unsigned)a.Hk);
    const long at = ((long)blockIdx.x * kThreads + threadIdx.x) * 4;
    if (at >= a.state) return;
    const Span sp = a.seq.of_sequence(b);
    const int place = r.first != nullptr || r.last != nullptr ? state_place(a, b) : -1;
    const int segs = (int)((sp.length + a.seq.seg - 1) / a.seq.seg);
    const float log_decay = a.g[hk];
    f4 x = f4{0.0f, 0.0f, 0.0f, 0.0f};
    if (r.first != nullptr && place >= 0) x = *reinterpret_cast<const f4 *>(r.first + ((long)place * a.Hk + hk) * a.state + at);
    float *p = r.sums_out + ((long)sp.unit * a.Hk + hk) * a.state + at;
    const long next = a.Hk * a.state;
    const float whole = decay_pow(log_decay, (int)a.seq.seg);
    for (int s = 0; s < segs; ++s, p += next) {
        const bool end = s + 1 == segs;
        f4 add = f4{0.0f, 0.0f, 0.0f, 0.0f};
        if (!end || r.last != nullptr) add = *reinterpret_cast<const f4 *>(p);
        *reinterpret_cast<f4 *>(p) = x;
        x = x * (end ? decay_pow(log_decay, (int)(sp.length - (long)s * a.seq.seg)) : whole) + add;
    }
    if (r.last != nullptr && place >= 0) *reinterpret_cast<f4 *>(r.last + ((long)place * a.Hk + hk) * a.state + at) = x;
}

// ------------------------------------------------------------------------------------------- plan --

struct Plan {
    long seg = 0;            // 0: one pass
    int per_sequence = 1;
};

// Segments where sequences and heads alone leave CUs without work, or where one long sequence among short ones would go on alone.
// `shared_states`: heads that share a state would each make the one behind the sequence, and one might write it before another has read the
// one before: then the states are made apart from the rows.
Plan make_plan(long T, int B, int Hk, long outs, bool ragged, bool shared_states) {
    Plan p;
    if (T == 0 || B == 0) return p;
    const long mean = (T + B - 1) / B, groups = (long)B * Hk * outs;
    constexpr long kWanted = 1024, kLeast = 256, kRagged = 2048;
    long seg = 0;
    if (groups < kWanted && mean > kLeast) {
        const long parts = (kWanted + groups - 1) / groups;
        seg = ((mean + parts - 1) / parts + kChunk - 1) / kChunk * kChunk;
        if (seg < kLeast) seg = kLeast;
    }
    if (ragged && T > kRagged && (seg == 0 || seg > kRagged)) seg = kRagged;
    if (seg == 0 && shared_states) seg = (T + kChunk - 1) / kChunk * kChunk;
    if (!ragged && !shared_states && seg >= T / B) seg = 0;
    p.seg = seg;
    if (seg > 0) p.per_sequence = (int)((T / B + seg - 1) / seg);
    return p;
}

Sequences sequences(const int32_t *offsets, long T, int B, const Plan &p) {
    if (p.seg > 0) return Sequences{offsets, T, B, p.seg, p.per_sequence};
    // one segment to a sequence: unit b is sequence b
    return Sequences{offsets, T, B, 1L << 31, 1};
}

size_t plan_bytes(const Plan &p, long T, int B, bool ragged, int Hk, int d, int dv) {
    if (p.seg == 0) return 0;
    const long units = ragged ? T / p.seg + B : (long)p.per_sequence * B;
    return (size_t)units * Hk * d * dv * sizeof(float);
}

constexpr int slices_of(int width) { return (width + kSlice - 1) / kSlice; }

template <class T, class F>
int by_width(int width, F f) {
    if (width <= 32) return f(std::integral_constant<int, 32>());
    if (width <= 64) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, 128>());
}

// The rows of all roles in one launch; the states' sums and their scan before it where there are segments.
int launch(const char *what, int type, Args a, const Plan &p, int states, hipStream_t st) {
    const long units = a.seq.units();
    if (units == 0) return SA_OK;
    int widest = 0;
    for (int r = 0; r < a.roles; ++r) widest = a.role[r].k.width > widest ? a.role[r].k.width : widest;
    long total = 0;
    for (int r = 0; r < a.roles; ++r) a.items[r] = total += units * a.Hk * a.role[r].outs * slices_of(a.role[r].out.width);
    SA_REQUIRE(total < (1L << 31) - 8, SA_ERR_UNSUPPORTED, "%s: too many heads and tokens for one launch", what);
    if (p.seg > 0) {
        Args s = a;
        s.roles = states;
        long sums = 0;
        for (int r = 0; r < states; ++r) s.items[r] = sums += units * a.Hk * slices_of(s.role[r].v.width);
        const int rc = by_type(type, [&](auto t) {
            return by_width<decltype(t)>(widest, [&](auto k) {
                decay_states_kernel<decltype(t), decltype(k)::value><<<dim3((unsigned)xcd_blocks(sums)), dim3(kThreads), 0, st>>>(s);
                return check_launch(what);
            });
        });
        if (rc != SA_OK) return rc;
        decay_scan_kernel<<<dim3((unsigned)((a.state / 4 + kThreads - 1) / kThreads), (unsigned)(a.Hk * a.seq.B), (unsigned)states), dim3(kThreads), 0, st>>>(s);
        if (const int rc2 = check_launch(what); rc2 != SA_OK) return rc2;
        for (int r = 0; r < a.roles; ++r) a.role[r].first = nullptr, a.role[r].last = nullptr;
    }
    return by_type(type, [&](auto t) {
        return by_width<decltype(t)>(widest, [&](auto k) {
            decay_rows_kernel<decltype(t), decltype(k)::value><<<dim3((unsigned)xcd_blocks(total)), dim3(kThreads), 0, st>>>(a);
            return check_launch(what);
        });
    });
}

int check_sequences(const char *what, int type, long T, int B, bool ragged, int H, int Hk, int d, int dv) {
    SA_TRY(check_heads(what, type, T, H, Hk, d, dv));
    SA_REQUIRE(B >= 0, SA_ERR_INVALID, "%s: B < 0", what);
    SA_REQUIRE(ragged || (B > 0 ? T % B == 0 : T == 0), SA_ERR_SHAPE, "%s: %ld tokens are no %d sequences of the same length", what, T, B);
    SA_REQUIRE((long)B * Hk <= 65535, SA_ERR_UNSUPPORTED, "%s: up to 65535 states a call (got %d x %d)", what, B, Hk);
    return SA_OK;
}

}  // namespace

extern "C" size_t sa_decay_attention_workspace_bytes(long T, int B, int H, int Hk, int d, int dv, int ragged) {
    if (check_sequences("", SA_F32, T, B, ragged != 0, H, Hk, d, dv) != SA_OK) return 0;
    const long outs = (long)(H / Hk) * slices_of(dv);
    const size_t a = plan_bytes(make_plan(T, B, Hk, outs, ragged != 0, false), T, B, ragged != 0, Hk, d, dv);
    const size_t b = plan_bytes(make_plan(T, B, Hk, outs, ragged != 0, H != Hk), T, B, ragged != 0, Hk, d, dv);
    return a > b ? a : b;
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
    SA_REQUIRE(sa::aligned16(log_decay) && sa::aligned16(state_in_or_null) && sa::aligned16(state_out_or_null) && sa::aligned16(workspace) &&
                   sa::aligned4(offsets_or_null) && sa::aligned4(slots_or_null),
               SA_ERR_ALIGN, "%s: pointers must be 16-byte aligned", what);
    if (B == 0 || (T == 0 && state_out_or_null == nullptr)) return SA_OK;
    const Plan p = make_plan(T, B, Hk, (long)(H / Hk) * slices_of(dv), ragged, H != Hk && state_out_or_null != nullptr);
    const size_t need = plan_bytes(p, T, B, ragged, Hk, d, dv);
    SA_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), SA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what,
               need, workspace_bytes);
    Args a{};
    a.roles = 1;
    a.seq = sequences(offsets_or_null, T, B, p);
    a.g = log_decay, a.Hk = Hk, a.dv = dv, a.state = (long)d * dv, a.slots = slots_or_null, a.places = n_slots;
    Role &r = a.role[0];
    r.q = {q, q_stride, d}, r.k = {k, k_stride, d}, r.v = {v, v_stride, dv}, r.out = {out, out_stride, dv};
    r.outs = H / Hk, r.sums = 1, r.shift = 1;
    r.inside = scale, r.into = scale, r.update = 1.0f;
    r.first = state_in_or_null, r.last = state_out_or_null;
    if (p.seg > 0) r.starts = r.sums_out = static_cast<float *>(workspace);
    return launch(what, type, a, p, 1, sa::as_stream(stream));
}

extern "C" size_t sa_decay_attention_backward_workspace_bytes(long T, int B, int H, int Hk, int d, int dv, int ragged) {
    if (check_sequences("", SA_F32, T, B, ragged != 0, H, Hk, d, dv) != SA_OK) return 0;
    return 2 * plan_bytes(make_plan(T, B, Hk, (long)(H / Hk + 1) * slices_of(d) + slices_of(dv), ragged != 0, false), T, B, ragged != 0, Hk, d, dv);
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
    SA_REQUIRE(sa::aligned16(log_decay) && sa::aligned16(state_in_or_null) && sa::aligned16(dstate_out_or_null) && sa::aligned16(dstate_in_or_null) &&
                   sa::aligned16(workspace) && sa::aligned4(offsets_or_null),
               SA_ERR_ALIGN, "%s: pointers must be 16-byte aligned", what);
    if (B == 0 || (T == 0 && dstate_in_or_null == nullptr)) return SA_OK;
    const Plan p = make_plan(T, B, Hk, (long)(H / Hk + 1) * slices_of(d) + slices_of(dv), ragged, false);
    const size_t each = plan_bytes(p, T, B, ragged, Hk, d, dv);
    SA_REQUIRE(each == 0 || (workspace != nullptr && workspace_bytes >= 2 * each), SA_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given",
               what, 2 * each, workspace_bytes);
    Args a{};
    a.roles = 3;
    a.seq = sequences(offsets_or_null, T, B, p);
    a.g = log_decay, a.Hk = Hk, a.dv = dv, a.state = (long)d * dv;
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
    if (p.seg > 0) {
        float *ws = static_cast<float *>(workspace);
        gv.starts = gv.sums_out = ws;
        gk.starts = ws;
        gq.starts = gq.sums_out = ws + each / sizeof(float);
    }
    return launch(what, type, a, p, 2, sa::as_stream(stream));
}
