// Linear attention with a decay for each head, one token of each sequence:
//   S = l S + k v^T,  o = scale q^T S,  l = exp(g)
// A workgroup has up to 64 columns of one state in registers, all loads of which are under way at once, and does for them all heads that share it: a state
// is read once and written once.  What bounds it: memory, 64 x 16 states of 128 x 128 30 us (135 MB, 4.5 TB/s), 333 x 4 of 80 x 40 9.3 (37 MB); a
// single sequence, 3 states of 64 x 64, the host: 8.1 us, 2.8 of them on the device.
#include "common.h"
#include "decay_attention.h"

namespace {

using namespace sa;
using namespace sa::decay;

struct StepArgs {
    HeadRows q, k, v, out;
    const float *g;
    int Hk, outs, blocks;                // blocks: of columns
    float scale;
    const float *in;
    float *to;
    const int32_t *slots;
    int places;
};

constexpr int kStepThreads = 256;

// Lanes of COLS threads have 4 columns each; NR rows to a thread, one behind the other, so that its part of q and k is one load.
template <class T, int COLS, int NR>
__global__ __launch_bounds__(kStepThreads) void decay_step_kernel(const StepArgs a) {
    constexpr int kHeads = 4;            // heads whose results wait in LDS at once
    __shared__ float red[4][kHeads][4 * COLS];
    const int tid = (int)threadIdx.x, lc = tid % COLS, row = tid / COLS * NR, lane = tid & 63, w = tid >> 6;
    int item = (int)blockIdx.x;
    const int col = (item % a.blocks) * 4 * COLS + 4 * lc;
    item /= a.blocks;
    const int hk = item % a.Hk;
    const long b = item / a.Hk;
    const int d = a.k.width, dv = a.v.width;
    const bool mine = row < d && col < dv;
    const int p = a.slots != nullptr ? a.slots[b] : (int)b;
    const bool there = a.slots == nullptr || (p >= 0 && p < a.places);
    const long at = ((long)p * a.Hk + hk) * d * dv + (long)row * dv + col;
    f4 s[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) s[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    if (mine && there) {
#pragma unroll
        for (int i = 0; i < NR; ++i) s[i] = *reinterpret_cast<const f4 *>(a.in + at + (long)i * dv);
    }
    if (mine) {
        Piece<T, NR> k;
        Piece<T, 4> v;
        k.load(static_cast<const T *>(a.k.p) + b * a.k.stride + (long)hk * d + row);
        v.load(static_cast<const T *>(a.v.p) + b * a.v.stride + (long)hk * dv + col);
        const float l = expf(a.g[hk]);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = __builtin_fmaf(l, s[i][j], k[i] * v[j]);
        }
        if (there) {
#pragma unroll
            for (int i = 0; i < NR; ++i) *reinterpret_cast<f4 *>(a.to + at + (long)i * dv) = s[i];
        }
    }
    for (int h0 = 0; h0 < a.outs; h0 += kHeads) {
        if (h0 > 0) __syncthreads();
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            if (h0 + h >= a.outs) break;
            float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (mine) {
                Piece<T, NR> q;
                q.load(static_cast<const T *>(a.q.p) + b * a.q.stride + (long)(hk * a.outs + h0 + h) * d + row);
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(q[i], s[i][j], o[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int far = COLS; far < 64; far *= 2) o[j] += __shfl_xor(o[j], far);
            }
            if (lane < COLS) *reinterpret_cast<f4 *>(&red[w][h][4 * lane]) = f4{o[0], o[1], o[2], o[3]};
        }
        __syncthreads();
        const int h = tid / (4 * COLS), c = tid % (4 * COLS), out_col = col - 4 * lc + c;
        if (h < kHeads && h0 + h < a.outs && out_col < dv) {
            const float o = (red[0][h][c] + red[1][h][c]) + (red[2][h][c] + red[3][h][c]);
            T *to = static_cast<T *>(const_cast<void *>(a.out.p));
            to[b * a.out.stride + (long)(hk * a.outs + h0 + h) * dv + out_col] = rounded<T>(o * a.scale);
        }
    }
}

template <class T>
int launch_step(const StepArgs &a, long B, hipStream_t st) {
    const dim3 grid((unsigned)(B * a.Hk * a.blocks));
    const int d = a.k.width;
    if (a.v.width <= 32) {
        decay_step_kernel<T, 8, 4><<<grid, dim3(kStepThreads), 0, st>>>(a);
    } else if (d <= 64) {
        decay_step_kernel<T, 16, 4><<<grid, dim3(kStepThreads), 0, st>>>(a);
    } else {
        decay_step_kernel<T, 16, 8><<<grid, dim3(kStepThreads), 0, st>>>(a);
    }
    return check_launch("sa_decay_attention_step");
}

}  // namespace

extern "C" int sa_decay_attention_step(const void *q, long q_stride, const void *k, long k_stride, const void *v, long v_stride, int type,
                                       const float *log_decay, long B, int H, int Hk, int d, int dv, float scale, const float *state_in,
                                       float *state_out, const int32_t *slots_or_null, int n_slots, void *out, long out_stride, void *stream) {
    const char *what = "sa_decay_attention_step";
    sa::clear_error();
    SA_TRY(check_heads(what, type, B, H, Hk, d, dv));
    SA_REQUIRE(slots_or_null == nullptr || n_slots >= 0, SA_ERR_INVALID, "%s: n_slots < 0", what);
    if (B == 0) return SA_OK;
    SA_TRY(check_rows(what, "q", q, q_stride, H, d, type));
    SA_TRY(check_rows(what, "k", k, k_stride, Hk, d, type));
    SA_TRY(check_rows(what, "v", v, v_stride, Hk, dv, type));
    SA_TRY(check_rows(what, "out", out, out_stride, H, dv, type));
    SA_REQUIRE(log_decay && state_in && state_out, SA_ERR_INVALID, "%s: NULL buffer", what);
    SA_REQUIRE(out != q && out != k && out != v, SA_ERR_INVALID, "%s: out must not be an input", what);
    SA_REQUIRE(sa::aligned4(log_decay) && sa::aligned16(state_in) && sa::aligned16(state_out) && sa::aligned4(slots_or_null), SA_ERR_ALIGN,
               "%s: pointers must be 16-byte aligned", what);
    StepArgs a{{q, q_stride, d}, {k, k_stride, d}, {v, v_stride, dv}, {out, out_stride, dv}, log_decay, Hk, H / Hk, dv > 64 ? 2 : 1, scale,
               state_in, state_out, slots_or_null, n_slots};
    // (a launch has less than 2^32 threads)
    SA_REQUIRE(B * Hk * a.blocks * kStepThreads < (1L << 32), SA_ERR_UNSUPPORTED, "%s: too many states for one launch", what);
    return by_type(type, [&](auto t) { return launch_step<decltype(t)>(a, B, sa::as_stream(stream)); });
}
