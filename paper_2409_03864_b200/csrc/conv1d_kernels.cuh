// Short causal depthwise convolution along a sequence, channels last.
//
//   pre[t, d] = bias[d] + sum_{k < W} weight[d, k] * e[t + k, d],   y = silu(pre) or pre
//
// where e is the sequence with the W - 1 rows of its state (zeros without one) in front: e[j] = state[j] for j < W - 1,
// x[j - (W - 1)] after.  The padded sequence is never built.
#pragma once
#include "seq_common.cuh"

namespace tdx {

struct Conv1dParams {
    long long batch, max_len, rows, channels;
    int width, silu;
    const void* x; long long ld_x;
    const float* weight;
    const float* bias;
    void* y; long long ld_y;
    const int* offsets;
    const void* state_in;
    void* state_out;
    long long state_stride;
    const int* slots;
    long long n_slots;
    const void* dy; long long ld_dy;
    void* dx; long long ld_dx;
    float* dweight;
    float* dbias;
    const void* dstate_out;
    void* dstate_in;
    float* partial;          // [pieces][channels][width + 1]
    long long dense;         // pieces per sequence of a dense batch
    int channel_tiles;
    int weight_aligned;      // to 16 bytes
    int* status;
};

constexpr int kConvRows = 32;        // rows of a run in the forward kernel
constexpr int kConvBwdRows = 64;     // rows of a run in the backward kernel
constexpr int kConvRuns = 4;         // runs (warps) of a block, one after the other in time
constexpr int kConvChunk = 16;       // rows that a thread loads at a time, forward
constexpr int kConvBwdChunk = 4;     // and backward (of x and dy)

template <typename T, int VEC>
__device__ __forceinline__ void conv_zero(float (&f)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = 0.0f;
}
// A row of a state: an ordinary load, because state_out may be the same memory.
template <typename T, int VEC>
__device__ __forceinline__ void conv_state_row(const T* p, float (&f)[VEC]) {
    SeqVec<T, VEC> r;
    r.bits = *reinterpret_cast<const typename SeqVec<T, VEC>::bits_t*>(p);
    seq_unpack<T, VEC>(r, f);
}
// e[j] of a sequence of len rows; zero in front of the state, behind the sequence, and where there is no state
template <typename T, int VEC>
__device__ __forceinline__ void conv_ext_row(const T* x, long long ld, const T* state, long long channels, int w1, int j, int len,
                                             float (&f)[VEC]) {
    if (j < w1) {
        if (j >= 0 && state != nullptr) conv_state_row<T, VEC>(state + j * channels, f);
        else conv_zero<T, VEC>(f);
    } else if (j - w1 < len) {
        seq_unpack<T, VEC>(seq_load<T, VEC>(x + (j - w1) * ld), f);
    } else {
        conv_zero<T, VEC>(f);
    }
}

// KW taps are kept in registers; a narrower filter (only with KW = 8) uses the last `width` of them, and the taps in front
// are skipped rather than multiplied by zero, so that an infinity outside the filter cannot reach the sum.
template <int KW>
__device__ __forceinline__ bool conv_tap(int k, int width) { return KW < 8 || k >= KW - width; }

template <int KW, int VEC>
__device__ __forceinline__ void conv_load_weights(const Conv1dParams& p, long long c, float (&w)[KW][VEC], float (&bias)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float* wp = p.weight + (c + i) * p.width - (KW - p.width);
        if (KW == 4 && p.weight_aligned) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(wp));
            w[0][i] = v.x; w[1][i] = v.y; w[KW - 2][i] = v.z; w[KW - 1][i] = v.w;
        } else {
#pragma unroll
            for (int k = 0; k < KW; ++k) w[k][i] = conv_tap<KW>(k, p.width) ? __ldg(wp + k) : 0.0f;
        }
        bias[i] = p.bias ? __ldg(p.bias + c + i) : 0.0f;
    }
}

// Forward.  A warp takes 32 * VEC neighbouring channels of a run of kConvRows rows; a thread keeps the last KW - 1 rows of
// its VEC channels in registers, so each row is read once (plus KW - 1 rows in front of a run).
// 22.0 us for 4470 packed rows of 4096 channels in bf16 (3.3 TB/s, half of the copy rate; the whole call): the loads of a chunk wait for
// memory at five blocks per SM, and SiLU takes two special functions a value.  The next chunk's rows in registers ahead of time cost more
// in moves and checks than they hid (32 us against 24.9 in the form of that time).
// The thread that reads the state (run 0) is also the one that writes the state after the sequence, so state_out may be
// state_in.
template <typename T, int VEC, int KW>
__global__ void __launch_bounds__(128, KW <= 4 ? 5 : 2) conv1d_fwd_kernel(const __grid_constant__ Conv1dParams p) {
    seq_grid_wait();
    const long long bid = blockIdx.x;
    const int ct = static_cast<int>(bid % p.channel_tiles);
    const long long number = bid / p.channel_tiles;
    const SeqPiece at = seq_piece(p.offsets, p.batch, p.dense, kConvRuns * kConvRows, number);
    if (ct == 0) seq_check(p.offsets, number, p.batch, p.max_len, p.rows, p.status);
    const long long b = at.b;
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const long long c = (static_cast<long long>(ct) * 32 + lane) * VEC;
    if (c >= p.channels) return;
    const SeqRange seq = seq_range(p.offsets, b, p.max_len, p.rows, p.status);
    const int tile = min(at.index, seq.len / (kConvRuns * kConvRows) + 1);
    const int t0 = (tile * kConvRuns + run) * kConvRows;
    const bool first = tile == 0 && run == 0;
    if (t0 >= seq.len && !first) return;
    const long long slot = p.state_in || p.state_out ? state_slot(p.slots, b, p.n_slots, p.status) : -1;
    const int w1 = p.width - 1;
    const T* x = static_cast<const T*>(p.x) + seq.first * p.ld_x + c;
    const T* state = p.state_in && slot >= 0 ? static_cast<const T*>(p.state_in) + slot * p.state_stride + c : nullptr;
    float w[KW][VEC], bias[VEC];
    conv_load_weights<KW, VEC>(p, c, w, bias);
    // the window: e rows t0 .. t0 + KW - 2 in terms of a KW-wide filter
    float win[KW - 1][VEC];
#pragma unroll
    for (int k = 0; k < KW - 1; ++k) conv_ext_row<T, VEC>(x, p.ld_x, state, p.channels, w1, t0 + k - (KW - p.width), seq.len, win[k]);
    const int rows = min(kConvRows, seq.len - t0);
    T* y = static_cast<T*>(p.y) + (seq.first + t0) * p.ld_y + c;
    const T* xr = x + t0 * p.ld_x;
    // A chunk of rows: all its loads, then its sums, so that the loads are in flight together.  Whole chunks go without checks.
    auto chunk = [&](auto checked, auto silu, int r0) {
        SeqVec<T, VEC> raw[kConvChunk];
#pragma unroll
        for (int r = 0; r < kConvChunk; ++r)
            if (!decltype(checked)::value || r0 + r < rows) raw[r] = seq_load<T, VEC>(xr + (r0 + r) * p.ld_x);
#pragma unroll
        for (int r = 0; r < kConvChunk; ++r) {
            if (!decltype(checked)::value || r0 + r < rows) {
                float now[VEC], out[VEC];
                seq_unpack<T, VEC>(raw[r], now);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    float acc = bias[i];
#pragma unroll
                    for (int k = 0; k < KW - 1; ++k)
                        if (conv_tap<KW>(k, p.width)) acc = fmaf(w[k][i], win[k][i], acc);
                    acc = fmaf(w[KW - 1][i], now[i], acc);
                    out[i] = decltype(silu)::value ? acc * sigmoid_f<T>(acc) : acc;
#pragma unroll
                    for (int k = 0; k + 1 < KW - 1; ++k) win[k][i] = win[k + 1][i];
                    win[KW - 2][i] = now[i];
                }
                seq_store<T, VEC>(y + (r0 + r) * p.ld_y, out);
            }
        }
    };
    auto run_rows = [&](auto silu) {
        int r0 = 0;
        for (; r0 + kConvChunk <= rows; r0 += kConvChunk) chunk(SeqNo(), silu, r0);
        if (r0 < rows) chunk(SeqYes(), silu, r0);
    };
    if (p.silu) run_rows(SeqYes());
    else run_rows(SeqNo());
    if (first && p.state_out && slot >= 0) {
        // the state after the sequence is e[len .. len + W - 2]; ascending, so that in place a row is read before it is written
        T* out = static_cast<T*>(p.state_out) + slot * p.state_stride + c;
        for (int j = 0; j < w1; ++j) {
            float f[VEC];
            conv_ext_row<T, VEC>(x, p.ld_x, state, p.channels, w1, seq.len + j, seq.len, f);
            seq_store<T, VEC>(out + j * p.channels, f);
        }
    }
}

// Backward.  With g[t] = dy[t] * act'(pre[t]):
//   de[j] = sum_k weight[k] g[j - k]  (+ dstate_out behind the sequence),  dweight[k] = sum_t g[t] e[t + k],  dbias = sum_t g[t].
// One pass over x and dy: a thread walks a run of rows with the last KW rows of x and of g in registers; row t of g completes
// de of the row KW - 1 before it.  A run re-reads KW - 1 rows on either side (from L2).  dweight and dbias are summed over the
// run in registers, over a block's runs in shared memory and over blocks by conv1d_dweight_kernel, always in the same order.
template <typename T, int VEC, int KW>
__global__ void __launch_bounds__(128, KW <= 4 ? 4 : 2) conv1d_bwd_kernel(const __grid_constant__ Conv1dParams p) {
    constexpr int kSums = VEC * (KW + 1);
    __shared__ float sums[kConvRuns][32][kSums + 1];
    seq_grid_wait();
    const long long bid = blockIdx.x;
    const int ct = static_cast<int>(bid % p.channel_tiles);
    const long long number = bid / p.channel_tiles;
    const SeqPiece at = seq_piece(p.offsets, p.batch, p.dense, kConvRuns * kConvBwdRows, number);
    if (ct == 0) seq_check(p.offsets, number, p.batch, p.max_len, p.rows, p.status);
    const long long b = at.b;
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const long long c = (static_cast<long long>(ct) * 32 + lane) * VEC;
    const bool live = c < p.channels;
    const SeqRange seq = seq_range(p.offsets, b, p.max_len, p.rows, p.status);
    const int tile = min(at.index, seq.len / (kConvRuns * kConvBwdRows) + 1);
    const int t0 = (tile * kConvRuns + run) * kConvBwdRows;
    const bool first = tile == 0 && run == 0;
    float dw[KW][VEC], db[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        db[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KW; ++k) dw[k][i] = 0.0f;
    }
    if (live && (t0 < seq.len || first)) {
        const long long slot = p.state_in || p.dstate_in || p.dstate_out ? state_slot(p.slots, b, p.n_slots, p.status) : -1;
        const int w1 = p.width - 1, len = seq.len;
        const T* x = static_cast<const T*>(p.x) + seq.first * p.ld_x + c;
        const T* dy = static_cast<const T*>(p.dy) + seq.first * p.ld_dy + c;
        T* dx = static_cast<T*>(p.dx) + seq.first * p.ld_dx + c;
        const T* state = p.state_in && slot >= 0 ? static_cast<const T*>(p.state_in) + slot * p.state_stride + c : nullptr;
        const T* dso = p.dstate_out && slot >= 0 ? static_cast<const T*>(p.dstate_out) + slot * p.state_stride + c : nullptr;
        T* dsi = p.dstate_in && slot >= 0 ? static_cast<T*>(p.dstate_in) + slot * p.state_stride + c : nullptr;
        float w[KW][VEC], bias[VEC], win[KW - 1][VEC], gw[KW][VEC];   // gw[m] = g[t - m]
        conv_load_weights<KW, VEC>(p, c, w, bias);
#pragma unroll
        for (int k = 0; k < KW - 1; ++k) conv_ext_row<T, VEC>(x, p.ld_x, state, p.channels, w1, t0 + k - (KW - p.width), len, win[k]);
#pragma unroll
        for (int m = 0; m < KW; ++m) conv_zero<T, VEC>(gw[m]);
        const int own_rows = min(kConvBwdRows, max(len - t0, 0)), stop = own_rows + KW - 1;   // the last row of dx of this run is emitted at stop - 1
        const T* xr = x + t0 * p.ld_x;
        const T* dyr = dy + t0 * p.ld_dy;
        T* dxr = dx + (t0 - (KW - 1)) * p.ld_dx;               // the row of x that is complete when row 0 of the run is reached
        auto chunk = [&](auto checked, auto silu, int i0) {
            constexpr bool kChecked = decltype(checked)::value;
            SeqVec<T, VEC> rx[kConvBwdChunk], rg[kConvBwdChunk];
#pragma unroll
            for (int r = 0; r < kConvBwdChunk; ++r) {
                if (!kChecked || (i0 + r < stop && t0 + i0 + r < len)) {
                    rx[r] = seq_load<T, VEC>(xr + (i0 + r) * p.ld_x);
                    rg[r] = seq_load<T, VEC>(dyr + (i0 + r) * p.ld_dy);
                }
            }
#pragma unroll
            for (int r = 0; r < kConvBwdChunk; ++r) {
                const int i = i0 + r, t = t0 + i;
                if (!kChecked || i < stop) {
                    float now[VEC], g[VEC], de[VEC];
                    const bool there = !kChecked || t < len, own = !kChecked || (i < kConvBwdRows && there);
                    if (there) {
                        seq_unpack<T, VEC>(rx[r], now);
                        seq_unpack<T, VEC>(rg[r], g);
                    } else {
                        conv_zero<T, VEC>(now);
                        conv_zero<T, VEC>(g);
                    }
                    const int j = t - (KW - 1);                          // the row of x completed by g[t]
                    const bool emit_x = !kChecked || (i >= KW - 1 && j < len), emit_s = kChecked && first && dsi != nullptr && j < 0 && j + w1 >= 0;
                    const bool from_state = kChecked && dso != nullptr && j + w1 >= len && (emit_x || emit_s);
                    if (from_state) conv_state_row<T, VEC>(dso + (j + w1 - len) * p.channels, de);
                    else conv_zero<T, VEC>(de);
#pragma unroll
                    for (int v = 0; v < VEC; ++v) {
                        if (there && decltype(silu)::value) {
                            float pre = bias[v];
#pragma unroll
                            for (int k = 0; k < KW - 1; ++k)
                                if (conv_tap<KW>(k, p.width)) pre = fmaf(w[k][v], win[k][v], pre);
                            pre = fmaf(w[KW - 1][v], now[v], pre);
                            const float s = sigmoid_f<T>(pre);
                            g[v] *= s * fmaf(pre, 1.0f - s, 1.0f);       // silu'(pre)
                        }
                        if (own) {
#pragma unroll
                            for (int k = 0; k < KW - 1; ++k)
                                if (conv_tap<KW>(k, p.width)) dw[k][v] = fmaf(g[v], win[k][v], dw[k][v]);
                            dw[KW - 1][v] = fmaf(g[v], now[v], dw[KW - 1][v]);
                            db[v] += g[v];
                        }
#pragma unroll
                        for (int k = 0; k + 1 < KW - 1; ++k) win[k][v] = win[k + 1][v];
                        win[KW - 2][v] = now[v];
#pragma unroll
                        for (int m = KW - 1; m > 0; --m) gw[m][v] = gw[m - 1][v];
                        gw[0][v] = g[v];
                        // lag l of row j: g[j + l] = gw[KW - 1 - l] and the tap KW - 1 - l
#pragma unroll
                        for (int k = 0; k < KW; ++k)
                            if (conv_tap<KW>(k, p.width)) de[v] = fmaf(w[k][v], gw[k][v], de[v]);
                    }
                    if (emit_x) seq_store<T, VEC>(dxr + i * p.ld_dx, de);
                    if (emit_s) seq_store<T, VEC>(dsi + (j + w1) * p.channels, de);
                }
            }
        };
        auto run_rows = [&](auto silu) {
            int i0 = 0;
            for (; i0 < KW - 1; i0 += kConvBwdChunk) chunk(SeqYes(), silu, i0);      // no row is complete before row KW - 1
            for (; i0 + kConvBwdChunk <= own_rows; i0 += kConvBwdChunk) chunk(SeqNo(), silu, i0);
            for (; i0 < stop; i0 += kConvBwdChunk) chunk(SeqYes(), silu, i0);
        };
        if (p.silu) run_rows(SeqYes());
        else run_rows(SeqNo());
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
#pragma unroll
        for (int k = 0; k < KW; ++k) sums[run][lane][v * (KW + 1) + k] = dw[k][v];
        sums[run][lane][v * (KW + 1) + KW] = db[v];
    }
    __syncthreads();
    const int per = p.width + 1, skip = KW - p.width;
    const long long base = number * p.channels;
    for (int e = threadIdx.x; e < 32 * VEC * per; e += 128) {
        const int ch = e / per, k = e - ch * per;
        const long long cc = static_cast<long long>(ct) * 32 * VEC + ch;
        if (cc >= p.channels) break;
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kConvRuns; ++r) s += sums[r][ch / VEC][(ch % VEC) * (KW + 1) + k + skip];
        p.partial[(base + cc) * per + k] = s;
    }
}

// dweight and dbias: the sum of `count` blocks' partial sums, eight interleaved partial orders joined in a fixed order.
__global__ void __launch_bounds__(256) conv1d_dweight_kernel(long long elems, long long count, int width, const float* __restrict__ partial,
                                                             float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float sums[8][33];
    seq_grid_wait();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const long long e = blockIdx.x * 32LL + lane;
    float s = 0.0f;
    if (e < elems)
        for (long long i = part; i < count; i += 8) s += __ldg(partial + i * elems + e);
    sums[part][lane] = s;
    __syncthreads();
    if (part == 0 && e < elems) {
#pragma unroll
        for (int q = 1; q < 8; ++q) s += sums[q][lane];
        const long long c = e / (width + 1);
        const int k = static_cast<int>(e - c * (width + 1));
        if (k < width) {
            if (dweight) dweight[c * width + k] = s;
        } else if (dbias) {
            dbias[c] = s;
        }
    }
}

// One new row for each of a batch of sequences: y from the state's W - 1 rows and x, and the state moved on by one row.
// A thread holds VEC channels of one batch row, so state_out may be state_in.  A batch row without a slot is padding: y = 0.
template <typename T, int VEC, int KW>
__global__ void __launch_bounds__(128) conv1d_step_kernel(const __grid_constant__ Conv1dParams p) {
    seq_launch_dependents();
    seq_grid_wait();
    const long long b = blockIdx.x / p.channel_tiles;
    const long long c = ((blockIdx.x % p.channel_tiles) * 128LL + threadIdx.x) * VEC;
    if (c >= p.channels) return;
    const long long slot = state_slot(p.slots, b, p.n_slots, p.status);
    float out[VEC];
    conv_zero<T, VEC>(out);
    if (slot >= 0) {
        const T* state = static_cast<const T*>(p.state_in) + slot * p.state_stride + c;
        T* next = static_cast<T*>(p.state_out) + slot * p.state_stride + c;
        const int w1 = p.width - 1;
        float w[KW][VEC], bias[VEC], win[KW][VEC];
#pragma unroll
        for (int k = 0; k < KW - 1; ++k)
            if (conv_tap<KW>(k, p.width)) conv_state_row<T, VEC>(state + (k - (KW - p.width)) * p.channels, win[k]);
        seq_unpack<T, VEC>(seq_load<T, VEC>(static_cast<const T*>(p.x) + b * p.ld_x + c), win[KW - 1]);
        conv_load_weights<KW, VEC>(p, c, w, bias);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float acc = bias[i];
#pragma unroll
            for (int k = 0; k < KW; ++k)
                if (conv_tap<KW>(k, p.width)) acc = fmaf(w[k][i], win[k][i], acc);
            out[i] = p.silu ? acc * sigmoid_f<T>(acc) : acc;
        }
#pragma unroll
        for (int k = 1; k < KW; ++k)
            if (k >= KW - w1) seq_store<T, VEC>(next + (k - (KW - w1)) * p.channels, win[k]);
    }
    seq_store<T, VEC>(static_cast<T*>(p.y) + b * p.ld_y + c, out);
}

}  // namespace tdx
