// Selective state-space scan, channels last.  With dt' = softplus(dt + dt_bias) (or dt + dt_bias), for every channel d and
// state n (B and C are shared by the channels of a group):
//
//   h[t] = exp(dt'[t, d] A[d, n]) h[t - 1] + dt'[t, d] x[t, d] B[t, n]
//   y[t, d] = sum_n C[t, n] h[t, d, n] + D[d] x[t, d],   out = y * silu(z)  (or y)
//
// The recurrence runs over rows in registers: a thread keeps four states of one channel, N / 4 threads hold a channel's states
// (N: the number of states rounded up to a power of two, the surplus stays zero), and a block of 128 threads walks 512 / N
// channels of one group through a sequence, or through one chunk of it.  It goes in tiles of a few dozen rows: the
// elementwise work of a tile (softplus, silu, the products with x) is spread over all threads and goes through shared memory,
// and so do the sums over a channel's threads.  Neighbouring lanes hold neighbouring channels of the same states, so B and C
// are read once per warp.
//
// Bound by issue and latency, not by memory: registers allow two blocks of four warps on an SM in the main kernels (N = 16), which issue
// in less than half of their cycles and wait for shared memory and for results.  In bf16 with 16 states, whole calls: 4096 x 4096
// forward 239 us (one exponential per state takes 58 at 16 a cycle and SM); 8192 x 2048 training 755 us (forward 158, backward 580, joining
// the sums 20); 128 single tokens of 4096 channels 17.5 us, state traffic at 4.1 TB/s, 63 % of the copy rate.
#pragma once
#include "seq_common.cuh"

namespace tdx {

struct ScanParams {
    long long batch, max_len, rows, channels;
    int states, groups, group_channels, softplus;
    const void* x; long long ld_x;
    const void* dt; long long ld_dt;
    const float* A;
    const void* B; long long ld_b;
    const void* C; long long ld_c;
    const float* D;
    const void* z; long long ld_z;
    const float* dt_bias;
    void* out; long long ld_out;
    const int* offsets;
    const float* state_in;
    float* state_out;
    long long state_stride;
    const int* slots;
    long long n_slots;
    float* saved;                    // per kScanSave rows of a sequence: the state before them (see scan_state_at)
    const void* dout; long long ld_dout;
    void* dx; long long ld_dx;
    void* ddt; long long ld_ddt;
    void* dB; long long ld_db;
    void* dC; long long ld_dc;
    void* dz; long long ld_dz;
    float* dA;
    float* dD;
    float* ddt_bias;
    const float* dstate_out;
    float* dstate_in;
    long long chunk, dense;          // rows of a chunk, chunks per sequence of a dense batch
    int cut;                         // some sequence has more than one chunk
    int channel_tiles;               // per group
    int sum_tiles;                   // channel tiles that have sums of dB and dC of their own, per group
    float* carry;                    // per chunk: its own contribution to the state (or gradient) behind it
    float* carry_dt;                 // [chunk number][channels]: the sum of dt' over a chunk
    float* part_bc;                  // [sum_tiles][rows][groups][2][N]
    float* part_a;                   // per chunk: its sums of dA
    float* part_d;                   // [chunk number][2][channels]: dD, ddt_bias
    int* status;
};

constexpr int kScanSave = 8;         // rows between two saved states; also the rows of a backward tile
constexpr int kScanThreads = 128;

constexpr int kScanStates = 4;       // of a thread

template <int N>
struct ScanShape {
    static constexpr int kPer = N / kScanStates;                          // threads of a channel
    static constexpr int kChannels = kScanThreads / kPer;
    static constexpr int kRows = kChannels >= 128 ? 8 : kChannels >= 64 ? 16 : N <= 32 ? 32 : N == 64 ? 16 : 8;   // rows of a forward tile
};

// Scratch and saved states: [number][state / 4][channel][state % 4], so that a warp reads and writes 512 bytes in one piece.
template <int N>
__device__ __forceinline__ long long scan_state_at(long long number, long long channels, long long c, int n0) {
    return ((number * (N / 4) + n0 / 4) * channels + c) * 4 + n0 % 4;
}
__device__ __forceinline__ void scan_load_states(const float* p, float (&h)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    h[0] = v.x; h[1] = v.y; h[2] = v.z; h[3] = v.w;
}
__device__ __forceinline__ void scan_store_states(float* p, const f32x2 (&h)[2]) { *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(h[0], h[1]); }
// four neighbouring floats of shared memory as pairs
__device__ __forceinline__ void scan_load_pairs(const float* p, f32x2 (&v)[2]) {
    const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(p);
    v[0] = q.x; v[1] = q.y;
}
constexpr float kDecayAddend = 2.4e-8f;
__device__ __forceinline__ f32x2 scan_decay(f32x2 dt, f32x2 a) {
    float lo, hi;
    unpack2(fma2(dt, a, pack2(kDecayAddend, kDecayAddend)), lo, hi);
    return pack2(fast_exp2(lo), fast_exp2(hi));
}

// Where a block works: channels [c0, c0 + live) of a group, a chunk of sequence b.
struct ScanPlace {
    long long b, c0, number;     // number: of the chunk, over all sequences
    int chunk, group, live, tile;
};
template <int CHANNELS>
__device__ __forceinline__ ScanPlace scan_place(const ScanParams& p) {
    ScanPlace r;
    const long long bid = blockIdx.x;
    const int per_chunk = p.channel_tiles * p.groups;
    r.number = bid / per_chunk;
    const int ct = static_cast<int>(bid - r.number * per_chunk);
    const SeqPiece piece = seq_piece(p.offsets, p.batch, p.dense, p.chunk, r.number);
    if (ct == 0) seq_check(p.offsets, r.number, p.batch, p.max_len, p.rows, p.status);
    r.b = piece.b;
    r.chunk = piece.index;
    r.group = ct / p.channel_tiles;
    r.tile = ct - r.group * p.channel_tiles;
    const int in_group = r.tile * CHANNELS;
    r.c0 = static_cast<long long>(r.group) * p.group_channels + in_group;
    r.live = min(CHANNELS, p.group_channels - in_group);
    return r;
}
// First saved state of a sequence that starts at row `first`: no two sequences overlap, and rows / kScanSave + batch
// states hold them all.
__device__ __forceinline__ long long saved_base(const ScanParams& p, long long b, long long first) {
    return p.offsets == nullptr ? b * ((p.max_len + kScanSave - 1) / kScanSave) : first / kScanSave + b;
}

// exp(dt' A) as 2^(dt' A2) with A2 = A log2(e)
__device__ __forceinline__ void scan_load_a(const ScanParams& p, long long c, int n0, bool live, float (&a)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = live && n0 + i < p.states ? __ldg(p.A + c * p.states + n0 + i) * kLog2e : 0.0f;
}
// The caller's state tensors: n_slots x channels x states
__device__ __forceinline__ void scan_read_state(const ScanParams& p, const float* state, long long slot, long long c, int n0, float (&h)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n0 + i < p.states) h[i] = state[slot * p.state_stride + c * p.states + n0 + i];
}
__device__ __forceinline__ void scan_write_state(const ScanParams& p, float* state, long long slot, long long c, int n0, const f32x2 (&h)[2]) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) unpack2(h[i / 2], v[i], v[i + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n0 + i < p.states) state[slot * p.state_stride + c * p.states + n0 + i] = v[i];
}
// The sum of a channel's threads' values, a row of kPer * kRows * kChannels floats [thread][row][channel]; VEC neighbouring channels
template <int PER, int STRIDE, int VEC>
__device__ __forceinline__ void scan_sum(const float* p, float (&s)[VEC]) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        if (VEC == 2) {
            const float2 v = *reinterpret_cast<const float2*>(p + q * STRIDE);
            s[0] += v.x;
            s[VEC - 1] += v.y;
        } else {
            s[0] += p[q * STRIDE];
        }
    }
}

enum ScanMode { kScanFull = 0, kScanState = 1, kScanAdjoint = 2 };

// States and channels that only fill up a thread or a block have a, B and C of zero and add nothing, as long as all is finite: an
// infinity (or an overflow) times their zeros is not a number, which stays in their states and spoils the sums.  Their states are
// zero by right, so that a look at them behind each tile shows it, and the tile is then gone through again with them kept at zero,
// by a function of its own that takes nothing from the kernel's loops.  (4096 x 4096 x 16 forward and 8192 x 2048 x 16 training: a
// look at every element in front of the tile cost 3.6 and 3.2 percent, the second walk as a part of the kernel 0.9 and 1.3, this form nothing;
// with states or channels to fill up it costs up to 5 percent.)
// States n and n + 1 of v:
__device__ __forceinline__ f32x2 scan_keep(f32x2 v, int n, int states) {
    const f32x2 low = n < states ? 0xffffffffull : 0ull, high = n + 1 < states ? 0xffffffff00000000ull : 0ull;
    return v & (low | high);
}
__device__ __forceinline__ bool scan_spoilt(const f32x2 (&v)[2], int n0, int states) {
    return v[0] != scan_keep(v[0], n0, states) || v[1] != scan_keep(v[1], n0 + 2, states);
}
struct ScanStates { f32x2 v[2]; };
// A tile of the forward kernel again, from the states `h` in front of it; dt, b, c and y: the tile in shared memory, y from this
// thread's first place on.
template <int N, int MODE>
__device__ __noinline__ ScanStates scan_again(ScanStates h, ScanStates a, const float4* dt, const float* b, const float* c, float* y, int ch, int n0,
                                              int states, float* saved, long long save_step, int left) {
    constexpr int kRows = ScanShape<N>::kRows, kCh = ScanShape<N>::kChannels;
    constexpr bool kBack = MODE == kScanAdjoint;
#pragma unroll 1
    for (int r = 0; r < kRows; ++r) {
        if (MODE == kScanFull && r % kScanSave == 0 && saved) {
            if (r < left) scan_store_states(saved, h.v);
            saved += save_step;
        }
        const int row = kBack ? kRows - 1 - r : r;
        const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(dt + row * kCh + ch);
        f32x2 bv[2], cv[2], sum = 0;
        scan_load_pairs(b + row * N + n0, bv);
        if (MODE == kScanFull) scan_load_pairs(c + row * N + n0, cv);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x2 w = scan_decay(d.x, a.v[i]), u = mul2(d.y, bv[i]);
            h.v[i] = scan_keep(kBack ? mul2(w, add2(u, h.v[i])) : fma2(w, h.v[i], u), n0 + 2 * i, states);
            if (MODE == kScanFull) sum = i == 0 ? mul2(h.v[i], cv[i]) : fma2(h.v[i], cv[i], sum);
        }
        if (MODE == kScanFull) {
            float lo, hi;
            unpack2(sum, lo, hi);
            y[r * kCh] = lo + hi;
        }
    }
    return h;
}

// kScanFull: the forward pass over a chunk, from the state before it.
// kScanState: only the state that a chunk adds to what comes before it, h from h = 0, and the sum of dt'.  (The chunk's
//   effect on an incoming state is then exp(A * sum dt').)  Run first when a sequence is cut into chunks, for all chunks but
//   the last; chunk 0 starts from the caller's state.
// kScanAdjoint: the same for the gradient, from the last row to the first: q <- exp(dt' A) (q + C dy).
//
// VEC neighbouring channels (2 where the rows' alignment allows) are one element of the elementwise work, which is as long as the
// recurrence itself unless its addresses and checks are kept cheap: a thread's offsets in a tile are computed once, and a full
// tile is read without checks.
// Blocks per SM that the register bound asks for; 0: no bound.  Three where they fit without spills and the compiler would take more (8
// states in bf16, two channels an access: 81 us instead of 107 for 2 x 2048 rows of 2048 channels); one with 32 states, where its
// own choice is less than two blocks may have (146 us instead of 158).
constexpr int scan_fwd_blocks(int n, int vec, int elem_bytes) { return n == 64 || (n == 8 && vec == 2 && elem_bytes == 2) ? 3 : n == 32 ? 1 : 0; }
template <typename T, int N, int MODE, int VEC>
__global__ void __launch_bounds__(kScanThreads, scan_fwd_blocks(N, VEC, sizeof(T))) scan_fwd_kernel(const __grid_constant__ ScanParams p) {
    typedef ScanShape<N> Shape;
    typedef SeqVec<T, VEC> raw_t;
    constexpr int kRows = Shape::kRows, kCh = Shape::kChannels, kPer = Shape::kPer, S = kScanStates, P = S / 2;
    constexpr int kAcross = kCh / VEC, kStep = kScanThreads / kAcross;                    // threads along a row, rows between a thread's elements
    constexpr int kEl = (kRows + kStep - 1) / kStep;
    constexpr int kBcStep = N >= kScanThreads ? 1 : kScanThreads / N, kBc = (kRows + kBcStep - 1) / kBcStep;
    __shared__ float4 s_dt[kRows][kCh];                  // dt', dt', dt' x, dt' x   (kScanAdjoint: dy for dt' x)
    __shared__ __align__(16) float s_b[kRows][N];
    __shared__ __align__(16) float s_c[MODE == kScanFull ? kRows : 1][N];
    __shared__ __align__(16) float s_y[MODE == kScanFull ? kPer : 1][kRows][kCh];
    seq_grid_wait();
    const ScanPlace at = scan_place<kCh>(p);
    const SeqRange seq = seq_range(p.offsets, at.b, p.max_len, p.rows, p.status);
    const int tid = threadIdx.x;
    const int chunk = static_cast<int>(p.chunk), last = seq.len > 0 ? (seq.len - 1) / chunk : 0;
    const int t0 = min(at.chunk, last + 1) * chunk, t1 = min(seq.len, t0 + chunk);
    if (MODE == kScanFull && t0 >= seq.len && at.chunk > 0) return;
    if (MODE == kScanState && t1 >= seq.len && at.chunk > 0) return;
    if (MODE == kScanAdjoint && (t0 >= seq.len || at.chunk == 0)) return;
    const int ch = tid % kCh, per = tid / kCh, n0 = per * S;
    const bool live = ch < at.live;
    const long long c = at.c0 + (live ? ch : 0);
    const long long slot = MODE != kScanAdjoint && (p.state_in || p.state_out) ? state_slot(p.slots, at.b, p.n_slots, p.status) : -1;
    float av[S], hv[S];
    scan_load_a(p, c, n0, live, av);
#pragma unroll
    for (int i = 0; i < S; ++i) hv[i] = 0.0f;
    // The state before chunk 0.  When a sequence is cut, the first launch keeps a copy of it where the last chunk's sum would
    // stand (which nobody needs): in the second launch the last chunk may write state_out over state_in before chunk 0 reads it.
    if (MODE != kScanAdjoint && at.chunk == 0 && p.state_in && slot >= 0 && live) {
        float* kept = p.carry + scan_state_at<N>(at.number + last, p.channels, c, n0);
        if (MODE == kScanFull && p.cut) {
            scan_load_states(kept, hv);
        } else {
            scan_read_state(p, p.state_in, slot, c, n0, hv);
            if (MODE == kScanState) {
#pragma unroll
                for (int i = 0; i < S; ++i) kept[i] = hv[i];
            }
        }
    }
    if (MODE == kScanState && t1 >= seq.len) return;
    if (MODE == kScanFull && at.chunk > 0 && live) {
        for (int k = 0; k < at.chunk; ++k) {
            const long long number = at.number - at.chunk + k;
            float add[S];
            scan_load_states(p.carry + scan_state_at<N>(number, p.channels, c, n0), add);
            const float sum = k == 0 ? 0.0f : p.carry_dt[number * p.channels + c];
#pragma unroll
            for (int i = 0; i < S; ++i) hv[i] = fmaf(hv[i], fast_exp2(av[i] * sum), add[i]);
        }
    }
    f32x2 h[P], a[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        h[i] = scan_keep(pack2(hv[2 * i], hv[2 * i + 1]), n0 + 2 * i, p.states);
        a[i] = pack2(av[2 * i], av[2 * i + 1]);
    }

    const long long ld_x = MODE == kScanAdjoint ? p.ld_dout : p.ld_x, ld_b = MODE == kScanAdjoint ? p.ld_c : p.ld_b;
    float* saved = MODE == kScanFull && p.saved && live ? p.saved + scan_state_at<N>(saved_base(p, at.b, seq.first) + t0 / kScanSave, p.channels, c, n0) : nullptr;
    const long long save_step = static_cast<long long>(N) * p.channels;

    // This thread's elements of a tile: channels cc .. cc + VEC - 1, rows er, er + kStep, ...; and its values of B and C.  Pointers
    // move on from tile to tile, offsets inside a tile fit 32 bits (ld <= 2^24).
    constexpr bool kBack = MODE == kScanAdjoint;
    const int tiles = (t1 - t0 + kRows - 1) / kRows, first_row = t0 + (kBack ? tiles - 1 : 0) * kRows;
    const int cc = (tid % kAcross) * VEC, er = tid / kAcross, bn = tid % N, br = tid / N;
    const bool col_live = cc < at.live;                  // VEC divides the live channels
    const T* px = static_cast<const T*>(kBack ? p.dout : p.x) + (seq.first + first_row + er) * ld_x + at.c0 + cc;
    const T* pdt = static_cast<const T*>(p.dt) + (seq.first + first_row + er) * p.ld_dt + at.c0 + cc;
    const T* pz = static_cast<const T*>(p.z) + (seq.first + first_row + er) * p.ld_z + at.c0 + cc;
    const T* pb = static_cast<const T*>(kBack ? p.C : p.B) + (seq.first + first_row + br) * ld_b + at.group * p.states + bn;
    const T* pc = static_cast<const T*>(p.C) + (seq.first + first_row + br) * p.ld_c + at.group * p.states + bn;
    T* pout = static_cast<T*>(p.out) + (seq.first + first_row + er) * p.ld_out + at.c0 + cc;
    const uint32_t step_x = static_cast<uint32_t>(kStep * ld_x), step_dt = static_cast<uint32_t>(kStep * p.ld_dt), step_z = static_cast<uint32_t>(kStep * p.ld_z),
                   step_out = static_cast<uint32_t>(kStep * p.ld_out), step_b = static_cast<uint32_t>(kBcStep * ld_b), step_c = static_cast<uint32_t>(kBcStep * p.ld_c);
    raw_t rx[kEl], rdt[kEl], rz[kEl];
    T rb[kBc], rc[kBc];
    // GATED and CHECKED are compile-time in the loops below: a branch per element would keep the elements from overlapping
    auto fetch_as = [&](auto gated, auto checked, int left) {
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            if (!decltype(checked)::value || (er + i * kStep < left && col_live)) {
                rx[i] = seq_load<T, VEC>(px + i * step_x);
                rdt[i] = seq_load<T, VEC>(pdt + i * step_dt);
                if (decltype(gated)::value) rz[i] = seq_load<T, VEC>(pz + i * step_z);
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            if (!decltype(checked)::value || (br + i * kBcStep < left && bn < p.states)) {
                rb[i] = __ldg(pb + i * step_b);
                if (MODE == kScanFull) rc[i] = __ldg(pc + i * step_c);
            }
        }
    };
    const bool gated = p.z != nullptr && MODE != kScanState;
    const bool whole = at.live == kCh && p.states == N && kRows % kStep == 0 && kRows % kBcStep == 0;
    auto fetch = [&](int row0) {
        const int left = min(t1 - row0, kRows);
        if (whole && left == kRows) {
            if (gated) fetch_as(SeqYes(), SeqNo(), left);
            else fetch_as(SeqNo(), SeqNo(), left);
        } else {
            if (gated) fetch_as(SeqYes(), SeqYes(), left);
            else fetch_as(SeqNo(), SeqYes(), left);
        }
        const long long move = kBack ? -kRows : kRows;
        px += move * ld_x;
        pdt += move * p.ld_dt;
        if (gated) pz += move * p.ld_z;
        pb += move * ld_b;
        pc += move * p.ld_c;
    };
    float bias[VEC], skip[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        bias[v] = p.dt_bias && col_live ? __ldg(p.dt_bias + at.c0 + cc + v) : 0.0f;
        skip[v] = MODE == kScanFull && p.D && col_live ? __ldg(p.D + at.c0 + cc + v) : 0.0f;
    }
    float ex[kEl][VEC], ez[kEl][VEC];
    auto elementwise_as = [&](auto gated, auto softplus, int left) {
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int r = er + i * kStep;
            if (kRows % kStep == 0 || r < kRows) {
                const bool there = r < left && col_live;
                float f[VEC], zf[VEC];
                seq_unpack<T, VEC>(rx[i], ex[i]);
                seq_unpack<T, VEC>(rdt[i], f);
                if (decltype(gated)::value) seq_unpack<T, VEC>(rz[i], zf);
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    float d = f[v] + bias[v];
                    if (decltype(softplus)::value) d = softplus_f<T>(d);
                    ez[i][v] = decltype(gated)::value ? zf[v] * sigmoid_f<T>(zf[v]) : 1.0f;
                    float w = kBack ? ex[i][v] * ez[i][v] : d * ex[i][v];
                    if (!there) d = w = 0.0f;
                    s_dt[r][cc + v] = make_float4(d, d, w, w);
                }
            }
        }
    };
    float sum_dt = 0.0f;
    // The recurrence over four rows, and beside it the decays of the four rows behind them and the loads of the four behind
    // those: decays and inputs do not depend on the state, and the special-function unit (one exponential per state and row, 16 a
    // cycle on an SM) is the narrowest part, so a warp alone should keep it busy.
    constexpr int kAhead = 4, kGroups = kRows / kAhead;
    ulonglong2 dv[2][kAhead];
    f32x2 bv[2][kAhead][P], cv[2][kAhead][P], w[2][kAhead][P], u[2][kAhead][P];
    auto load_row = [&](int r, ulonglong2& d, f32x2 (&b)[P]) {
        const int row = kBack ? kRows - 1 - r : r;
        d = *reinterpret_cast<const ulonglong2*>(&s_dt[row][ch]);
        scan_load_pairs(&s_b[row][n0], b);
    };
    auto decay_row = [&](int r, const ulonglong2& d, const f32x2 (&b)[P], f32x2 (&ww)[P], f32x2 (&uu)[P], f32x2 (&c4)[P]) {
        if (MODE == kScanFull) scan_load_pairs(&s_c[r][n0], c4);
        else sum_dt += __uint_as_float(static_cast<uint32_t>(d.x));
#pragma unroll
        for (int i = 0; i < P; ++i) {
            ww[i] = scan_decay(d.x, a[i]);
            uu[i] = mul2(d.y, b[i]);
        }
    };
    auto walk_row = [&](int r, const f32x2 (&ww)[P], const f32x2 (&uu)[P], const f32x2 (&c4)[P]) {
#pragma unroll
        for (int i = 0; i < P; ++i) h[i] = kBack ? mul2(ww[i], add2(uu[i], h[i])) : fma2(ww[i], h[i], uu[i]);
        if (MODE == kScanFull) {
            f32x2 y = mul2(h[0], c4[0]);
#pragma unroll
            for (int i = 1; i < P; ++i) y = fma2(h[i], c4[i], y);
            float lo, hi;
            unpack2(y, lo, hi);
            s_y[per][r][ch] = lo + hi;
        }
    };
    const bool padded = p.states < N;                    // see scan_again
    if (tiles > 0) fetch(first_row);
    for (int tile = 0; tile < tiles; ++tile) {
        const int row0 = kBack ? first_row - tile * kRows : first_row + tile * kRows, left = min(t1 - row0, kRows);
        if (p.softplus) {
            if (gated) elementwise_as(SeqYes(), SeqYes(), left);
            else elementwise_as(SeqNo(), SeqYes(), left);
        } else {
            if (gated) elementwise_as(SeqYes(), SeqNo(), left);
            else elementwise_as(SeqNo(), SeqNo(), left);
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int r = br + i * kBcStep;
            if (kRows % kBcStep == 0 || r < kRows) {
                const bool there = r < left && bn < p.states;
                s_b[r][bn] = there ? seq_to_float(rb[i]) : 0.0f;
                if (MODE == kScanFull) s_c[r][bn] = there ? seq_to_float(rc[i]) : 0.0f;
            }
        }
        __syncthreads();
        if (tile + 1 < tiles) fetch(kBack ? row0 - kRows : row0 + kRows);
        const ScanStates before = {{h[0], h[1]}};
        float* saved_before = saved;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) load_row(k, dv[0][k], bv[0][k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            load_row(kAhead + k, dv[1][k], bv[1][k]);
            decay_row(k, dv[0][k], bv[0][k], w[0][k], u[0][k], cv[0][k]);
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int now = g & 1, next = now ^ 1;
            if (MODE == kScanFull && g * kAhead % kScanSave == 0 && saved) {
                if (g * kAhead < left) scan_store_states(saved, h);
                saved += save_step;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (g + 2 < kGroups) load_row((g + 2) * kAhead + k, dv[now][k], bv[now][k]);
                if (g + 1 < kGroups) decay_row((g + 1) * kAhead + k, dv[next][k], bv[next][k], w[next][k], u[next][k], cv[next][k]);
                walk_row(g * kAhead + k, w[now][k], u[now][k], cv[now][k]);
            }
        }
        if (padded && scan_spoilt(h, n0, p.states)) {
            const ScanStates again = scan_again<N, MODE>(before, {{a[0], a[1]}}, &s_dt[0][0], &s_b[0][0], &s_c[0][0], &s_y[MODE == kScanFull ? per : 0][0][ch], ch,
                                                         n0, p.states, saved_before, save_step, left);
            h[0] = again.v[0];
            h[1] = again.v[1];
        }
        __syncthreads();
        if (MODE == kScanFull) {
#pragma unroll
            for (int i = 0; i < kEl; ++i) {
                const int r = er + i * kStep;
                if (r < left && col_live) {
                    float y[VEC];
#pragma unroll
                    for (int v = 0; v < VEC; ++v) y[v] = skip[v] * ex[i][v];
                    scan_sum<kPer, kRows * kCh, VEC>(&s_y[0][r][cc], y);
#pragma unroll
                    for (int v = 0; v < VEC; ++v) y[v] *= ez[i][v];
                    seq_store<T, VEC>(pout + i * step_out, y);
                }
            }
            pout += kRows * p.ld_out;
        }
    }
    if (MODE != kScanFull) {
        if (live) {
            scan_store_states(p.carry + scan_state_at<N>(at.number, p.channels, c, n0), h);
            if (per == 0) p.carry_dt[at.number * p.channels + c] = sum_dt;
        }
    } else if (p.state_out && slot >= 0 && live && t1 >= seq.len) {
        scan_write_state(p, p.state_out, slot, c, n0, h);
    }
}

// dB and dC are sums over channels, that is, over a warp's lanes (groups of CHANNELS lanes where a warp holds several sets of
// states).  Four rows' terms of a warp go through shared memory: eight lists of 32 x four states, each summed by four lanes, an
// eighth of 16-byte loads apart so that no two lanes of a quarter-warp meet in a bank.  (Two other ways were measured on the
// backward pass of 8192 rows x 2048 channels x 16 states: sums on the tensor cores, with terms cut into two tf32 parts, were
// bound by the rate of mma.m16n8k8 there, 8 cycles for 64 terms; butterflies of shuffles by their selects.)
constexpr int kScanSumPitch = 33;      // 16-byte places per list
template <int CHANNELS>
__device__ __forceinline__ void scan_sum_lanes(const float4* list, int lane, float* to, long long row_step, int n_states, int rows) {
    const int v = lane / 4, part = lane % 4, row = v / 2, which = v % 2;       // lists: [row][dB, dC]
    const float4* from = list + v * kScanSumPitch;
    float* out = to + row * row_step + which * n_states;
    const bool there = row < rows;
    if (CHANNELS == 4) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 q = from[part * 8 + half * 4 + i];
                s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
            }
            if (there) *reinterpret_cast<float4*>(out + (part * 2 + half) * 4) = s;
        }
        return;
    }
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 q = from[part * 8 + ((i + 2 * part) & 7)];
        s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
    }
    if (CHANNELS == 8) {
        if (there) *reinterpret_cast<float4*>(out + part * 4) = s;
        return;
    }
    // lanes with bit 0 go on with the last two states, the others with the first two
    const bool odd = lane & 1;
    float x = odd ? s.z : s.x, y = odd ? s.w : s.y;
    x += __shfl_xor_sync(0xffffffffu, odd ? s.x : s.z, 1);
    y += __shfl_xor_sync(0xffffffffu, odd ? s.y : s.w, 1);
    if (CHANNELS == 16) {
        if (there) *reinterpret_cast<float2*>(out + part / 2 * 4 + 2 * odd) = make_float2(x, y);
        return;
    }
    const bool second = lane & 2;
    const float mine = (second ? y : x) + __shfl_xor_sync(0xffffffffu, second ? x : y, 2);
    if (there) out[2 * odd + second] = mine;
}

// A tile of the backward kernel again, with the states that only fill up kept at zero, and the sum of dA over the tile's own rows only
// (dlog dt' is zero behind them only while dlog is finite).  h: states in front of the tile; q: gradient behind it; sum: this thread's
// place for row 0 in s_sum.
struct ScanBwdStates { ScanStates q, ta; };
template <int N>
__device__ __noinline__ ScanBwdStates scan_bwd_again(ScanStates h, ScanStates q, ScanStates a, const float2* dt, const float* g, const float* b, const float* c,
                                                     float* sum, float4* list, int ch, int n0, int states, int left, float* part_bc, long long bc_step) {
    constexpr int kRows = kScanSave, kCh = ScanShape<N>::kChannels, kSum = ScanShape<N>::kPer * kRows * kCh;
    const int lane = threadIdx.x & 31;
    f32x2 hs[kRows + 1][2], w[kRows][2];
    ScanBwdStates r = {q, {{0, 0}}};
    hs[0][0] = h.v[0];
    hs[0][1] = h.v[1];
#pragma unroll 1
    for (int t = 0; t < kRows; ++t) {
        const float2 d = dt[t * kCh + ch];
        f32x2 bv[2];
        scan_load_pairs(b + t * N + n0, bv);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            w[t][i] = scan_keep(scan_decay(pack2(d.x, d.x), a.v[i]), n0 + 2 * i, states);
            hs[t + 1][i] = scan_keep(fma2(w[t][i], hs[t][i], mul2(pack2(d.y, d.y), bv[i])), n0 + 2 * i, states);
        }
    }
#pragma unroll 1
    for (int t = kRows - 1; t >= 0; --t) {
        const float2 d = dt[t * kCh + ch];
        const float gv = g[t * kCh + ch];
        f32x2 bv[2], cv[2], db[2], dc[2], y = 0, du = 0, dl = 0;
        scan_load_pairs(b + t * N + n0, bv);
        scan_load_pairs(c + t * N + n0, cv);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x2 dh = scan_keep(fma2(pack2(gv, gv), cv[i], r.q.v[i]), n0 + 2 * i, states);
            r.q.v[i] = mul2(w[t][i], dh);
            const f32x2 dlog = mul2(r.q.v[i], hs[t][i]);
            if (t < left) r.ta.v[i] = fma2(dlog, pack2(d.x, d.x), r.ta.v[i]);
            y = i == 0 ? mul2(hs[t + 1][i], cv[i]) : fma2(hs[t + 1][i], cv[i], y);
            du = i == 0 ? mul2(dh, bv[i]) : fma2(dh, bv[i], du);
            dl = i == 0 ? mul2(dlog, a.v[i]) : fma2(dlog, a.v[i], dl);
            db[i] = mul2(dh, pack2(d.y, d.y));
            dc[i] = mul2(hs[t + 1][i], pack2(gv, gv));
        }
        float lo, hi;
        unpack2(y, lo, hi);
        sum[t * kCh] = lo + hi;
        unpack2(dl, lo, hi);
        sum[kSum + t * kCh] = lo + hi;
        unpack2(du, lo, hi);
        sum[2 * kSum + t * kCh] = lo + hi;
        *reinterpret_cast<ulonglong2*>(&list[(t % 4 * 2) * kScanSumPitch + lane]) = make_ulonglong2(db[0], db[1]);
        *reinterpret_cast<ulonglong2*>(&list[(t % 4 * 2 + 1) * kScanSumPitch + lane]) = make_ulonglong2(dc[0], dc[1]);
        if (t % 4 == 0) {
            __syncwarp();
            scan_sum_lanes<kCh>(list, lane, part_bc + t * bc_step, bc_step, N, left - t);
            __syncwarp();
        }
    }
    return r;
}

// Backward.  With g = dout * silu(z) (or dout), for one channel and state
//   dh[t] = C[t] g[t] + a[t + 1] dh[t + 1],   a[t] = exp(dt'[t] A)
//   dC[t] = sum_d g h,   dB[t] = sum_d dh dt' x,   dlog = dh a h[t - 1],   dA = sum_t dlog dt'
//   dx = dt' sum_n dh B + D g,   ddt' = sum_n dlog A + x sum_n dh B,   dz = dout y silu'(z),   dD = sum_t g x.
// A block walks its chunk from the last tile of kScanSave rows to the first.  For each it starts from the saved state in
// front of the tile, recomputes the tile's states and decays into registers, and then goes back through them.  Sums over
// states and over the block's channels go through shared memory; sums over blocks are left to scan_bwd_join_kernel, so every
// sum has a fixed order.
template <typename T, int N, int VEC>
__global__ void __launch_bounds__(kScanThreads) scan_bwd_kernel(const __grid_constant__ ScanParams p) {
    typedef ScanShape<N> Shape;
    typedef SeqVec<T, VEC> raw_t;
    constexpr int kRows = kScanSave, kCh = Shape::kChannels, kPer = Shape::kPer, S = kScanStates, P = S / 2;
    constexpr int kAcross = kCh / VEC, kStep = kScanThreads / kAcross;
    constexpr int kEl = (kRows + kStep - 1) / kStep;
    constexpr int kBcStep = N >= kScanThreads ? 1 : kScanThreads / N, kBc = (kRows + kBcStep - 1) / kBcStep;
    constexpr int kSubs = kCh > 32 ? kCh / 32 : 1;         // warps that share their states
    // (each once: twice, as in the forward kernel, saves moves, but shared memory is busier here; 781 instead of 766 us for the
    // training step of 8192 rows x 2048 channels x 16 states)
    __shared__ float2 s_dt[kRows][kCh];                    // dt', dt' x
    __shared__ float s_g[kRows][kCh];
    auto dt_at = [&](int r, int c) { return make_ulonglong2(pack2(s_dt[r][c].x, s_dt[r][c].x), pack2(s_dt[r][c].y, s_dt[r][c].y)); };
    __shared__ __align__(16) float s_b[kRows][N];
    __shared__ __align__(16) float s_c[kRows][N];
    __shared__ float4 s_list[kScanThreads / 32][8][kScanSumPitch];      // see scan_sum_lanes
    __shared__ __align__(16) float s_sum[3][kPer][kRows][kCh];         // per thread: its states' share of y, sum dlog A2, sum dh B
    seq_grid_wait();
    const ScanPlace at = scan_place<kCh>(p);
    const SeqRange seq = seq_range(p.offsets, at.b, p.max_len, p.rows, p.status);
    const int tid = threadIdx.x, lane = tid & 31;
    const int chunk = static_cast<int>(p.chunk), last = seq.len > 0 ? (seq.len - 1) / chunk : 0;
    const int t0 = min(at.chunk, last + 1) * chunk, t1 = min(seq.len, t0 + chunk);
    const int ch = tid % kCh, per = tid / kCh, n0 = per * S;
    const bool live = ch < at.live;
    const long long c = at.c0 + (live ? ch : 0);
    const long long slot = p.dstate_in || p.dstate_out ? state_slot(p.slots, at.b, p.n_slots, p.status) : -1;
    float av[S], qv[S];
    scan_load_a(p, c, n0, live, av);
    // the gradient that comes from behind the chunk
#pragma unroll
    for (int i = 0; i < S; ++i) qv[i] = 0.0f;
    if (live) {
        if (p.dstate_out && slot >= 0) scan_read_state(p, p.dstate_out, slot, c, n0, qv);
        for (int k = last; k > at.chunk; --k) {
            const long long number = at.number - at.chunk + k;
            float add[S];
            scan_load_states(p.carry + scan_state_at<N>(number, p.channels, c, n0), add);
            const float sum = p.carry_dt[number * p.channels + c];
#pragma unroll
            for (int i = 0; i < S; ++i) qv[i] = fmaf(qv[i], fast_exp2(av[i] * sum), add[i]);
        }
    }
    const int live_states = live ? p.states : 0;
    f32x2 q[P], a[P], da[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        q[i] = scan_keep(pack2(qv[2 * i], qv[2 * i + 1]), n0 + 2 * i, p.states);
        a[i] = pack2(av[2 * i], av[2 * i + 1]);
        da[i] = pack2(0.f, 0.f);
    }
    const T* x = static_cast<const T*>(p.x) + seq.first * p.ld_x + at.c0;
    const T* dt = static_cast<const T*>(p.dt) + seq.first * p.ld_dt + at.c0;
    const T* z = p.z ? static_cast<const T*>(p.z) + seq.first * p.ld_z + at.c0 : nullptr;
    const T* dout = static_cast<const T*>(p.dout) + seq.first * p.ld_dout + at.c0;
    const T* B = static_cast<const T*>(p.B) + seq.first * p.ld_b + at.group * p.states;
    const T* C = static_cast<const T*>(p.C) + seq.first * p.ld_c + at.group * p.states;
    const float* saved = p.saved + scan_state_at<N>(saved_base(p, at.b, seq.first), p.channels, c, n0);

    // this thread's elements of a tile: channels cc .. cc + VEC - 1, rows er, er + kStep, ...; offsets fit 32 bits (ld <= 2^24)
    const int cc = (tid % kAcross) * VEC, er = tid / kAcross, bn = tid % N, br = tid / N;
    const bool col_live = cc < at.live;                    // VEC divides the live channels
    raw_t rx[kEl], rdt[kEl], rz[kEl], rg[kEl];
    T rb[kBc], rc[kBc];
    float rh[S];
    auto fetch = [&](int row0) {
        const T* xt = x + row0 * p.ld_x;
        const T* dtt = dt + row0 * p.ld_dt;
        const T* gt = dout + row0 * p.ld_dout;
        const T* zt = z + row0 * p.ld_z;
        const T* bt = B + row0 * p.ld_b;
        const T* ct = C + row0 * p.ld_c;
        const int left = min(t1 - row0, kRows);
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int r = er + i * kStep;
            if (r < left && col_live) {
                rx[i] = seq_load<T, VEC>(xt + static_cast<uint32_t>(r * p.ld_x + cc));
                rdt[i] = seq_load<T, VEC>(dtt + static_cast<uint32_t>(r * p.ld_dt + cc));
                rg[i] = seq_load<T, VEC>(gt + static_cast<uint32_t>(r * p.ld_dout + cc));
                if (z) rz[i] = seq_load<T, VEC>(zt + static_cast<uint32_t>(r * p.ld_z + cc));
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int r = br + i * kBcStep;
            if (r < left && bn < p.states) {
                rb[i] = bt[static_cast<uint32_t>(r * p.ld_b + bn)];
                rc[i] = ct[static_cast<uint32_t>(r * p.ld_c + bn)];
            }
        }
        if (live) scan_load_states(saved + row0 / kRows * (N * p.channels), rh);
    };
#pragma unroll
    for (int i = 0; i < S; ++i) rh[i] = 0.0f;
    float bias[VEC], skip[VEC], sum_d[VEC], sum_bias[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        bias[v] = p.dt_bias && col_live ? __ldg(p.dt_bias + at.c0 + cc + v) : 0.0f;
        skip[v] = p.D && col_live ? __ldg(p.D + at.c0 + cc + v) : 0.0f;
        sum_d[v] = sum_bias[v] = 0.0f;
    }
    const long long sum_tile = at.tile * kSubs + (kCh > 32 ? tid % kCh / 32 : 0);
    const long long bc_step = static_cast<long long>(p.groups) * 2 * N;            // from row to row
    float* part_bc = p.part_bc + (sum_tile * p.rows + seq.first) * bc_step + at.group * 2 * N + (kCh >= 32 ? n0 : tid / 32 * (32 / kCh) * S);
    float4* list = &s_list[tid / 32][0][0];

    const int tiles = (max(t1 - t0, 0) + kRows - 1) / kRows;
    if (tiles > 0) fetch(t0 + (tiles - 1) * kRows);
    for (int tile = tiles - 1; tile >= 0; --tile) {
        const int row0 = t0 + tile * kRows, left = min(t1 - row0, kRows);
        const bool padded = at.live < kCh || p.states < N || left < kRows;       // see scan_bwd_again
        // x, dt', d dt' / d dt, z, sigmoid(z), dout, g
        float ex[kEl][VEC], ed[kEl][VEC], eds[kEl][VEC], ez[kEl][VEC], ezs[kEl][VEC], eo[kEl][VEC], eg[kEl][VEC];
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int r = er + i * kStep;
            if (kRows % kStep == 0 || r < kRows) {
                const bool there = r < left && col_live;
                seq_unpack<T, VEC>(rx[i], ex[i]);
                seq_unpack<T, VEC>(rdt[i], ed[i]);
                seq_unpack<T, VEC>(rg[i], eo[i]);
                seq_unpack<T, VEC>(rz[i], ez[i]);
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    ed[i][v] += bias[v];
                    const float soft = softplus_grad_f<T>(ed[i][v], eds[i][v]);
                    ed[i][v] = p.softplus ? soft : ed[i][v];
                    eds[i][v] = p.softplus ? eds[i][v] : 1.0f;
                    ezs[i][v] = sigmoid_f<T>(ez[i][v]);
                    eg[i][v] = z ? eo[i][v] * (ez[i][v] * ezs[i][v]) : eo[i][v];
                    float w = ed[i][v] * ex[i][v];
                    if (!there) ed[i][v] = w = eg[i][v] = 0.0f;
                    s_dt[r][cc + v] = make_float2(ed[i][v], w);
                    s_g[r][cc + v] = eg[i][v];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int r = br + i * kBcStep;
            if (kRows % kBcStep == 0 || r < kRows) {
                const bool there = r < left && bn < p.states;
                s_b[r][bn] = there ? seq_to_float(rb[i]) : 0.0f;
                s_c[r][bn] = there ? seq_to_float(rc[i]) : 0.0f;
            }
        }
        f32x2 hs[kRows + 1][P], w[kRows][P];
#pragma unroll
        for (int i = 0; i < P; ++i) hs[0][i] = pack2(rh[2 * i], rh[2 * i + 1]);
        __syncthreads();
        if (tile > 0) fetch(row0 - kRows);
        const ScanStates behind = {{q[0], q[1]}};
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const ulonglong2 dv = dt_at(r, ch);
            f32x2 b[P];
            scan_load_pairs(&s_b[r][n0], b);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                w[r][i] = scan_decay(dv.x, a[i]);
                hs[r + 1][i] = fma2(w[r][i], hs[r][i], mul2(dv.y, b[i]));
            }
        }
        bool spoilt = padded && scan_spoilt(hs[kRows], n0, live_states);
        f32x2 ta[P];
#pragma unroll
        for (int i = 0; i < P; ++i) ta[i] = pack2(0.f, 0.f);
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r) {
            const ulonglong2 dv = dt_at(r, ch);
            const f32x2 g2 = pack2(s_g[r][ch], s_g[r][ch]);
            f32x2 b[P], cv[P], db[P], dc[P], y, du, dl;
            scan_load_pairs(&s_b[r][n0], b);
            scan_load_pairs(&s_c[r][n0], cv);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const f32x2 dh = fma2(g2, cv[i], q[i]);
                q[i] = mul2(w[r][i], dh);
                const f32x2 dlog = mul2(q[i], hs[r][i]);
                ta[i] = fma2(dlog, dv.x, ta[i]);
                y = i == 0 ? mul2(hs[r + 1][i], cv[i]) : fma2(hs[r + 1][i], cv[i], y);
                du = i == 0 ? mul2(dh, b[i]) : fma2(dh, b[i], du);
                dl = i == 0 ? mul2(dlog, a[i]) : fma2(dlog, a[i], dl);
                db[i] = mul2(dh, dv.y);
                dc[i] = mul2(hs[r + 1][i], g2);
            }
            float lo, hi;
            unpack2(y, lo, hi);
            s_sum[0][per][r][ch] = lo + hi;
            unpack2(dl, lo, hi);
            s_sum[1][per][r][ch] = lo + hi;
            unpack2(du, lo, hi);
            s_sum[2][per][r][ch] = lo + hi;
            *reinterpret_cast<ulonglong2*>(&list[(r % 4 * 2) * kScanSumPitch + lane]) = make_ulonglong2(db[0], db[1]);
            *reinterpret_cast<ulonglong2*>(&list[(r % 4 * 2 + 1) * kScanSumPitch + lane]) = make_ulonglong2(dc[0], dc[1]);
            if (r % 4 == 0) {
                __syncwarp();
                scan_sum_lanes<kCh>(list, lane, part_bc + (row0 + r) * bc_step, bc_step, N, left - r);
                __syncwarp();
            }
        }
        if (padded) {
            spoilt |= scan_spoilt(q, n0, live_states);
            if (left < kRows) {
                float lo, hi;
                unpack2(add2(ta[0], ta[1]), lo, hi);
                spoilt |= lo + hi != lo + hi;
            }
            if (__any_sync(0xffffffffu, spoilt)) {         // lanes share the sums of dB and dC
                const ScanBwdStates again = scan_bwd_again<N>({{hs[0][0], hs[0][1]}}, behind, {{a[0], a[1]}}, &s_dt[0][0], &s_g[0][0], &s_b[0][0], &s_c[0][0],
                                                              &s_sum[0][per][0][ch], list, ch, n0, live_states, left, part_bc + row0 * bc_step, bc_step);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    q[i] = again.q.v[i];
                    ta[i] = again.ta.v[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) da[i] = add2(da[i], ta[i]);           // a tile's sum first: shorter chains of roundings
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int r = er + i * kStep;
            if (r < left && col_live) {
                float dx[VEC], ddt[VEC], dz[VEC], y[VEC], dl[VEC], du[VEC];
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    y[v] = skip[v] * ex[i][v];
                    dl[v] = du[v] = 0.0f;
                }
                scan_sum<kPer, kRows * kCh, VEC>(&s_sum[1][0][r][cc], dl);
                scan_sum<kPer, kRows * kCh, VEC>(&s_sum[2][0][r][cc], du);
                if (z) scan_sum<kPer, kRows * kCh, VEC>(&s_sum[0][0][r][cc], y);
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    dx[v] = fmaf(du[v], ed[i][v], skip[v] * eg[i][v]);
                    ddt[v] = fmaf(dl[v], 0.6931471805599453f, du[v] * ex[i][v]) * eds[i][v];      // a holds A log2(e)
                    if (z) dz[v] = eo[i][v] * y[v] * ezs[i][v] * fmaf(ez[i][v], 1.0f - ezs[i][v], 1.0f);
                    sum_d[v] = fmaf(eg[i][v], ex[i][v], sum_d[v]);
                    sum_bias[v] += ddt[v];
                }
                const long long row = seq.first + row0 + r, col = at.c0 + cc;
                seq_store<T, VEC>(static_cast<T*>(p.dx) + row * p.ld_dx + col, dx);
                seq_store<T, VEC>(static_cast<T*>(p.ddt) + row * p.ld_ddt + col, ddt);
                if (z) seq_store<T, VEC>(static_cast<T*>(p.dz) + row * p.ld_dz + col, dz);
            }
        }
    }
    if (live) {
        scan_store_states(p.part_a + scan_state_at<N>(at.number, p.channels, c, n0), da);
        if (p.dstate_in && slot >= 0 && at.chunk == 0) scan_write_state(p, p.dstate_in, slot, c, n0, q);
    }
    __syncthreads();
    // per channel, the sums of the kStep threads that shared it
    float* sums = &s_sum[0][0][0][0];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        sums[er * kCh + cc + v] = sum_d[v];
        sums[kStep * kCh + er * kCh + cc + v] = sum_bias[v];
    }
    __syncthreads();
    if (tid < at.live) {
        float d = 0.0f, v = 0.0f;
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            d += sums[k * kCh + tid];
            v += sums[kStep * kCh + k * kCh + tid];
        }
        const long long row = 2 * at.number * p.channels + at.c0 + tid;
        p.part_d[row] = d;
        p.part_d[row + p.channels] = v;
    }
}

// Joins the blocks' sums: dB and dC over the channel tiles of a group (one thread per four states), dA, dD and ddt_bias over
// all chunks (32 elements per block, eight interleaved partial orders joined in a fixed order).
template <typename T>
__global__ void __launch_bounds__(256) scan_bwd_join_kernel(const __grid_constant__ ScanParams p, int states_pad, long long bc_blocks, long long a_blocks,
                                                            long long numbers) {
    __shared__ float sums[8][33];
    seq_grid_wait();
    if (blockIdx.x < bc_blocks) {
        const long long per_row = static_cast<long long>(p.groups) * 2 * states_pad;
        const long long e = (blockIdx.x * 256LL + threadIdx.x) * 4, total = p.rows * per_row;
        if (e >= total) return;
        const long long row = e / per_row;
        // rows outside every sequence, and those of a sequence that was skipped, have no sums
        if (p.offsets != nullptr && !seq_has_row(p.offsets, p.batch, p.max_len, p.rows, row)) return;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < p.sum_tiles; ++k) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p.part_bc + k * total + e));
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const int in_row = static_cast<int>(e - row * per_row), n = in_row % states_pad, which = (in_row / states_pad) & 1,
                  group = in_row / (2 * states_pad);
        T* out = which ? static_cast<T*>(p.dC) + row * p.ld_dc : static_cast<T*>(p.dB) + row * p.ld_db;
        const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.states) out[group * p.states + n + i] = seq_from_float<T>(v[i]);
        return;
    }
    const long long blk = blockIdx.x - bc_blocks;
    const bool is_a = blk < a_blocks;
    const long long elems = is_a ? p.channels * states_pad : 2 * p.channels;
    const float* part = is_a ? p.part_a : p.part_d;
    const int lane = threadIdx.x & 31, order = threadIdx.x >> 5;
    const long long e = (is_a ? blk : blk - a_blocks) * 32 + lane, count = numbers;
    float s = 0.0f;
    if (e < elems)
        for (long long i = order; i < count; i += 8) s += __ldg(part + i * elems + e);
    sums[order][lane] = s;
    __syncthreads();
    if (order != 0 || e >= elems) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) s += sums[k][lane];
    if (is_a) {
        // [four states][channel][4], see scan_state_at
        const long long quad = e / (4 * p.channels), c = (e - quad * 4 * p.channels) / 4;
        const int n = static_cast<int>(quad * 4 + e % 4);
        if (n < p.states) p.dA[c * p.states + n] = s;
    } else if (e < p.channels) {
        if (p.dD) p.dD[e] = s;
    } else if (p.ddt_bias) {
        p.ddt_bias[e - p.channels] = s;
    }
}

// One new row for each of a batch of sequences.  A warp takes 32 channels of batch rows in turn (blockIdx.y, + gridDim.y, ...), with A
// in registers: a lane does the elementwise work of one channel, then the warp goes through the states in PER rounds of 32 / PER
// channels, four states (16 bytes) a lane.  Bound by reading and writing the states.  A thread writes only the states that it
// read, so state_out may be state_in.  A batch row without a slot is padding: out = 0.
template <typename T, int PER, bool VEC4>
__global__ void __launch_bounds__(128) scan_step_kernel(const __grid_constant__ ScanParams p) {
    constexpr int kCh = 32 / PER;                          // channels of a round
    constexpr int kHeld = PER <= 8 ? PER : 1;              // rounds whose A is held
    seq_launch_dependents();
    const int lane = threadIdx.x & 31, sub = lane / PER, n0 = (lane % PER) * 4;
    const long long tile = blockIdx.x * 4LL + (threadIdx.x >> 5), c0 = tile * 32, mine = c0 + lane;
    if (tile >= p.channel_tiles) return;
    const bool live = mine < p.channels;
    const int group0 = static_cast<int>(c0 / p.group_channels);
    const bool one_group = min(c0 + 31, p.channels - 1) / p.group_channels == group0;
    seq_grid_wait();
    float a[kHeld][4];
    auto load_a = [&](long long c, float (&v)[4]) {
        if (VEC4) {
            const float4 q = c < p.channels ? __ldg(reinterpret_cast<const float4*>(p.A + c * p.states + n0)) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[0] = q.x * kLog2e; v[1] = q.y * kLog2e; v[2] = q.z * kLog2e; v[3] = q.w * kLog2e;
        } else {
            scan_load_a(p, c, n0, c < p.channels, v);
        }
    };
    if (PER <= 8) {
#pragma unroll
        for (int round = 0; round < kHeld; ++round) load_a(c0 + round * kCh + sub, a[round]);
    }
    const float bias = p.dt_bias && live ? __ldg(p.dt_bias + mine) : 0.0f, skip = p.D && live ? __ldg(p.D + mine) : 0.0f;
    for (long long b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const long long slot = state_slot(p.slots, b, p.n_slots, p.status);
        T* out = static_cast<T*>(p.out) + b * p.ld_out + mine;
        if (slot < 0) {
            if (live) *out = seq_from_float<T>(0.0f);
            continue;
        }
        float xv = 0.0f, d = 0.0f, gate = 1.0f;
        if (live) {
            xv = seq_to_float(static_cast<const T*>(p.x)[b * p.ld_x + mine]);
            d = seq_to_float(static_cast<const T*>(p.dt)[b * p.ld_dt + mine]) + bias;
            if (p.z) gate = seq_to_float(static_cast<const T*>(p.z)[b * p.ld_z + mine]);
        }
        // B and C of a lane's states: the same in every round, unless the warp's channels lie in several groups
        float bv[4] = {0.f, 0.f, 0.f, 0.f}, cv[4] = {0.f, 0.f, 0.f, 0.f};
        auto load_bc = [&](long long group) {
            const T* B = static_cast<const T*>(p.B) + b * p.ld_b + group * p.states + n0;
            const T* C = static_cast<const T*>(p.C) + b * p.ld_c + group * p.states + n0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (VEC4 || n0 + i < p.states) {
                    bv[i] = seq_to_float(__ldg(B + i));
                    cv[i] = seq_to_float(__ldg(C + i));
                }
            }
        };
        load_bc(group0);
        const float* from = p.state_in + slot * p.state_stride + n0;
        float* to = p.state_out + slot * p.state_stride + n0;
        auto load_h = [&](long long c, float (&h)[4]) {
            if (c >= p.channels) return;
            if (VEC4) {
                const float4 q = *reinterpret_cast<const float4*>(from + c * p.states);
                h[0] = q.x; h[1] = q.y; h[2] = q.z; h[3] = q.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + i < p.states) h[i] = from[c * p.states + i];
            }
        };
        float held[kHeld][4];
        if (PER <= 8) {                                     // all states are in flight before the first is used
#pragma unroll
            for (int round = 0; round < kHeld; ++round) {
#pragma unroll
                for (int i = 0; i < 4; ++i) held[round][i] = 0.0f;
                load_h(c0 + round * kCh + sub, held[round]);
            }
        }
        if (p.softplus) d = softplus_f<T>(d);
        if (p.z) gate *= sigmoid_f<T>(gate);
        const float u = d * xv;
        float y = skip * xv;
#pragma unroll
        for (int round = 0; round < PER; ++round) {
            const int src = round * kCh + sub;
            const long long c = c0 + src;
            float (&h)[4] = held[PER <= 8 ? round : 0];
            float (&aa)[4] = a[PER <= 8 ? round : 0];
            if (PER > 8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = 0.0f;
                load_h(c, h);
                load_a(c, aa);
            }
            const float dd = __shfl_sync(0xffffffffu, d, src), uu = __shfl_sync(0xffffffffu, u, src);
            if (!one_group && c < p.channels) load_bc(c / p.group_channels);
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = fmaf(fast_exp2(fmaf(dd, aa[i], kDecayAddend)), h[i], uu * bv[i]);
                if (VEC4 || n0 + i < p.states) part = fmaf(h[i], cv[i], part);      // 0 * infinity is not a number
            }
            if (c < p.channels) {
                if (VEC4) {
                    *reinterpret_cast<float4*>(to + c * p.states) = make_float4(h[0], h[1], h[2], h[3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n0 + i < p.states) to[c * p.states + i] = h[i];
                }
            }
#pragma unroll
            for (int m = 1; m < PER; m *= 2) part += __shfl_xor_sync(0xffffffffu, part, m);
            const float got = __shfl_sync(0xffffffffu, part, (lane % kCh) * PER);
            if (lane / kCh == round) y += got;
        }
        if (live) *out = seq_from_float<T>(y * gate);
    }
}

}  // namespace tdx
