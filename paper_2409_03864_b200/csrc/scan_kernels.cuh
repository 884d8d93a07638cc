// Selective state-space scan, channels last.  With dt' = softplus(dt + dt_bias) (or dt + dt_bias), for every channel d and
// state n (B and C are shared by the channels of a group):
//
//   h[t] = exp(dt'[t, d] A[d, n]) h[t - 1] + dt'[t, d] x[t, d] B[t, n]
//   y[t, d] = sum_n C[t, n] h[t, d, n] + D[d] x[t, d],   out = y * silu(z)  (or y)
//
// A thread keeps four states of one channel in registers, TPC threads hold a channel's states (up to 4 * TPC; the rest are
// zero), and a block of 128 threads walks 128 / TPC channels of one group through a sequence, or through one chunk of it, in
// tiles of a few dozen rows: the elementwise work of a tile is spread over all threads and goes through shared memory.
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
    float* saved;                    // [saved_rows][channels][4 * TPC]: the state before every kScanSave-th row
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
    float* carry;                    // [chunk number][channels][4 * TPC]: a chunk's own contribution to the state behind it
    float* carry_dt;                 // [chunk number][channels]: the sum of dt' over a chunk
    float* part_bc;                  // [channel_tiles][rows][groups][2][4 * TPC]
    float* part_a;                   // [chunk number][channels][4 * TPC]
    float* part_d;                   // [chunk number][2][channels]: dD, ddt_bias
    int* status;
};

constexpr int kScanSave = 8;         // rows between two saved states; also the rows of a backward tile
constexpr int kScanThreads = 128;

template <int TPC>
struct ScanShape {
    static constexpr int kChannels = kScanThreads / TPC;
    static constexpr int kStates = 4 * TPC;
    static constexpr int kRows = TPC == 1 ? 8 : TPC == 2 ? 16 : TPC <= 8 ? 32 : TPC == 16 ? 16 : 8;   // rows of a forward tile
};

// Where a block works: channels [c0, c0 + live) of group g, rows [t0, t1) of sequence b.
struct ScanPlace {
    long long b, c0, number;     // number: of the chunk, over all sequences
    int chunk, group, live, tile;
};
template <int TPC>
__device__ __forceinline__ ScanPlace scan_place(const ScanParams& p) {
    ScanPlace r;
    const long long bid = blockIdx.x;
    const int per_chunk = p.channel_tiles * p.groups;
    r.number = bid / per_chunk;
    const int ct = static_cast<int>(bid - r.number * per_chunk);
    const SeqPiece piece = seq_piece(p.offsets, p.batch, p.dense, p.chunk, r.number);
    r.b = piece.b;
    r.chunk = piece.index;
    r.group = ct / p.channel_tiles;
    r.tile = ct - r.group * p.channel_tiles;
    const int in_group = r.tile * ScanShape<TPC>::kChannels;
    r.c0 = static_cast<long long>(r.group) * p.group_channels + in_group;
    r.live = min(ScanShape<TPC>::kChannels, p.group_channels - in_group);
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

enum ScanMode { kScanFull = 0, kScanState = 1, kScanAdjoint = 2 };

// kScanFull: the forward pass over a chunk, from the state before it.
// kScanState: only the state that a chunk adds to what comes before it, h from h = 0, and the sum of dt'.  (The chunk's
//   effect on an incoming state is then exp(A * sum dt').)  Run first when a sequence is cut into chunks, for all chunks but
//   the last; chunk 0 starts from the caller's state.
// kScanAdjoint: the same for the gradient, from the last row to the first: q <- exp(dt' A) (q + C dy).
template <typename T, int TPC, int MODE>
__global__ void __launch_bounds__(kScanThreads) scan_fwd_kernel(const __grid_constant__ ScanParams p) {
    typedef ScanShape<TPC> S;
    constexpr int kRows = S::kRows, kCh = S::kChannels, kN = S::kStates;
    constexpr int kEl = (kRows * kCh + kScanThreads - 1) / kScanThreads;       // elements of a tile per thread
    constexpr int kBc = (kRows * kN + kScanThreads - 1) / kScanThreads;
    __shared__ float2 s_dt[kRows][kCh];                  // dt', dt' x   (kScanAdjoint: dt', dy)
    __shared__ __align__(16) float s_b[kRows][kN];
    __shared__ __align__(16) float s_c[kRows][kN];
    __shared__ __align__(16) float s_y[MODE == kScanFull ? kRows : 1][kScanThreads];
    seq_launch_dependents();
    seq_grid_wait();
    const ScanPlace at = scan_place<TPC>(p);
    const SeqRange seq = seq_range(p.offsets, at.b, p.max_len, p.rows, p.status);
    const int tid = threadIdx.x;
    const int chunk = static_cast<int>(p.chunk), last = seq.len > 0 ? (seq.len - 1) / chunk : 0;
    const int t0 = min(at.chunk, last + 1) * chunk, t1 = min(seq.len, t0 + chunk);
    if (MODE == kScanFull && t0 >= seq.len && at.chunk > 0) return;
    if (MODE == kScanState && t1 >= seq.len && at.chunk > 0) return;
    if (MODE == kScanAdjoint && (t0 >= seq.len || at.chunk == 0)) return;
    const int ch = tid / TPC, n0 = (tid % TPC) * 4;
    const bool live = ch < at.live;
    const long long c = at.c0 + (live ? ch : 0);
    const long long slot = MODE != kScanAdjoint && (p.state_in || p.state_out) ? state_slot(p.slots, at.b, p.n_slots, p.status) : -1;
    float a[4], h[4] = {0.f, 0.f, 0.f, 0.f};
    scan_load_a(p, c, n0, live, a);
    const long long carry_row = at.number * p.channels + c;
    // The state before chunk 0.  When a sequence is cut, the first launch keeps a copy of it where the last chunk's sum would
    // stand (which nobody needs): in the second launch the last chunk may write state_out over state_in before chunk 0 reads it.
    if (MODE != kScanAdjoint && at.chunk == 0 && p.state_in && slot >= 0 && live) {
        const long long kept = ((at.number + last) * p.channels + c) * kN + n0;
        if (MODE == kScanFull && p.cut) {
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = p.carry[kept + i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < p.states) h[i] = p.state_in[slot * p.state_stride + c * p.states + n0 + i];
            if (MODE == kScanState) *reinterpret_cast<float4*>(p.carry + kept) = make_float4(h[0], h[1], h[2], h[3]);
        }
    }
    if (MODE == kScanState && t1 >= seq.len) return;
    if (MODE == kScanFull && at.chunk > 0 && live) {
        for (int k = 0; k < at.chunk; ++k) {
            const long long row = (at.number - at.chunk + k) * p.channels + c;
            const float4 add = *reinterpret_cast<const float4*>(p.carry + row * kN + n0);
            const float sum = k == 0 ? 0.0f : p.carry_dt[row];
            h[0] = fmaf(h[0], fast_exp2(a[0] * sum), add.x);
            h[1] = fmaf(h[1], fast_exp2(a[1] * sum), add.y);
            h[2] = fmaf(h[2], fast_exp2(a[2] * sum), add.z);
            h[3] = fmaf(h[3], fast_exp2(a[3] * sum), add.w);
        }
    }
    f32x2 h01 = pack2(h[0], h[1]), h23 = pack2(h[2], h[3]);
    const f32x2 a01 = pack2(a[0], a[1]), a23 = pack2(a[2], a[3]);

    const T* x = static_cast<const T*>(MODE == kScanAdjoint ? p.dout : p.x) + seq.first * (MODE == kScanAdjoint ? p.ld_dout : p.ld_x) + at.c0;
    const long long ld_x = MODE == kScanAdjoint ? p.ld_dout : p.ld_x;
    const T* dt = static_cast<const T*>(p.dt) + seq.first * p.ld_dt + at.c0;
    const bool gated = p.z != nullptr && MODE != kScanState;
    const T* z = gated ? static_cast<const T*>(p.z) + seq.first * p.ld_z + at.c0 : nullptr;
    const T* B = static_cast<const T*>(MODE == kScanAdjoint ? p.C : p.B) + seq.first * (MODE == kScanAdjoint ? p.ld_c : p.ld_b) + at.group * p.states;
    const long long ld_b = MODE == kScanAdjoint ? p.ld_c : p.ld_b;
    const T* C = static_cast<const T*>(p.C) + seq.first * p.ld_c + at.group * p.states;

    T rx[kEl], rdt[kEl], rz[kEl], rb[kBc], rc[kBc];
    auto fetch = [&](int row0) {
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh, t = row0 + r;
            if (r < kRows && t >= t0 && t < t1 && cc < at.live) {
                rx[i] = x[t * ld_x + cc];
                rdt[i] = dt[t * p.ld_dt + cc];
                if (gated) rz[i] = z[t * p.ld_z + cc];
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int e = tid + i * kScanThreads, r = e / kN, n = e % kN, t = row0 + r;
            if (r < kRows && t >= t0 && t < t1 && n < p.states) {
                rb[i] = B[t * ld_b + n];
                if (MODE == kScanFull) rc[i] = C[t * p.ld_c + n];
            }
        }
    };

    // every element of a thread belongs to the same channel where 128 is a multiple of the tile's channels
    float bias[kEl], skip[kEl];
#pragma unroll
    for (int i = 0; i < kEl; ++i) {
        const int cc = (tid + i * kScanThreads) % kCh;
        bias[i] = p.dt_bias && cc < at.live ? __ldg(p.dt_bias + at.c0 + cc) : 0.0f;
        skip[i] = MODE == kScanFull && p.D && cc < at.live ? __ldg(p.D + at.c0 + cc) : 0.0f;
    }
    float sum_dt = 0.0f;
    const int tiles = (t1 - t0 + kRows - 1) / kRows;
    constexpr bool kBack = MODE == kScanAdjoint;
    if (tiles > 0) fetch(t0 + (kBack ? tiles - 1 : 0) * kRows);
    for (int tile = 0; tile < tiles; ++tile) {
        const int row0 = t0 + (kBack ? tiles - 1 - tile : tile) * kRows;
        float ex[kEl], ez[kEl];
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh;
            const bool there = r < kRows && row0 + r < t1 && cc < at.live;
            float d = 0.0f, v = 0.0f;
            ex[i] = 0.0f;
            ez[i] = 1.0f;
            if (there) {
                d = seq_to_float(rdt[i]) + bias[i];
                if (p.softplus) d = softplus_f(d);
                ex[i] = seq_to_float(rx[i]);
                if (gated) {
                    const float zz = seq_to_float(rz[i]);
                    ez[i] = zz * sigmoid_f(zz);
                }
                v = MODE == kScanAdjoint ? ex[i] * ez[i] : d * ex[i];
            }
            if (r < kRows) s_dt[r][cc] = make_float2(d, v);
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int e = tid + i * kScanThreads, r = e / kN, n = e % kN;
            const bool there = row0 + r < t1 && n < p.states;
            if (r < kRows) {
                s_b[r][n] = there ? seq_to_float(rb[i]) : 0.0f;
                if (MODE == kScanFull) s_c[r][n] = there ? seq_to_float(rc[i]) : 0.0f;
            }
        }
        __syncthreads();
        if (tile + 1 < tiles) fetch(t0 + (kBack ? tiles - 2 - tile : tile + 1) * kRows);
#pragma unroll 8
        for (int k = 0; k < kRows; ++k) {
            const int r = kBack ? kRows - 1 - k : k;
            if (MODE == kScanFull && r % kScanSave == 0) {
                if (p.saved != nullptr && row0 + r < t1 && live) {
                    float4 keep;
                    unpack2(h01, keep.x, keep.y);
                    unpack2(h23, keep.z, keep.w);
                    *reinterpret_cast<float4*>(p.saved + ((saved_base(p, at.b, seq.first) + (row0 + r) / kScanSave) * p.channels + c) * kN + n0) = keep;
                }
            }
            const float2 dv = s_dt[r][ch];
            const ulonglong2 bb = *reinterpret_cast<const ulonglong2*>(&s_b[r][n0]);
            const f32x2 d2 = pack2(dv.x, dv.x), v2 = pack2(dv.y, dv.y);
            float e0, e1, e2, e3;
            unpack2(mul2(d2, a01), e0, e1);
            unpack2(mul2(d2, a23), e2, e3);
            const f32x2 w01 = pack2(fast_exp2(e0), fast_exp2(e1)), w23 = pack2(fast_exp2(e2), fast_exp2(e3));
            if (kBack) {
                h01 = mul2(w01, fma2(v2, bb.x, h01));
                h23 = mul2(w23, fma2(v2, bb.y, h23));
            } else {
                h01 = fma2(w01, h01, mul2(v2, bb.x));
                h23 = fma2(w23, h23, mul2(v2, bb.y));
            }
            if (MODE == kScanFull) {
                const ulonglong2 cc = *reinterpret_cast<const ulonglong2*>(&s_c[r][n0]);
                float lo, hi;
                unpack2(fma2(h23, cc.y, mul2(h01, cc.x)), lo, hi);
                s_y[r][tid] = lo + hi;
            } else {
                sum_dt += dv.x;
            }
        }
        __syncthreads();
        if (MODE == kScanFull) {
            T* out = static_cast<T*>(p.out) + (seq.first + row0) * p.ld_out + at.c0;
#pragma unroll
            for (int i = 0; i < kEl; ++i) {
                const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh;
                if (r < kRows && row0 + r < t1 && cc < at.live) {
                    const float y = sum_row<TPC>(&s_y[r][cc * TPC], skip[i] * ex[i]);
                    out[r * p.ld_out + cc] = seq_from_float<T>(y * ez[i]);
                }
            }
        }
    }
    unpack2(h01, h[0], h[1]);
    unpack2(h23, h[2], h[3]);
    if (MODE != kScanFull) {
        if (live) {
            *reinterpret_cast<float4*>(p.carry + carry_row * kN + n0) = make_float4(h[0], h[1], h[2], h[3]);
            if (n0 == 0) p.carry_dt[carry_row] = sum_dt;
        }
    } else if (p.state_out && slot >= 0 && live && t1 >= seq.len) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < p.states) p.state_out[slot * p.state_stride + c * p.states + n0 + i] = h[i];
    }
}

// Backward.  With g = dout * silu(z) (or dout), for one channel and state
//   dh[t] = C[t] g[t] + a[t + 1] dh[t + 1],   a[t] = exp(dt'[t] A)
//   dC[t] = sum_d g h,   dB[t] = sum_d dh dt' x,   dlog = dh a h[t - 1],   dA = sum_t dlog dt'
//   dx = dt' sum_n dh B + D g,   ddt' = sum_n dlog A + x sum_n dh B,   dz = dout y silu'(z),   dD = sum_t g x.
// A block walks its chunk from the last tile of kScanSave rows to the first.  For each it starts from the saved state in
// front of the tile, recomputes the tile's states and decays into registers, and then goes back through them.  Sums over
// states and over the block's channels go through shared memory; sums over blocks are left to scan_bwd_join_kernel, so every
// sum has a fixed order.
template <int TPC>
struct ScanBwdSmem {
    float4 red[2 * kScanSave][kScanThreads];      // per thread: its channel's share of dB and dC
    float sum[3][kScanSave][kScanThreads];        // per thread: its states' share of y, sum dlog A2, sum dh B
    float b[kScanSave][ScanShape<TPC>::kStates];
    float c[kScanSave][ScanShape<TPC>::kStates];
    float2 dt[kScanSave][ScanShape<TPC>::kChannels];   // dt', dt' x
    float g[kScanSave][ScanShape<TPC>::kChannels];
};
template <typename T, int TPC>
__global__ void __launch_bounds__(kScanThreads) scan_bwd_kernel(const __grid_constant__ ScanParams p) {
    typedef ScanShape<TPC> S;
    constexpr int kRows = kScanSave, kCh = S::kChannels, kN = S::kStates;
    constexpr int kEl = (kRows * kCh + kScanThreads - 1) / kScanThreads;
    constexpr int kBc = (kRows * kN + kScanThreads - 1) / kScanThreads;
    extern __shared__ __align__(16) unsigned char scan_bwd_smem[];
    ScanBwdSmem<TPC>& sm = *reinterpret_cast<ScanBwdSmem<TPC>*>(scan_bwd_smem);
    seq_launch_dependents();
    seq_grid_wait();
    const ScanPlace at = scan_place<TPC>(p);
    const SeqRange seq = seq_range(p.offsets, at.b, p.max_len, p.rows, p.status);
    const int tid = threadIdx.x;
    const int chunk = static_cast<int>(p.chunk), last = seq.len > 0 ? (seq.len - 1) / chunk : 0;
    const int t0 = min(at.chunk, last + 1) * chunk, t1 = min(seq.len, t0 + chunk);
    const int ch = tid / TPC, n0 = (tid % TPC) * 4;
    const bool live = ch < at.live;
    const long long c = at.c0 + (live ? ch : 0);
    const long long slot = p.dstate_in || p.dstate_out ? state_slot(p.slots, at.b, p.n_slots, p.status) : -1;
    float a[4], h[4];
    scan_load_a(p, c, n0, live, a);
    // the gradient that comes from behind the chunk
    float q[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.dstate_out && slot >= 0 && live) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < p.states) q[i] = __ldg(p.dstate_out + slot * p.state_stride + c * p.states + n0 + i);
    }
    if (live) {
        for (int k = last; k > at.chunk; --k) {
            const long long row = (at.number - at.chunk + k) * p.channels + c;
            const float4 add = *reinterpret_cast<const float4*>(p.carry + row * kN + n0);
            const float sum = p.carry_dt[row];
            q[0] = fmaf(q[0], fast_exp2(a[0] * sum), add.x);
            q[1] = fmaf(q[1], fast_exp2(a[1] * sum), add.y);
            q[2] = fmaf(q[2], fast_exp2(a[2] * sum), add.z);
            q[3] = fmaf(q[3], fast_exp2(a[3] * sum), add.w);
        }
    }
    f32x2 q01 = pack2(q[0], q[1]), q23 = pack2(q[2], q[3]);
    const f32x2 a01 = pack2(a[0], a[1]), a23 = pack2(a[2], a[3]);
    f32x2 da01 = pack2(0.f, 0.f), da23 = pack2(0.f, 0.f);

    const T* x = static_cast<const T*>(p.x) + seq.first * p.ld_x + at.c0;
    const T* dt = static_cast<const T*>(p.dt) + seq.first * p.ld_dt + at.c0;
    const T* z = p.z ? static_cast<const T*>(p.z) + seq.first * p.ld_z + at.c0 : nullptr;
    const T* dout = static_cast<const T*>(p.dout) + seq.first * p.ld_dout + at.c0;
    const T* B = static_cast<const T*>(p.B) + seq.first * p.ld_b + at.group * p.states;
    const T* C = static_cast<const T*>(p.C) + seq.first * p.ld_c + at.group * p.states;
    const float* saved = p.saved + (saved_base(p, at.b, seq.first) * p.channels + c) * kN + n0;

    T rx[kEl], rdt[kEl], rz[kEl], rg[kEl], rb[kBc], rc[kBc];
    float4 rh;
    auto fetch = [&](int row0) {
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh, t = row0 + r;
            if (r < kRows && t < t1 && cc < at.live) {
                rx[i] = x[t * p.ld_x + cc];
                rdt[i] = dt[t * p.ld_dt + cc];
                rg[i] = dout[t * p.ld_dout + cc];
                if (z) rz[i] = z[t * p.ld_z + cc];
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int e = tid + i * kScanThreads, r = e / kN, n = e % kN, t = row0 + r;
            if (r < kRows && t < t1 && n < p.states) {
                rb[i] = B[t * p.ld_b + n];
                rc[i] = C[t * p.ld_c + n];
            }
        }
        rh = live ? __ldg(reinterpret_cast<const float4*>(saved + (row0 / kRows) * p.channels * kN)) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    const int my_cc = tid % kCh;                           // the channel of all elements of this thread
    const bool my_live = my_cc < at.live;
    const float bias = p.dt_bias && my_live ? __ldg(p.dt_bias + at.c0 + my_cc) : 0.0f;
    const float skip = p.D && my_live ? __ldg(p.D + at.c0 + my_cc) : 0.0f;
    float sum_d = 0.0f, sum_bias = 0.0f;

    const int tiles = (max(t1 - t0, 0) + kRows - 1) / kRows;
    if (tiles > 0) fetch(t0 + (tiles - 1) * kRows);
    for (int tile = tiles - 1; tile >= 0; --tile) {
        const int row0 = t0 + tile * kRows;
        float ex[kEl], ed[kEl], eds[kEl], ez[kEl], ezs[kEl], eo[kEl];   // x, dt', d dt' / d dt, z, sigmoid(z), dout
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh;
            const bool there = r < kRows && row0 + r < t1 && cc < at.live;
            ex[i] = ed[i] = ez[i] = ezs[i] = eo[i] = 0.0f;
            eds[i] = 1.0f;
            float g = 0.0f;
            if (there) {
                ed[i] = seq_to_float(rdt[i]) + bias;
                if (p.softplus) ed[i] = softplus_grad_f(ed[i], eds[i]);
                ex[i] = seq_to_float(rx[i]);
                eo[i] = g = seq_to_float(rg[i]);
                if (z) {
                    ez[i] = seq_to_float(rz[i]);
                    ezs[i] = sigmoid_f(ez[i]);
                    g *= ez[i] * ezs[i];
                }
            }
            if (r < kRows) {
                sm.dt[r][cc] = make_float2(ed[i], ed[i] * ex[i]);
                sm.g[r][cc] = g;
            }
        }
#pragma unroll
        for (int i = 0; i < kBc; ++i) {
            const int e = tid + i * kScanThreads, r = e / kN, n = e % kN;
            const bool there = row0 + r < t1 && n < p.states;
            if (r < kRows) {
                sm.b[r][n] = there ? seq_to_float(rb[i]) : 0.0f;
                sm.c[r][n] = there ? seq_to_float(rc[i]) : 0.0f;
            }
        }
        f32x2 hs01[kRows + 1], hs23[kRows + 1], w01[kRows], w23[kRows];
        hs01[0] = pack2(rh.x, rh.y);
        hs23[0] = pack2(rh.z, rh.w);
        __syncthreads();
        if (tile > 0) fetch(row0 - kRows);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float2 dv = sm.dt[r][ch];
            const ulonglong2 bb = *reinterpret_cast<const ulonglong2*>(&sm.b[r][n0]);
            const f32x2 d2 = pack2(dv.x, dv.x), v2 = pack2(dv.y, dv.y);
            float e0, e1, e2, e3;
            unpack2(mul2(d2, a01), e0, e1);
            unpack2(mul2(d2, a23), e2, e3);
            w01[r] = pack2(fast_exp2(e0), fast_exp2(e1));
            w23[r] = pack2(fast_exp2(e2), fast_exp2(e3));
            hs01[r + 1] = fma2(w01[r], hs01[r], mul2(v2, bb.x));
            hs23[r + 1] = fma2(w23[r], hs23[r], mul2(v2, bb.y));
        }
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r) {
            const float2 dv = sm.dt[r][ch];
            const float g = sm.g[r][ch];
            const ulonglong2 bb = *reinterpret_cast<const ulonglong2*>(&sm.b[r][n0]);
            const ulonglong2 cc = *reinterpret_cast<const ulonglong2*>(&sm.c[r][n0]);
            const f32x2 d2 = pack2(dv.x, dv.x), v2 = pack2(dv.y, dv.y), g2 = pack2(g, g);
            float lo, hi;
            unpack2(fma2(hs23[r + 1], cc.y, mul2(hs01[r + 1], cc.x)), lo, hi);
            sm.sum[0][r][tid] = lo + hi;
            const f32x2 dh01 = fma2(g2, cc.x, q01), dh23 = fma2(g2, cc.y, q23);
            unpack2(fma2(dh23, bb.y, mul2(dh01, bb.x)), lo, hi);
            sm.sum[2][r][tid] = lo + hi;
            q01 = mul2(w01[r], dh01);
            q23 = mul2(w23[r], dh23);
            const f32x2 l01 = mul2(q01, hs01[r]), l23 = mul2(q23, hs23[r]);
            unpack2(fma2(l23, a23, mul2(l01, a01)), lo, hi);
            sm.sum[1][r][tid] = lo + hi;
            da01 = fma2(l01, d2, da01);
            da23 = fma2(l23, d2, da23);
            ulonglong2 keep;
            keep.x = mul2(dh01, v2);
            keep.y = mul2(dh23, v2);
            *reinterpret_cast<ulonglong2*>(&sm.red[2 * r][tid]) = keep;
            keep.x = mul2(hs01[r + 1], g2);
            keep.y = mul2(hs23[r + 1], g2);
            *reinterpret_cast<ulonglong2*>(&sm.red[2 * r + 1][tid]) = keep;
        }
        __syncthreads();
        // dB and dC of the tile: sums over the block's channels.  kParts neighbouring threads share an output of four states.
        {
            constexpr int kParts = TPC <= 8 ? 8 / TPC : 1, kOut = 2 * kRows * TPC, kPer = kCh / kParts;
#pragma unroll
            for (int o0 = 0; o0 < kOut * kParts; o0 += kScanThreads) {
                const int o = (o0 + tid) / kParts, part = tid % kParts, rw = o / TPC, qq = o % TPC;
                float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const float4 v = sm.red[rw][(part + kParts * i) * TPC + qq];
                    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                }
#pragma unroll
                for (int m = 1; m < kParts; m *= 2) {
                    s.x += __shfl_xor_sync(0xffffffffu, s.x, m);
                    s.y += __shfl_xor_sync(0xffffffffu, s.y, m);
                    s.z += __shfl_xor_sync(0xffffffffu, s.z, m);
                    s.w += __shfl_xor_sync(0xffffffffu, s.w, m);
                }
                const int r = rw >> 1;
                if (part == 0 && row0 + r < t1) {
                    const long long row = static_cast<long long>(at.tile) * p.rows + seq.first + row0 + r;
                    *reinterpret_cast<float4*>(p.part_bc + ((row * p.groups + at.group) * 2 + (rw & 1)) * kN + qq * 4) = s;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kEl; ++i) {
            const int e = tid + i * kScanThreads, r = e / kCh, cc = e % kCh;
            if (r < kRows && row0 + r < t1 && cc < at.live) {
                const float y = sum_row<TPC>(&sm.sum[0][r][cc * TPC], skip * ex[i]);
                const float dlog = sum_row<TPC>(&sm.sum[1][r][cc * TPC], 0.0f), du = sum_row<TPC>(&sm.sum[2][r][cc * TPC], 0.0f);
                const float g = sm.g[r][cc];
                const long long row = seq.first + row0 + r, col = at.c0 + cc;
                static_cast<T*>(p.dx)[row * p.ld_dx + col] = seq_from_float<T>(fmaf(du, ed[i], skip * g));
                float dd = fmaf(dlog, 0.6931471805599453f, du * ex[i]);
                dd *= eds[i];
                static_cast<T*>(p.ddt)[row * p.ld_ddt + col] = seq_from_float<T>(dd);
                if (z) {
                    static_cast<T*>(p.dz)[row * p.ld_dz + col] = seq_from_float<T>(eo[i] * y * ezs[i] * fmaf(ez[i], 1.0f - ezs[i], 1.0f));
                }
                sum_d = fmaf(g, ex[i], sum_d);
                sum_bias += dd;
            }
        }
    }
    const long long part = at.number * p.channels;
    if (live) {
        float v[4];
        unpack2(da01, v[0], v[1]);
        unpack2(da23, v[2], v[3]);
        *reinterpret_cast<float4*>(p.part_a + (part + c) * kN + n0) = make_float4(v[0], v[1], v[2], v[3]);
        unpack2(q01, q[0], q[1]);
        unpack2(q23, q[2], q[3]);
        if (p.dstate_in && slot >= 0 && at.chunk == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < p.states) p.dstate_in[slot * p.state_stride + c * p.states + n0 + i] = q[i];
        }
    }
    __syncthreads();
    sm.sum[0][0][tid] = sum_d;
    sm.sum[1][0][tid] = sum_bias;
    __syncthreads();
    if (tid < kCh && my_live) {
        float d = 0.0f, v = 0.0f;
#pragma unroll
        for (int k = 0; k < TPC; ++k) {
            d += sm.sum[0][0][tid + k * kCh];
            v += sm.sum[1][0][tid + k * kCh];
        }
        const long long row = 2 * part + at.c0 + tid;
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
        // rows outside every sequence have no sums
        if (p.offsets != nullptr && (row < __ldg(p.offsets) || row >= __ldg(p.offsets + p.batch))) return;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < p.channel_tiles; ++k) {
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
        const long long c = e / states_pad;
        const int n = static_cast<int>(e - c * states_pad);
        if (n < p.states) p.dA[c * p.states + n] = s;
    } else if (e < p.channels) {
        if (p.dD) p.dD[e] = s;
    } else if (p.ddt_bias) {
        p.ddt_bias[e - p.channels] = s;
    }
}

// One new row for each of a batch of sequences.  A warp takes 32 channels of one batch row: a lane does the elementwise work
// of one channel, then the warp goes through the states in TPC rounds of 32 / TPC channels, four states (16 bytes) a lane.
// Bound by reading and writing the states.  A thread writes only the states that it read, so state_out may be state_in.  A
// batch row without a slot is padding: out = 0.
template <typename T, int TPC, bool VEC4>
__global__ void __launch_bounds__(128) scan_step_kernel(const __grid_constant__ ScanParams p) {
    constexpr int kPer = 32 / TPC;                         // channels of a round
    seq_launch_dependents();
    seq_grid_wait();
    const int lane = threadIdx.x & 31;
    const long long warp = blockIdx.x * 4LL + (threadIdx.x >> 5);
    const long long b = warp / p.channel_tiles;
    if (b >= p.batch) return;
    const long long c0 = (warp - b * p.channel_tiles) * 32, mine = c0 + lane;
    const bool live = mine < p.channels;
    const long long slot = state_slot(p.slots, b, p.n_slots, p.status);
    float xv = 0.0f, d = 0.0f, gate = 1.0f, y = 0.0f;
    if (live && slot >= 0) {
        xv = seq_to_float(static_cast<const T*>(p.x)[b * p.ld_x + mine]);
        d = seq_to_float(static_cast<const T*>(p.dt)[b * p.ld_dt + mine]) + (p.dt_bias ? __ldg(p.dt_bias + mine) : 0.0f);
        if (p.softplus) d = softplus_f(d);
        if (p.z) {
            const float zz = seq_to_float(static_cast<const T*>(p.z)[b * p.ld_z + mine]);
            gate = zz * sigmoid_f(zz);
        }
        y = p.D ? __ldg(p.D + mine) * xv : 0.0f;
    }
    if (slot >= 0) {
        const float u = d * xv;
        const int sub = lane / TPC, n0 = (lane % TPC) * 4;
#pragma unroll
        for (int round = 0; round < TPC; ++round) {
            const int from = round * kPer + sub;
            const long long c = c0 + from;
            const float dd = __shfl_sync(0xffffffffu, d, from), uu = __shfl_sync(0xffffffffu, u, from);
            float part = 0.0f;
            if (c < p.channels) {
                const long long at = slot * p.state_stride + c * p.states + n0;
                const long long group = c / p.group_channels;
                const T* B = static_cast<const T*>(p.B) + b * p.ld_b + group * p.states + n0;
                const T* C = static_cast<const T*>(p.C) + b * p.ld_c + group * p.states + n0;
                float h[4], av[4];
                if (VEC4) {
                    const float4 hv = *reinterpret_cast<const float4*>(p.state_in + at);
                    const float4 aa = __ldg(reinterpret_cast<const float4*>(p.A + c * p.states + n0));
                    h[0] = hv.x; h[1] = hv.y; h[2] = hv.z; h[3] = hv.w;
                    av[0] = aa.x; av[1] = aa.y; av[2] = aa.z; av[3] = aa.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        h[i] = n0 + i < p.states ? p.state_in[at + i] : 0.0f;
                        av[i] = n0 + i < p.states ? __ldg(p.A + c * p.states + n0 + i) : 0.0f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (VEC4 || n0 + i < p.states) {
                        h[i] = fmaf(fast_exp2(dd * (av[i] * kLog2e)), h[i], uu * seq_to_float(B[i]));
                        part = fmaf(h[i], seq_to_float(C[i]), part);
                    }
                }
                if (VEC4) {
                    *reinterpret_cast<float4*>(p.state_out + at) = make_float4(h[0], h[1], h[2], h[3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n0 + i < p.states) p.state_out[at + i] = h[i];
                }
            }
#pragma unroll
            for (int m = 1; m < TPC; m *= 2) part += __shfl_xor_sync(0xffffffffu, part, m);
            const float got = __shfl_sync(0xffffffffu, part, (lane % kPer) * TPC);
            if (lane / kPer == round) y += got;
        }
    }
    if (live) static_cast<T*>(p.out)[b * p.ld_out + mine] = seq_from_float<T>(slot >= 0 ? y * gate : 0.0f);
}

}  // namespace tdx
