// Norms before and after a block with its gate and residual scale, in one pass over a row and back.
//
//   u = x * rstd_in * weight_in   (rstd_in over a group of channels; or u = x)      a = u * silu(gate)   (or a = u)
//   s = residual + scale * a      (or s = scale * a)                                y = s * rstd_out * weight_out
//
// Bandwidth bounds both directions, so a row is read once: `warps` warps hold it in registers, NV vectors of VEC channels a
// thread, all loads issued before the first use.  Sums over a row go through shuffles and one barrier of the row's own warps;
// sums over groups of channels through shuffles alone where a group is 1, 2, 4, ... 32 vectors, else through shared memory.
// Measured, bf16, rows of 4096: norm and gate of heads of 128, 8192 rows, 37.5 us (201 MB: 5.4 of the 6.6 TB/s that a copy reaches); 4 rows 7 us,
// which is the call itself.
#pragma once
#include "seq_common.cuh"

namespace tdx {

struct NormParams {
    long long rows;
    int channels, group;             // group: channels per norm of x
    int norm_in;
    int warps;                       // warps a row
    int vectors;                     // VEC-wide vectors a row
    int group_lanes;                 // vectors a group where that is a power of two up to 32; 0: the whole row; -1: any other number
    int group_vectors;
    float eps, inv_group, inv_channels;
    const void *x, *gate, *residual;
    long long ld_x, ld_gate, ld_residual;
    const float *weight_in, *scale, *weight_out;
    void *sum, *y;
    long long ld_sum, ld_y;
    const void *dsum, *dy;
    long long ld_dsum, ld_dy;
    void *dx, *dgate, *dresidual;
    long long ld_dx, ld_dgate, ld_dresidual;
    float* partial;                  // backward: per set of rows, three rows of `channels` sums (dweight_in, dscale, dweight_out)
    int want_in, want_scale, want_out;
};

constexpr int kNormThreads = 512;    // at most; 16 channels a thread are then rows of up to 8192
constexpr int kNormShared = 2 * 32;  // two row sums of up to 16 warps, twice

// The threads that share a row, and the sums they take.
struct NormRow {
    int lane, warp, warps, thread, threads, slot;   // thread: within the row; slot: the row's number within the block
    float* sums;                                    // [2][32] of this row
    float* vec;                                     // [vectors] of this row (group_lanes = -1)
    int turn;
    __device__ __forceinline__ void sync() const {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(slot + 1), "r"(threads) : "memory");
    }
    // the sum over the row, in a fixed order; two sets of shared sums take turns, so that one barrier is enough
    __device__ __forceinline__ float row_sum(float v) {
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
        if (warps == 1) return v;
        float* s = sums + turn * 32;
        turn ^= 1;
        if (lane == 0) s[warp] = v;
        sync();
        float t = (lane & 15) < warps ? s[lane & 15] : 0.0f;
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) t += __shfl_xor_sync(0xffffffffu, t, m);
        return t;
    }
    // two sums over the row behind one barrier
    __device__ __forceinline__ void row_sums(float& v, float& w) {
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) {
            v += __shfl_xor_sync(0xffffffffu, v, m);
            w += __shfl_xor_sync(0xffffffffu, w, m);
        }
        if (warps == 1) return;
        float* s = sums + turn * 32;
        turn ^= 1;
        if (lane == 0) *reinterpret_cast<float2*>(s + 2 * warp) = make_float2(v, w);
        sync();
        const float2 t = (lane & 15) < warps ? *reinterpret_cast<const float2*>(s + 2 * (lane & 15)) : make_float2(0.0f, 0.0f);
        v = t.x;
        w = t.y;
#pragma unroll
        for (int m = 8; m > 0; m >>= 1) {
            v += __shfl_xor_sync(0xffffffffu, v, m);
            w += __shfl_xor_sync(0xffffffffu, w, m);
        }
    }
    // v[i]: this thread's part of vector thread + i * threads; becomes the sum over the vector's group
    template <int NV>
    __device__ __forceinline__ void group_sum(const NormParams& p, float (&v)[NV]) {
        if (p.group_lanes == 0) {
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) t += v[i];
            t = row_sum(t);
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = t;
        } else if (p.group_lanes > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                for (int m = p.group_lanes >> 1; m > 0; m >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], m);
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (thread + i * threads < p.vectors) vec[thread + i * threads] = v[i];
            sync();
            for (int g = thread; g * p.group_vectors < p.vectors; g += threads) {
                float t = 0.0f;
                for (int j = 0; j < p.group_vectors; ++j) t += vec[g * p.group_vectors + j];
                vec[g * p.group_vectors] = t;
            }
            sync();
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (thread + i * threads < p.vectors) v[i] = vec[(thread + i * threads) / p.group_vectors * p.group_vectors];
            sync();
        }
    }
};

// Channels are worked on in pairs (one instruction for two), or alone where rows allow no wider access.
template <int VEC> struct NormLanes { typedef f32x2 type; static constexpr int kCount = VEC / 2; };
template <> struct NormLanes<1> { typedef float type; static constexpr int kCount = 1; };
__device__ __forceinline__ f32x2 nmul(f32x2 a, f32x2 b) { return mul2(a, b); }
__device__ __forceinline__ float nmul(float a, float b) { return a * b; }
__device__ __forceinline__ f32x2 nfma(f32x2 a, f32x2 b, f32x2 c) { return fma2(a, b, c); }
__device__ __forceinline__ float nfma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ void nall(float v, f32x2& r) { r = pack2(v, v); }
__device__ __forceinline__ void nall(float v, float& r) { r = v; }
__device__ __forceinline__ float nsum(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}
__device__ __forceinline__ float nsum(float v) { return v; }
template <typename T>
__device__ __forceinline__ f32x2 nsigmoid(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return pack2(sigmoid_f<T>(a), sigmoid_f<T>(b));
}
template <typename T>
__device__ __forceinline__ float nsigmoid(float v) { return sigmoid_f<T>(v); }
template <int VEC, int N>
__device__ __forceinline__ void norm_unpack(const SeqVec<float, VEC>& r, f32x2 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = pack2(r.v[2 * i], r.v[2 * i + 1]);
}
// (through the words: one operation a value, where taking the halves out as bf16 is two)
template <int VEC, int N>
__device__ __forceinline__ void norm_unpack(const SeqVec<__nv_bfloat16, VEC>& r, f32x2 (&f)[N]) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(&r.bits);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = pack2(__uint_as_float(words[i] << 16), __uint_as_float(words[i] & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ void norm_unpack(const SeqVec<T, 1>& r, float (&f)[1]) { f[0] = seq_to_float(r.v[0]); }
template <int VEC, int N>
__device__ __forceinline__ void norm_flat(const f32x2 (&f)[N], float (&r)[VEC]) {
#pragma unroll
    for (int i = 0; i < N; ++i) unpack2(f[i], r[2 * i], r[2 * i + 1]);
}
template <int VEC>
__device__ __forceinline__ void norm_flat(const float (&f)[1], float (&r)[VEC]) { r[0] = f[0]; }
template <int VEC>
__device__ __forceinline__ void norm_param(const float* p, int c, typename NormLanes<VEC>::type (&f)[NormLanes<VEC>::kCount]) {
    constexpr int kN = NormLanes<VEC>::kCount, kStep = VEC >= 4 ? 4 : VEC;
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < kN; ++i) nall(1.0f, f[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < VEC; i += kStep) {
        const SeqVec<float, kStep> part = seq_load<float, kStep>(p + c + i);
        typename NormLanes<kStep>::type g[NormLanes<kStep>::kCount];
        norm_unpack(part, g);
#pragma unroll
        for (int j = 0; j < NormLanes<kStep>::kCount; ++j) f[i / 2 + j] = g[j];
    }
}
// What a call has.  Kernels for the usual combinations know it when they are compiled (HAS >= 0), which saves them the operations of
// what is not there; the others look it up.
enum : int { kNormIn = 1, kNormGate = 2, kNormScale = 4, kNormResidual = 8, kNormY = 16, kNormSum = 32 };
template <int HAS>
__device__ __forceinline__ bool norm_has(int flag, bool looked_up) { return HAS >= 0 ? (HAS & flag) != 0 : looked_up; }
// One vector of every activation that a row has; what it lacks stays zero.
template <typename T, int VEC>
__device__ __forceinline__ SeqVec<T, VEC> norm_load(const void* base, long long ld, long long row, int c, bool there) {
    SeqVec<T, VEC> r;
    if (base != nullptr && there) return seq_load<T, VEC>(static_cast<const T*>(base) + row * ld + c);
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = seq_from_float<T>(0.0f);
    return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void norm_store(void* base, long long ld, long long row, int c, const typename NormLanes<VEC>::type (&f)[NormLanes<VEC>::kCount]) {
    float flat[VEC];
    norm_flat<VEC>(f, flat);
    T* to = static_cast<T*>(base) + row * ld + c;
    if constexpr (sizeof(T) == 2 && VEC > 1) {
        SeqVec<T, VEC> r;
        __nv_bfloat162* pairs = reinterpret_cast<__nv_bfloat162*>(&r.bits);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) pairs[i] = __floats2bfloat162_rn(flat[2 * i], flat[2 * i + 1]);
        *reinterpret_cast<typename SeqVec<T, VEC>::bits_t*>(to) = r.bits;
    } else {
        seq_store<T, VEC>(to, flat);
    }
}
__device__ __forceinline__ NormRow norm_row(const NormParams& p, float* shared) {
    NormRow r;
    const int warp = threadIdx.x >> 5;
    r.lane = threadIdx.x & 31;
    r.warps = p.warps;
    r.slot = warp / p.warps;
    r.warp = warp - r.slot * p.warps;
    r.thread = r.warp * 32 + r.lane;
    r.threads = p.warps * 32;
    r.sums = shared + r.slot * kNormShared;
    r.vec = shared + (blockDim.x >> 5) / p.warps * kNormShared + r.slot * p.vectors;
    r.turn = 0;
    return r;
}

template <typename T, int VEC, int NV, int HAS>
__global__ void __launch_bounds__(kNormThreads, NV * VEC <= 8 ? 2 : 1) norm_fwd_kernel(const __grid_constant__ NormParams p) {
    typedef typename NormLanes<VEC>::type Lane;
    constexpr int N = NormLanes<VEC>::kCount;
    extern __shared__ float norm_shared[];
    NormRow r = norm_row(p, norm_shared);
    const int sets = (blockDim.x >> 5) / p.warps;
    const bool in = norm_has<HAS>(kNormIn, p.norm_in), gate = norm_has<HAS>(kNormGate, p.gate != nullptr), scale = norm_has<HAS>(kNormScale, p.scale != nullptr),
               residual = norm_has<HAS>(kNormResidual, p.residual != nullptr), out = norm_has<HAS>(kNormY, p.y != nullptr), sum = norm_has<HAS>(kNormSum, p.sum != nullptr);
    seq_grid_wait();
    const long long step = static_cast<long long>(gridDim.x) * sets;
    SeqVec<T, VEC> nx[NV], ng[NV], nr[NV];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            const bool there = c < p.channels && row < p.rows;
            nx[i] = norm_load<T, VEC>(p.x, p.ld_x, row, c, there);
            if (gate) ng[i] = norm_load<T, VEC>(p.gate, p.ld_gate, row, c, there);
            if (residual) nr[i] = norm_load<T, VEC>(p.residual, p.ld_residual, row, c, there);
        }
    };
    constexpr bool kAhead = NV * VEC <= 8;                       // wider threads have no registers to spare
    long long row = static_cast<long long>(blockIdx.x) * sets + r.slot;
    if (kAhead) fetch(row);
    for (; row < p.rows; row += step) {
        SeqVec<T, VEC> vg[NV], vr[NV];
        Lane s[NV][N];
        if (!kAhead) fetch(row);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            norm_unpack(nx[i], s[i]);
            vg[i] = ng[i];
            vr[i] = nr[i];
        }
        if (kAhead) fetch(row + step);                           // on its way while this row is worked on
        float rstd[NV];
        if (in) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                Lane square;
                nall(0.0f, square);
#pragma unroll
                for (int j = 0; j < N; ++j) square = nfma(s[i][j], s[i][j], square);
                rstd[i] = nsum(square);
            }
            r.group_sum(p, rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_group, p.eps));
        }
        Lane square;
        nall(0.0f, square);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                if (in) {
                    Lane w[N], rs;
                    nall(rstd[i], rs);
                    norm_param<VEC>(p.weight_in, c, w);
#pragma unroll
                    for (int j = 0; j < N; ++j) s[i][j] = nmul(nmul(s[i][j], rs), w[j]);
                }
                if (gate) {
                    Lane g[N];
                    norm_unpack(vg[i], g);
#pragma unroll
                    for (int j = 0; j < N; ++j) s[i][j] = nmul(s[i][j], nmul(g[j], nsigmoid<T>(g[j])));
                }
                Lane k[N], add[N];
                if (scale) norm_param<VEC>(p.scale, c, k);
                if (residual) norm_unpack(vr[i], add);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    Lane one;
                    nall(1.0f, one);
                    if (scale && !residual) s[i][j] = nmul(k[j], s[i][j]);
                    if (residual) s[i][j] = nfma(scale ? k[j] : one, s[i][j], add[j]);
                    if (out) square = nfma(s[i][j], s[i][j], square);
                }
                if (sum) norm_store<T, VEC>(p.sum, p.ld_sum, row, c, s[i]);
            }
        }
        if (out) {
            Lane rs;
            nall(rsqrtf(fmaf(r.row_sum(nsum(square)), p.inv_channels, p.eps)), rs);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (r.thread + i * r.threads) * VEC;
                if (c < p.channels) {
                    Lane w[N];
                    norm_param<VEC>(p.weight_out, c, w);
#pragma unroll
                    for (int j = 0; j < N; ++j) w[j] = nmul(w[j], nmul(s[i][j], rs));
                    norm_store<T, VEC>(p.y, p.ld_y, row, c, w);
                }
            }
        }
    }
}

// With xh = x rstd_in, sh = s rstd_out, t = dy weight_out:
//   ds = dsum + rstd_out (t - sh mean(t sh)),  dresidual = ds,  da = ds scale,  dgate = da u silu'(gate),  du = da silu(gate),
//   dx = rstd_in (t' - xh mean_group(t' xh)) with t' = du weight_in,
//   dweight_out = sum over rows of dy sh,  dscale = of ds a,  dweight_in = of du xh.
// s is computed again from x, gate and residual, which costs no more bytes than reading it and keeps its 32 bits.  A thread keeps
// its channels' parameter sums in registers over all rows of its set; a second kernel adds the sets in a fixed order.
// Sixteen warps an SM is all that 128 registers leave (8 channels a thread with three sums each and the next row on its way), so
// latency bounds it, at half the issue rate and a third of the memory's.  Everything at once (norm in and out, gate, scale, residual),
// 8192 x 4096 in bf16, forward and backward: 252 us for 873 MB; without the next row's loads 336.
// Wider threads (bf16 rows of more than 4096 channels, fp32 ones of more than 2048) and combinations that no instance knows spill: the
// same bytes take 185 us backwards at 4096 channels, 465 there without dsum, 734, 657 and 641 at 5120, 6144 and 8192; fp32, 4096 x 4096: 474.
template <typename T, int VEC, int NV, int HAS>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const __grid_constant__ NormParams p) {
    typedef typename NormLanes<VEC>::type Lane;
    constexpr int N = NormLanes<VEC>::kCount;
    // with up to 8 channels a thread the registers hold the next row's vectors too
    constexpr bool kAhead = NV * VEC <= 8;
    extern __shared__ float norm_shared[];
    NormRow r = norm_row(p, norm_shared);
    const int sets = (blockDim.x >> 5) / p.warps;
    const long long set = static_cast<long long>(blockIdx.x) * sets + r.slot;
    const bool in = norm_has<HAS>(kNormIn, p.norm_in), gate = norm_has<HAS>(kNormGate, p.gate != nullptr), scale = norm_has<HAS>(kNormScale, p.scale != nullptr),
               residual = norm_has<HAS>(kNormResidual, p.residual != nullptr), out = norm_has<HAS>(kNormY, p.dy != nullptr), sum = norm_has<HAS>(kNormSum, p.dsum != nullptr);
    Lane sum_in[NV][N], sum_scale[NV][N], sum_out[NV][N], zero, one, minus;
    nall(0.0f, zero);
    nall(1.0f, one);
    nall(-1.0f, minus);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) sum_in[i][j] = sum_scale[i][j] = sum_out[i][j] = zero;
    seq_grid_wait();
    const long long step = static_cast<long long>(gridDim.x) * sets;
    SeqVec<T, VEC> vx[NV], vg[NV], vr[NV], vs[NV], vy[NV], nx[NV], ng[NV], nr[NV], ns[NV], ny[NV];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            const bool there = c < p.channels && row < p.rows;
            nx[i] = norm_load<T, VEC>(p.x, p.ld_x, row, c, there);
            if (gate) ng[i] = norm_load<T, VEC>(p.gate, p.ld_gate, row, c, there);
            if (out && residual) nr[i] = norm_load<T, VEC>(p.residual, p.ld_residual, row, c, there);
            if (sum) ns[i] = norm_load<T, VEC>(p.dsum, p.ld_dsum, row, c, there);
            if (out) ny[i] = norm_load<T, VEC>(p.dy, p.ld_dy, row, c, there);
        }
    };
    if (kAhead) fetch(set);
    for (long long row = set; row < p.rows; row += step) {
        if (!kAhead) fetch(row);
#pragma unroll
        for (int i = 0; i < NV; ++i) { vx[i] = nx[i]; vg[i] = ng[i]; vr[i] = nr[i]; vs[i] = ns[i]; vy[i] = ny[i]; }
        if (kAhead) fetch(row + step);
        float rstd[NV];
        if (in) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                Lane x[N], square = zero;
                norm_unpack(vx[i], x);
#pragma unroll
                for (int j = 0; j < N; ++j) square = nfma(x[j], x[j], square);
                rstd[i] = nsum(square);
            }
            r.group_sum(p, rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_group, p.eps));
        }
        // The way forward once more: u, a and, for y's part of ds, the sums of s^2 and t s.
        Lane u[NV][N], sig[NV][N], squares = zero, inners = zero;
        auto gated = [&](int i, int j, Lane g) { return gate ? nmul(u[i][j], nmul(g, sig[i][j])) : u[i][j]; };
        auto total = [&](Lane k, Lane a, Lane add) { return residual ? nfma(scale ? k : one, a, add) : scale ? nmul(k, a) : a; };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                Lane g[N];
                norm_unpack(vx[i], u[i]);
                if (in) {
                    Lane w[N], rs;
                    nall(rstd[i], rs);
                    norm_param<VEC>(p.weight_in, c, w);
#pragma unroll
                    for (int j = 0; j < N; ++j) u[i][j] = nmul(nmul(u[i][j], rs), w[j]);
                }
                if (gate) {
                    norm_unpack(vg[i], g);
#pragma unroll
                    for (int j = 0; j < N; ++j) sig[i][j] = nsigmoid<T>(g[j]);
                }
                if (out) {
                    Lane k[N], add[N], dy[N], wo[N];
                    if (scale) norm_param<VEC>(p.scale, c, k);
                    norm_param<VEC>(p.weight_out, c, wo);
                    if (residual) norm_unpack(vr[i], add);
                    norm_unpack(vy[i], dy);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const Lane s = total(k[j], gated(i, j, g[j]), add[j]);
                        squares = nfma(s, s, squares);
                        inners = nfma(nmul(dy[j], wo[j]), s, inners);
                    }
                }
            }
        }
        Lane rs_out = zero, less = zero;                         // rstd_out, and -mean(t sh)
        if (out) {
            float square = nsum(squares), inner = nsum(inners);
            r.row_sums(square, inner);
            const float rs = rsqrtf(fmaf(square, p.inv_channels, p.eps));
            nall(rs, rs_out);
            nall(-inner * rs * p.inv_channels, less);
        }
        Lane t[NV][N];
        float group[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            group[i] = 0.0f;
            if (c < p.channels) {
                Lane k[N], ds[N], g[N];
                if (scale) norm_param<VEC>(p.scale, c, k);
                if (sum) norm_unpack(vs[i], ds);
                if (gate) norm_unpack(vg[i], g);
                if (out) {
                    Lane add[N], dy[N], wo[N];
                    norm_param<VEC>(p.weight_out, c, wo);
                    if (residual) norm_unpack(vr[i], add);
                    norm_unpack(vy[i], dy);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const Lane sh = nmul(total(k[j], gated(i, j, g[j]), add[j]), rs_out), part = nfma(sh, less, nmul(dy[j], wo[j]));
                        ds[j] = sum ? nfma(rs_out, part, ds[j]) : nmul(rs_out, part);
                        sum_out[i][j] = nfma(dy[j], sh, sum_out[i][j]);
                    }
                }
                if (residual) norm_store<T, VEC>(p.dresidual, p.ld_dresidual, row, c, ds);
                Lane dg[N], groups = zero, w[N], x[N], rs;
                if (in) {
                    nall(rstd[i], rs);
                    norm_param<VEC>(p.weight_in, c, w);
                    norm_unpack(vx[i], x);
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (scale || p.want_scale) sum_scale[i][j] = nfma(ds[j], gated(i, j, g[j]), sum_scale[i][j]);
                    Lane d = scale ? nmul(ds[j], k[j]) : ds[j];
                    if (gate) {
                        // silu' = sig (1 + g (1 - sig))
                        dg[j] = nmul(nmul(d, u[i][j]), nmul(sig[i][j], nfma(g[j], nfma(sig[i][j], minus, one), one)));
                        d = nmul(d, nmul(g[j], sig[i][j]));
                    }
                    t[i][j] = d;
                    if (in) {
                        const Lane xh = nmul(x[j], rs);
                        sum_in[i][j] = nfma(d, xh, sum_in[i][j]);
                        t[i][j] = nmul(d, w[j]);
                        groups = nfma(t[i][j], xh, groups);
                    }
                }
                if (gate) norm_store<T, VEC>(p.dgate, p.ld_dgate, row, c, dg);
                group[i] = nsum(groups);
            }
        }
        if (in) r.group_sum(p, group);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                if (in) {
                    Lane x[N], m, rs;
                    norm_unpack(vx[i], x);
                    nall(-group[i] * p.inv_group * rstd[i], m);
                    nall(rstd[i], rs);
#pragma unroll
                    for (int j = 0; j < N; ++j) t[i][j] = nmul(rs, nfma(x[j], m, t[i][j]));
                }
                norm_store<T, VEC>(p.dx, p.ld_dx, row, c, t[i]);
            }
        }
    }
    float* part = p.partial + set * 3 * p.channels;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (r.thread + i * r.threads) * VEC;
        if (c < p.channels) {
            float flat[3][VEC];
            norm_flat<VEC>(sum_in[i], flat[0]);
            norm_flat<VEC>(sum_scale[i], flat[1]);
            norm_flat<VEC>(sum_out[i], flat[2]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (p.want_in) part[c + j] = flat[0][j];
                if (p.want_scale) part[p.channels + c + j] = flat[1][j];
                if (p.want_out) part[2 * p.channels + c + j] = flat[2][j];
            }
        }
    }
}

// Rows of more than 8192 channels: the same with nothing kept in registers, the row read again for every pass over it (from L2).
template <typename T>
struct NormWide {
    const NormParams& p;
    NormRow r;
    long long row;
    __device__ __forceinline__ float at(const void* base, long long ld, int c) const {
        return base == nullptr ? 0.0f : seq_to_float(static_cast<const T*>(base)[row * ld + c]);
    }
    __device__ __forceinline__ float param(const float* w, int c) const { return w == nullptr ? 1.0f : __ldg(w + c); }
    __device__ __forceinline__ void store(void* base, long long ld, int c, float v) const { static_cast<T*>(base)[row * ld + c] = seq_from_float<T>(v); }
    // rstd_in of channel c's group: the row's, or the group's from shared memory
    __device__ __forceinline__ float rstd(const float* shared, int c) const { return p.norm_in ? shared[c / p.group] : 1.0f; }
    // sums over groups of f(c), taken by one warp a group; `shared` gets scale(sum)
    template <typename F, typename G>
    __device__ __forceinline__ void groups(float* shared, F f, G finish) {
        const int count = p.channels / p.group;
        if (count == 1) {
            float v = 0.0f;
            for (int c = r.thread; c < p.channels; c += r.threads) v += f(c);
            v = r.row_sum(v);
            if (r.thread == 0) shared[0] = finish(v);
        } else {
            for (int g = r.warp; g < count; g += r.warps) {
                float v = 0.0f;
                for (int c = r.lane; c < p.group; c += 32) v += f(g * p.group + c);
#pragma unroll
                for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
                if (r.lane == 0) shared[g] = finish(v);
            }
        }
        r.sync();
    }
    __device__ __forceinline__ float gated(const float* rs, int c) const {
        float u = at(p.x, p.ld_x, c) * rstd(rs, c) * (p.norm_in ? param(p.weight_in, c) : 1.0f);
        if (p.gate != nullptr) {
            const float g = at(p.gate, p.ld_gate, c);
            u *= g * sigmoid_f<T>(g);
        }
        return u;
    }
};
template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_wide_kernel(const __grid_constant__ NormParams p) {
    extern __shared__ float norm_shared[];
    NormWide<T> n{p, norm_row(p, norm_shared), 0};
    float* rs = norm_shared + kNormShared;
    seq_grid_wait();
    for (n.row = blockIdx.x; n.row < p.rows; n.row += gridDim.x) {
        if (p.norm_in)
            n.groups(rs, [&](int c) { const float v = n.at(p.x, p.ld_x, c); return v * v; }, [&](float v) { return rsqrtf(fmaf(v, p.inv_group, p.eps)); });
        auto total = [&](int c) { return fmaf(n.param(p.scale, c), n.gated(rs, c), n.at(p.residual, p.ld_residual, c)); };
        float square = 0.0f, ro = 0.0f;
        if (p.y != nullptr) {
            for (int c = n.r.thread; c < p.channels; c += n.r.threads) {
                const float s = total(c);
                square = fmaf(s, s, square);
            }
            ro = rsqrtf(fmaf(n.r.row_sum(square), p.inv_channels, p.eps));
        }
        for (int c = n.r.thread; c < p.channels; c += n.r.threads) {
            const float s = total(c);                            // before sum overwrites a residual that it shares memory with
            if (p.sum != nullptr) n.store(p.sum, p.ld_sum, c, s);
            if (p.y != nullptr) n.store(p.y, p.ld_y, c, s * ro * n.param(p.weight_out, c));
        }
        n.r.sync();
    }
}
template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_wide_kernel(const __grid_constant__ NormParams p) {
    extern __shared__ float norm_shared[];
    NormWide<T> n{p, norm_row(p, norm_shared), 0};
    float* rs = norm_shared + kNormShared;
    float* gm = rs + p.channels / p.group;                       // sums over groups of t' xh
    float* part = p.partial + static_cast<long long>(blockIdx.x) * 3 * p.channels;
    seq_grid_wait();
    for (int c = n.r.thread; c < 3 * p.channels; c += n.r.threads) part[c] = 0.0f;
    n.r.sync();
    for (n.row = blockIdx.x; n.row < p.rows; n.row += gridDim.x) {
        if (p.norm_in)
            n.groups(rs, [&](int c) { const float v = n.at(p.x, p.ld_x, c); return v * v; }, [&](float v) { return rsqrtf(fmaf(v, p.inv_group, p.eps)); });
        float square = 0.0f, inner = 0.0f, ro = 0.0f, mean = 0.0f;
        if (p.dy != nullptr) {
            for (int c = n.r.thread; c < p.channels; c += n.r.threads) {
                const float s = fmaf(n.param(p.scale, c), n.gated(rs, c), n.at(p.residual, p.ld_residual, c));
                square = fmaf(s, s, square);
                inner = fmaf(n.at(p.dy, p.ld_dy, c) * n.param(p.weight_out, c), s, inner);
            }
            square = n.r.row_sum(square);
            inner = n.r.row_sum(inner);
            ro = rsqrtf(fmaf(square, p.inv_channels, p.eps));
            mean = inner * ro * p.inv_channels;
        }
        auto sh = [&](int c) { return fmaf(n.param(p.scale, c), n.gated(rs, c), n.at(p.residual, p.ld_residual, c)) * ro; };
        auto ds = [&](int c) {
            float d = n.at(p.dsum, p.ld_dsum, c);
            if (p.dy != nullptr) d = fmaf(ro, fmaf(-sh(c), mean, n.at(p.dy, p.ld_dy, c) * n.param(p.weight_out, c)), d);
            return d;
        };
        auto du = [&](int c) {
            float d = ds(c) * n.param(p.scale, c);
            if (p.gate != nullptr) {
                const float g = n.at(p.gate, p.ld_gate, c);
                d *= g * sigmoid_f<T>(g);
            }
            return d;
        };
        auto weight = [&](int c) { return p.norm_in ? n.param(p.weight_in, c) : 1.0f; };
        if (p.norm_in) n.groups(gm, [&](int c) { return du(c) * weight(c) * n.at(p.x, p.ld_x, c) * n.rstd(rs, c); }, [&](float v) { return v * p.inv_group; });
        for (int c = n.r.thread; c < p.channels; c += n.r.threads) {
            const float d = ds(c), t = du(c), x = n.at(p.x, p.ld_x, c), r1 = n.rstd(rs, c);
            if (p.want_in) part[c] = fmaf(t, x * r1, part[c]);
            if (p.want_scale) part[p.channels + c] = fmaf(d, n.gated(rs, c), part[p.channels + c]);
            if (p.want_out) part[2 * p.channels + c] = fmaf(n.at(p.dy, p.ld_dy, c), p.dy != nullptr ? sh(c) : 0.0f, part[2 * p.channels + c]);
            if (p.dresidual != nullptr) n.store(p.dresidual, p.ld_dresidual, c, d);
            if (p.dgate != nullptr) {
                const float g = n.at(p.gate, p.ld_gate, c), sig = sigmoid_f<T>(g);
                n.store(p.dgate, p.ld_dgate, c, d * n.param(p.scale, c) * (x * r1 * weight(c)) * sig * fmaf(g, 1.0f - sig, 1.0f));
            }
            if (p.dx != nullptr) n.store(p.dx, p.ld_dx, c, p.norm_in ? r1 * fmaf(-x * r1, gm[c / p.group], t * weight(c)) : t * weight(c));
        }
        n.r.sync();
    }
}

// Parameter gradients from the sets' sums: one block per 32 channels, each of its eight warps an eighth of the sets.
__global__ void __launch_bounds__(256) norm_join_kernel(int channels, long long sets, const float* __restrict__ partial, float* __restrict__ dweight_in,
                                                        float* __restrict__ dscale, float* __restrict__ dweight_out) {
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float* const out = blockIdx.y == 0 ? dweight_in : blockIdx.y == 1 ? dscale : dweight_out;
    if (out == nullptr) return;
    seq_grid_wait();
    float v = 0.0f;
    if (c < channels)
        for (long long s = warp; s < sets; s += 8) v += partial[(s * 3 + blockIdx.y) * channels + c];
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < channels) {
#pragma unroll
        for (int w = 1; w < 8; ++w) v += sums[w][lane];
        out[c] = v;
    }
}

}  // namespace tdx
