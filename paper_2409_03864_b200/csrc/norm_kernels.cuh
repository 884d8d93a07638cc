// Norms before and after a block with its gate and residual scale, in one pass over a row and back.
//
//   u = x * rstd_in * weight_in   (rstd_in over a group of channels; or u = x)      a = u * silu(gate)   (or a = u)
//   s = residual + scale * a      (or s = scale * a)                                y = s * rstd_out * weight_out
//
// Bandwidth bounds both directions, so a row is read once: `warps` warps hold it in registers, NV vectors of VEC channels a
// thread, all loads issued before the first use.  Sums over a row go through shuffles and one barrier of the row's own warps;
// sums over groups of channels through shuffles alone where a group is 1, 2, 4, ... 32 vectors, else through shared memory.
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

template <int VEC>
__device__ __forceinline__ void norm_param(const float* p, int c, float (&f)[VEC]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = 1.0f;
        return;
    }
    constexpr int kStep = VEC >= 4 ? 4 : VEC;
#pragma unroll
    for (int i = 0; i < VEC; i += kStep) {
        float part[kStep];
        seq_unpack(seq_load<float, kStep>(p + c + i), part);
#pragma unroll
        for (int j = 0; j < kStep; ++j) f[i + j] = part[j];
    }
}
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
__device__ __forceinline__ void norm_store(void* base, long long ld, long long row, int c, const float (&f)[VEC]) {
    seq_store<T, VEC>(static_cast<T*>(base) + row * ld + c, f);
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

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kNormThreads, NV * VEC <= 8 ? 2 : 1) norm_fwd_kernel(const __grid_constant__ NormParams p) {
    extern __shared__ float norm_shared[];
    NormRow r = norm_row(p, norm_shared);
    const int sets = (blockDim.x >> 5) / p.warps;
    seq_grid_wait();
    const long long step = static_cast<long long>(gridDim.x) * sets;
    SeqVec<T, VEC> nx[NV], ng[NV], nr[NV];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            const bool there = c < p.channels && row < p.rows;
            nx[i] = norm_load<T, VEC>(p.x, p.ld_x, row, c, there);
            ng[i] = norm_load<T, VEC>(p.gate, p.ld_gate, row, c, there);
            nr[i] = norm_load<T, VEC>(p.residual, p.ld_residual, row, c, there);
        }
    };
    constexpr bool kAhead = NV * VEC <= 8;                       // wider threads have no registers to spare
    long long row = static_cast<long long>(blockIdx.x) * sets + r.slot;
    if (kAhead) fetch(row);
    for (; row < p.rows; row += step) {
        if (!kAhead) fetch(row);
        SeqVec<T, VEC> vx[NV], vg[NV], vr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) { vx[i] = nx[i]; vg[i] = ng[i]; vr[i] = nr[i]; }
        if (kAhead) fetch(row + step);                           // on its way while this row is worked on
        float rstd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[VEC];
            seq_unpack(vx[i], f);
            rstd[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < VEC; ++j) rstd[i] = fmaf(f[j], f[j], rstd[i]);
        }
        if (p.norm_in) {
            r.group_sum(p, rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_group, p.eps));
        }
        float s[NV][VEC], square = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                seq_unpack(vx[i], s[i]);
                if (p.norm_in) {
                    float w[VEC];
                    norm_param(p.weight_in, c, w);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s[i][j] = s[i][j] * rstd[i] * w[j];
                }
                if (p.gate != nullptr) {
                    float g[VEC];
                    seq_unpack(vg[i], g);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s[i][j] *= g[j] * sigmoid_f<T>(g[j]);
                }
                float k[VEC], add[VEC];
                norm_param(p.scale, c, k);
                seq_unpack(vr[i], add);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    s[i][j] = fmaf(k[j], s[i][j], add[j]);
                    square = fmaf(s[i][j], s[i][j], square);
                }
                if (p.sum != nullptr) norm_store<T, VEC>(p.sum, p.ld_sum, row, c, s[i]);
            }
        }
        if (p.y != nullptr) {
            const float rs = rsqrtf(fmaf(r.row_sum(square), p.inv_channels, p.eps));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (r.thread + i * r.threads) * VEC;
                if (c < p.channels) {
                    float w[VEC];
                    norm_param(p.weight_out, c, w);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) w[j] *= s[i][j] * rs;
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
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const __grid_constant__ NormParams p) {
    extern __shared__ float norm_shared[];
    NormRow r = norm_row(p, norm_shared);
    const int sets = (blockDim.x >> 5) / p.warps;
    const long long set = static_cast<long long>(blockIdx.x) * sets + r.slot;
    float sum_in[NV][VEC], sum_scale[NV][VEC], sum_out[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum_in[i][j] = sum_scale[i][j] = sum_out[i][j] = 0.0f;
    seq_grid_wait();
    const long long step = static_cast<long long>(gridDim.x) * sets;
    // with up to 8 channels a thread the registers hold the next row's vectors and the parameters too
    constexpr bool kAhead = NV * VEC <= 8;
    SeqVec<T, VEC> vx[NV], vg[NV], vr[NV], vs[NV], vy[NV], nx[NV], ng[NV], nr[NV], ns[NV], ny[NV];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            const bool there = c < p.channels && row < p.rows;
            nx[i] = norm_load<T, VEC>(p.x, p.ld_x, row, c, there);
            ng[i] = norm_load<T, VEC>(p.gate, p.ld_gate, row, c, there);
            nr[i] = norm_load<T, VEC>(p.residual, p.ld_residual, row, c, there && p.dy != nullptr);
            ns[i] = norm_load<T, VEC>(p.dsum, p.ld_dsum, row, c, there);
            ny[i] = norm_load<T, VEC>(p.dy, p.ld_dy, row, c, there);
        }
    };
    if (kAhead) fetch(set);
    float keep_in[NV][VEC], keep_scale[NV][VEC], keep_out[NV][VEC];
    if (kAhead) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                norm_param(p.norm_in ? p.weight_in : nullptr, c, keep_in[i]);
                norm_param(p.scale, c, keep_scale[i]);
                norm_param(p.weight_out, c, keep_out[i]);
            }
        }
    }
    auto param = [&](const float* from, const float (&kept)[VEC], int c, float (&f)[VEC]) {
        if (kAhead) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = kept[j];
        } else {
            norm_param(from, c, f);
        }
    };
    for (long long row = set; row < p.rows; row += step) {
        if (!kAhead) fetch(row);
#pragma unroll
        for (int i = 0; i < NV; ++i) { vx[i] = nx[i]; vg[i] = ng[i]; vr[i] = nr[i]; vs[i] = ns[i]; vy[i] = ny[i]; }
        if (kAhead) fetch(row + step);
        float rstd[NV];
        if (p.norm_in) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float f[VEC];
                seq_unpack(vx[i], f);
                rstd[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < VEC; ++j) rstd[i] = fmaf(f[j], f[j], rstd[i]);
            }
            r.group_sum(p, rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_group, p.eps));
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) rstd[i] = 1.0f;
        }
        // the way forward once more: xh = x rstd, a; then ds
        float ds[NV][VEC], a[NV][VEC], sig[NV][VEC];
        float square = 0.0f, inner = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            if (c < p.channels) {
                float w[VEC];
                seq_unpack(vx[i], a[i]);
                param(p.norm_in ? p.weight_in : nullptr, keep_in[i], c, w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) a[i][j] *= rstd[i] * w[j];
                if (p.gate != nullptr) {
                    float g[VEC];
                    seq_unpack(vg[i], g);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        sig[i][j] = sigmoid_f<T>(g[j]);
                        a[i][j] *= g[j] * sig[i][j];
                    }
                }
                if (p.dy != nullptr) {
                    float k[VEC], add[VEC], dy[VEC], wo[VEC];
                    param(p.scale, keep_scale[i], c, k);
                    param(p.weight_out, keep_out[i], c, wo);
                    seq_unpack(vr[i], add);
                    seq_unpack(vy[i], dy);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float s = fmaf(k[j], a[i][j], add[j]);
                        square = fmaf(s, s, square);
                        inner = fmaf(dy[j] * wo[j], s, inner);
                    }
                }
            }
        }
        float rs = 0.0f, mean = 0.0f;
        if (p.dy != nullptr) {
            r.row_sums(square, inner);
            rs = rsqrtf(fmaf(square, p.inv_channels, p.eps));
            mean = inner * rs * p.inv_channels;                  // mean(t sh)
        }
        float group[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (r.thread + i * r.threads) * VEC;
            group[i] = 0.0f;
            if (c < p.channels) {
                float k[VEC], w[VEC], x[VEC];
                param(p.scale, keep_scale[i], c, k);
                seq_unpack(vs[i], ds[i]);
                if (p.dy != nullptr) {
                    float add[VEC], dy[VEC], wo[VEC];
                    param(p.weight_out, keep_out[i], c, wo);
                    seq_unpack(vr[i], add);
                    seq_unpack(vy[i], dy);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float sh = fmaf(k[j], a[i][j], add[j]) * rs;
                        ds[i][j] = fmaf(rs, fmaf(-sh, mean, dy[j] * wo[j]), ds[i][j]);
                        sum_out[i][j] = fmaf(dy[j], sh, sum_out[i][j]);
                    }
                }
                if (p.dresidual != nullptr) norm_store<T, VEC>(p.dresidual, p.ld_dresidual, row, c, ds[i]);
                seq_unpack(vx[i], x);
                param(p.norm_in ? p.weight_in : nullptr, keep_in[i], c, w);
                float g[VEC], dg[VEC];
                seq_unpack(vg[i], g);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    sum_scale[i][j] = fmaf(ds[i][j], a[i][j], sum_scale[i][j]);
                    const float da = ds[i][j] * k[j], xh = x[j] * rstd[i];
                    float du = da;
                    if (p.gate != nullptr) {
                        dg[j] = da * (xh * w[j]) * sig[i][j] * fmaf(g[j], 1.0f - sig[i][j], 1.0f);
                        du = da * (g[j] * sig[i][j]);
                    }
                    sum_in[i][j] = fmaf(du, xh, sum_in[i][j]);
                    ds[i][j] = du * w[j];                        // t' from here on
                    group[i] = fmaf(ds[i][j], xh, group[i]);
                }
                if (p.dgate != nullptr) norm_store<T, VEC>(p.dgate, p.ld_dgate, row, c, dg);
            }
        }
        if (p.norm_in) r.group_sum(p, group);
        if (p.dx != nullptr) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (r.thread + i * r.threads) * VEC;
                if (c < p.channels) {
                    if (p.norm_in) {
                        float x[VEC];
                        seq_unpack(vx[i], x);
                        const float m = group[i] * p.inv_group * rstd[i];
#pragma unroll
                        for (int j = 0; j < VEC; ++j) ds[i][j] = rstd[i] * fmaf(-x[j], m, ds[i][j]);
                    }
                    norm_store<T, VEC>(p.dx, p.ld_dx, row, c, ds[i]);
                }
            }
        }
    }
    float* part = p.partial + set * 3 * p.channels;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (r.thread + i * r.threads) * VEC;
        if (c < p.channels) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (p.want_in) part[c + j] = sum_in[i][j];
                if (p.want_scale) part[p.channels + c + j] = sum_scale[i][j];
                if (p.want_out) part[2 * p.channels + c + j] = sum_out[i][j];
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
