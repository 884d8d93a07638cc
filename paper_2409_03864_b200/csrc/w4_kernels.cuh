// Products with 4-bit weights:  y[m, n] = sum_k x[m, k] * scale[n, k / group] * (q[n, k] - zero[n, k / group]).
//
// q is stored two values to a byte, the even k in the low half, rows of ceil(K / 2) bytes; scales have the type of x; zeros
// are one byte per group (8 where there are none).
#pragma once
#include "seq_common.cuh"

namespace tdx {

struct W4Params {
    long long M, N, K;
    int group;
    const void* x; long long ld_x;
    const uint8_t* weight;
    const void* scales;
    const uint8_t* zeros;
    void* y; long long ld_y;
};

// Any group size, stride and alignment: a warp per output column n goes over K for up to four rows of x at a time.
template <typename T>
__global__ void __launch_bounds__(128) w4_generic_kernel(const __grid_constant__ W4Params p) {
    seq_launch_dependents();
    seq_grid_wait();
    const int lane = threadIdx.x & 31;
    const long long n = blockIdx.x * 4LL + (threadIdx.x >> 5);
    if (n >= p.N) return;
    const long long pitch = (p.K + 1) / 2, groups = (p.K + p.group - 1) / p.group;
    const uint8_t* w = p.weight + n * pitch;
    const T* scales = static_cast<const T*>(p.scales) + n * groups;
    const uint8_t* zeros = p.zeros ? p.zeros + n * groups : nullptr;
    for (long long m0 = 4LL * blockIdx.y; m0 < p.M; m0 += 4LL * gridDim.y) {
        const T* x = static_cast<const T*>(p.x) + m0 * p.ld_x;
        const int rows = static_cast<int>(min(4LL, p.M - m0));
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (long long k = lane; k < p.K; k += 32) {
            const long long g = k / p.group;
            const int byte = __ldg(w + (k >> 1)), q = k & 1 ? byte >> 4 : byte & 15;
            const float wv = static_cast<float>(q - (zeros ? __ldg(zeros + g) : 8)) * seq_to_float(scales[g]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < rows) acc[r] = fmaf(seq_to_float(x[r * p.ld_x + k]), wv, acc[r]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r >= rows) break;
#pragma unroll
            for (int m = 16; m > 0; m /= 2) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], m);
            if (lane == 0) static_cast<T*>(p.y)[(m0 + r) * p.ld_y + n] = seq_from_float<T>(acc[r]);
        }
    }
}

// Quantisation: one warp per group.  Symmetric (zeros == nullptr): scale = max |w| / 7 and q = round(w / scale) + 8 in 1..15.
// With zeros: scale = (max(w, 0) - min(w, 0)) / 15, zero = round(-min / scale), q = round(w / scale) + zero in 0..15.  The scale
// is rounded to its stored type before it divides; halves round to even; a group of zeros gets the scale 1.
template <typename T>
__global__ void __launch_bounds__(128) w4_quantize_kernel(long long N, long long K, int group, const T* __restrict__ w, long long ld_w,
                                                          uint8_t* __restrict__ q, T* __restrict__ scales, uint8_t* __restrict__ zeros) {
    seq_grid_wait();
    const int lane = threadIdx.x & 31;
    const long long groups = (K + group - 1) / group, id = blockIdx.x * 4LL + (threadIdx.x >> 5);
    if (id >= N * groups) return;
    const long long n = id / groups, g = id - n * groups, k0 = g * group, k1 = min(K, k0 + group);
    const T* row = w + n * ld_w;
    float lo = 0.0f, hi = 0.0f;
    for (long long k = k0 + lane; k < k1; k += 32) {
        const float v = seq_to_float(row[k]);
        lo = fminf(lo, v);
        hi = fmaxf(hi, v);
    }
#pragma unroll
    for (int m = 16; m > 0; m /= 2) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, m));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    const T stored = seq_from_float<T>(zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f);
    float scale = seq_to_float(stored);
    if (!(scale > 0.0f)) scale = 1.0f;
    const float zero = zeros ? fminf(fmaxf(rintf(-lo / scale), 0.0f), 15.0f) : 8.0f, least = zeros ? 0.0f : 1.0f;
    if (lane == 0) {
        scales[id] = seq_from_float<T>(scale);
        if (zeros) zeros[id] = static_cast<uint8_t>(zero);
    }
    const long long pitch = (K + 1) / 2;
    // group is even or the only one, so that no byte is shared by two groups
    for (long long k = k0 + 2 * lane; k < k1; k += 64) {
        const int a = static_cast<int>(fminf(fmaxf(rintf(seq_to_float(row[k]) / scale) + zero, least), 15.0f));
        const int b = k + 1 < k1 ? static_cast<int>(fminf(fmaxf(rintf(seq_to_float(row[k + 1]) / scale) + zero, least), 15.0f)) : static_cast<int>(zero);
        q[n * pitch + (k >> 1)] = static_cast<uint8_t>(a | (b << 4));
    }
}

// ---------------------------------------------------------------- tensor-core kernel
// Bound by reading the weights: every weight is read once from global memory straight into the registers from which it is a
// matrix operand, by 4-, 8- or 16-byte loads (group / 4 weights: the four threads that share a weight row hold one group).
//
// mma.m16n8k16 with 16 rows of weights as A and 8 columns of x^T as B.  Which k of x meets which k of W within an instruction
// is free as long as both sides agree, so nothing is moved between threads: from a word of eight weights of neighbouring k a
// shift, a mask and the exponent of 128 make bf16 pairs (128 + q[j], 128 + q[j + 4]), and subtracting 128 + zero leaves the exact
// integer q - zero.  The products of a group are summed in fp32 by the tensor cores and enter the result times the group's
// scale, so weights are never rounded.
//
// bf16: a column of B is a row of x.  fp32: each value of x is cut into three bf16 pieces (8 + 8 + 8 significant bits, no
// remainder), three neighbouring columns, so that the products are those of the full fp32 value.
//
// A block has 16 rows of W and all of K: its warps take groups in turn and their sums are joined in shared memory in the
// order of the warps.  blockIdx.y goes over the columns.
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t w4_pair(uint32_t word, int j, __nv_bfloat162 offset) {
    const uint32_t bits = ((word >> (4 * j)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&bits), offset);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The three bf16 pieces of an fp32 value, by truncation; what is not finite is all in the first.
__device__ __forceinline__ uint32_t w4_piece(float v, int piece) {
    const uint32_t bits = __float_as_uint(v);
    if ((bits & 0x7f800000u) == 0x7f800000u) return piece ? 0u : (bits >> 16) | (bits & 0x007fffffu ? 0x40u : 0u);
    const float r1 = v - __uint_as_float(bits & 0xffff0000u);
    const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
    return __float_as_uint(piece == 0 ? v : piece == 1 ? r1 : r2) >> 16;
}

template <typename T> struct W4Columns;
template <> struct W4Columns<__nv_bfloat16> { static constexpr int kRows = 8, kPieces = 1; };   // rows of x in 8 columns
template <> struct W4Columns<float> { static constexpr int kRows = 2, kPieces = 3; };

// WORDS = group / 32 words of weights per thread, row and group.  TILES: tiles of 8 columns.
template <typename T, int WORDS, int TILES>
__global__ void __launch_bounds__(256) w4_mma_kernel(const __grid_constant__ W4Params p) {
    constexpr int kWarps = 8, kGroup = 32 * WORDS, kPer = 8 * WORDS;   // kPer: weights of a thread, row and group
    constexpr int kAhead = 8 / WORDS;                                  // groups in flight: 32 bytes a row
    __shared__ float red[kWarps][16][TILES * 8 + 1];
    seq_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const long long n0 = blockIdx.x * 16LL, m0 = static_cast<long long>(blockIdx.y) * W4Columns<T>::kRows * TILES;
    const int groups = static_cast<int>(p.K / kGroup);
    const long long pitch = p.K / 2;
    const long long r0 = min(n0 + g, p.N - 1), r1 = min(n0 + g + 8, p.N - 1);
    const uint8_t* wp0 = p.weight + r0 * pitch + t * (4 * WORDS);
    const uint8_t* wp1 = p.weight + r1 * pitch + t * (4 * WORDS);
    const T* sp0 = static_cast<const T*>(p.scales) + r0 * groups;
    const T* sp1 = static_cast<const T*>(p.scales) + r1 * groups;
    const uint8_t* zp0 = p.zeros ? p.zeros + r0 * groups : nullptr;
    const uint8_t* zp1 = p.zeros ? p.zeros + r1 * groups : nullptr;
    // this thread's column of each tile
    const T* xp[TILES];
    bool has[TILES];
    const int piece = W4Columns<T>::kPieces == 1 ? 0 : g % 3;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int in_tile = W4Columns<T>::kPieces == 1 ? g : g / 3;
        const long long m = m0 + i * W4Columns<T>::kRows + in_tile;
        has[i] = in_tile < W4Columns<T>::kRows && m < p.M;
        xp[i] = static_cast<const T*>(p.x) + (has[i] ? m : 0) * p.ld_x + t * kPer;
    }
    float acc[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;

    typedef typename SeqBits<4 * WORDS>::type word_t;
    union Words { word_t v; uint32_t w[WORDS]; };
    Words q0[kAhead], q1[kAhead];
    float s0[kAhead], s1[kAhead];
    int z0[kAhead], z1[kAhead];
    auto fetch = [&](int slot, int grp) {
        if (grp < groups) {
            q0[slot].v = __ldg(reinterpret_cast<const word_t*>(wp0 + static_cast<long long>(grp) * (kGroup / 2)));
            q1[slot].v = __ldg(reinterpret_cast<const word_t*>(wp1 + static_cast<long long>(grp) * (kGroup / 2)));
            s0[slot] = seq_to_float(sp0[grp]);
            s1[slot] = seq_to_float(sp1[grp]);
            z0[slot] = zp0 ? __ldg(zp0 + grp) : 8;
            z1[slot] = zp1 ? __ldg(zp1 + grp) : 8;
        }
    };
    seq_grid_wait();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(i, warp + i * kWarps);
    for (int base = warp; base < groups; base += kWarps * kAhead) {
#pragma unroll
        for (int slot = 0; slot < kAhead; ++slot) {
            const int grp = base + slot * kWarps;
            if (grp >= groups) break;
            const __nv_bfloat162 o0 = __float2bfloat162_rn(static_cast<float>(128 + z0[slot]));
            const __nv_bfloat162 o1 = __float2bfloat162_rn(static_cast<float>(128 + z1[slot]));
            float sum[TILES][4];
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[i][j] = 0.0f;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                uint32_t a0[4], a1[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    a0[j] = w4_pair(q0[slot].w[w], j, o0);
                    a1[j] = w4_pair(q1[slot].w[w], j, o1);
                }
#pragma unroll
                for (int i = 0; i < TILES; ++i) {
                    uint32_t b[4] = {0u, 0u, 0u, 0u};                  // pairs (x[j], x[j + 4])
                    if (has[i]) {
                        const T* x = xp[i] + static_cast<long long>(grp) * kGroup + w * 8;
                        if (sizeof(T) == 2) {
                            const uint4 v = __ldg(reinterpret_cast<const uint4*>(x));
                            b[0] = __byte_perm(v.x, v.z, 0x5410);
                            b[1] = __byte_perm(v.x, v.z, 0x7632);
                            b[2] = __byte_perm(v.y, v.w, 0x5410);
                            b[3] = __byte_perm(v.y, v.w, 0x7632);
                        } else {
                            const float4 lo = __ldg(reinterpret_cast<const float4*>(x)), hi = __ldg(reinterpret_cast<const float4*>(x) + 1);
                            b[0] = w4_piece(lo.x, piece) | w4_piece(hi.x, piece) << 16;
                            b[1] = w4_piece(lo.y, piece) | w4_piece(hi.y, piece) << 16;
                            b[2] = w4_piece(lo.z, piece) | w4_piece(hi.z, piece) << 16;
                            b[3] = w4_piece(lo.w, piece) | w4_piece(hi.w, piece) << 16;
                        }
                    }
                    mma_bf16(sum[i], a0[0], a1[0], a0[1], a1[1], b[0], b[1]);
                    mma_bf16(sum[i], a0[2], a1[2], a0[3], a1[3], b[2], b[3]);
                }
            }
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                acc[i][0] = fmaf(s0[slot], sum[i][0], acc[i][0]);
                acc[i][1] = fmaf(s0[slot], sum[i][1], acc[i][1]);
                acc[i][2] = fmaf(s1[slot], sum[i][2], acc[i][2]);
                acc[i][3] = fmaf(s1[slot], sum[i][3], acc[i][3]);
            }
            fetch(slot, grp + kWarps * kAhead);
        }
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        red[warp][g][i * 8 + 2 * t] = acc[i][0];
        red[warp][g][i * 8 + 2 * t + 1] = acc[i][1];
        red[warp][g + 8][i * 8 + 2 * t] = acc[i][2];
        red[warp][g + 8][i * 8 + 2 * t + 1] = acc[i][3];
    }
    __syncthreads();
    constexpr int kOut = 16 * W4Columns<T>::kRows * TILES;
    for (int o = threadIdx.x; o < kOut; o += 256) {
        const int row = o % 16, in = o / 16;
        const long long m = m0 + in, n = n0 + row;
        if (m >= p.M || n >= p.N) continue;
        constexpr int kP = W4Columns<T>::kPieces;
        const int col = in / W4Columns<T>::kRows * 8 + in % W4Columns<T>::kRows * kP;
        float s = 0.0f;
#pragma unroll
        for (int piece_of = kP - 1; piece_of >= 0; --piece_of)         // the small pieces first
#pragma unroll
            for (int w = 0; w < kWarps; ++w) s += red[w][row][col + piece_of];
        static_cast<T*>(p.y)[m * p.ld_y + n] = seq_from_float<T>(s);
    }
}

}  // namespace tdx
