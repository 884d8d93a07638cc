// Matrix products grouped by expert: rows offsets[e] .. offsets[e + 1] - 1 of the activations meet expert e's matrix.
//
//   forward   y[t, n]  = sum_k x[t, k] w[e, n, k]
//   dx        dx[t, k] = sum_n dy[t, n] w[e, n, k]
//   dw        dw[e, n, k] = sum_t dy[t, n] x[t, k]
//
// grouped_umma_kernel runs them on the tensor cores (bf16, 16-byte aligned rows), grouped_simt_kernel on the CUDA cores (fp32, and
// any alignment).  The offsets live on the device, so both work out there which tiles there are.
#pragma once
#include "bounded_wait.cuh"
#include "seq_common.cuh"

namespace tdx {

enum GroupedPass { kGroupedForward, kGroupedDx, kGroupedDw };

struct GroupedParams {
    long long rows;
    int experts, N, K;
    const int* offsets;
    const void* a;                   // activations that the sum runs over: x, dy, or (dw) dy
    const void* b;                   // weight, weight, or (dw) x
    void* out;
    long long ld_a, ld_b, ld_out;
    int* status;
    // tensor-core kernel
    int stages;
    int out_tiles;                   // tiles of 128 * HALVES output features
    int red_blocks;                  // blocks of 64 of the reduction (forward, dx)
    int col_tiles;                   // dw: tiles of kBT columns
};

// The range of an expert's rows; one that leaves [0, rows] or descends is reported and empty.
__device__ __forceinline__ SeqRange grouped_range(const GroupedParams& p, int e) { return seq_range(p.offsets, e, p.rows, p.rows, p.status); }

// ---------------------------------------------------------------- CUDA cores
constexpr int kSimtN = 128, kSimtK = 16;

// One (8 BM / 64 x 8 a thread) tile of BM x 128 outputs, 16 of the reduction at a time through shared memory; the next 16 are on their
// way while these are multiplied.  BM = 16 serves experts of few rows, where a tile of 64 would be mostly empty.
template <typename T, int PASS, int BM>
__global__ void __launch_bounds__(128) grouped_simt_kernel(const __grid_constant__ GroupedParams p) {
    constexpr int TM = BM / 8;                                    // rows a thread
    __shared__ __align__(16) float sa[2][kSimtK][BM + 4];
    __shared__ __align__(16) float sb[2][kSimtK][kSimtN + 4];
    const T* a = static_cast<const T*>(p.a);
    const T* b = static_cast<const T*>(p.b);
    T* out = static_cast<T*>(p.out);
    const int tid = threadIdx.x;
    seq_grid_wait();
    int m_count, n_count, m0, n0;
    long long depth;
    if (PASS == kGroupedDw) {
        const int tiles_n = (p.K + kSimtN - 1) / kSimtN, tiles_m = (p.N + BM - 1) / BM;
        const long long item = blockIdx.x;
        const int e = static_cast<int>(item / (static_cast<long long>(tiles_n) * tiles_m)), in = static_cast<int>(item - static_cast<long long>(e) * tiles_n * tiles_m);
        const SeqRange r = grouped_range(p, e);
        m0 = in / tiles_n * BM; n0 = in % tiles_n * kSimtN;
        m_count = p.N; n_count = p.K; depth = r.len;
        a += r.first * p.ld_a; b += r.first * p.ld_b; out += static_cast<long long>(e) * p.N * p.K;
    } else {
        n_count = PASS == kGroupedForward ? p.N : p.K;
        const int tiles_n = (n_count + kSimtN - 1) / kSimtN;
        const long long number = blockIdx.x / tiles_n;
        n0 = (blockIdx.x - number * tiles_n) * kSimtN;
        if (n0 == 0) seq_check(p.offsets, number, p.experts, p.rows, p.rows, p.status);
        const SeqPiece piece = seq_piece(p.offsets, p.experts, 1, BM, number);
        const SeqRange r = grouped_range(p, static_cast<int>(piece.b));
        if (static_cast<long long>(piece.index) * BM >= r.len) return;
        m0 = piece.index * BM; m_count = r.len; depth = PASS == kGroupedForward ? p.K : p.N;
        a += r.first * p.ld_a; b += piece.b * static_cast<long long>(p.N) * p.K; out += r.first * p.ld_out;
    }
    const long long ld_b = PASS == kGroupedDw ? p.ld_b : p.K, ld_out = PASS == kGroupedDw ? p.K : p.ld_out;
    constexpr bool kADeep = PASS != kGroupedDw, kBDeep = PASS == kGroupedForward;   // the reduction is the contiguous dimension
    constexpr int kAOf = BM * kSimtK / 128, kBOf = kSimtN * kSimtK / 128;
    float ra[kAOf], rb[kBOf];
    auto fetch = [&](long long k0) {
#pragma unroll
        for (int i = 0; i < kAOf; ++i) {
            const int at = tid + i * 128;
            const int m = kADeep ? at / kSimtK : at % BM, k = kADeep ? at % kSimtK : at / BM;
            const bool there = m0 + m < m_count && k0 + k < depth;
            ra[i] = there ? seq_to_float(kADeep ? a[(m0 + m) * p.ld_a + k0 + k] : a[(k0 + k) * p.ld_a + m0 + m]) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kBOf; ++i) {
            const int at = tid + i * 128;
            const int n = kBDeep ? at / kSimtK : at % kSimtN, k = kBDeep ? at % kSimtK : at / kSimtN;
            const bool there = n0 + n < n_count && k0 + k < depth;
            rb[i] = there ? seq_to_float(kBDeep ? b[(n0 + n) * ld_b + k0 + k] : b[(k0 + k) * ld_b + n0 + n]) : 0.0f;
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kAOf; ++i) {
            const int at = tid + i * 128;
            sa[buf][kADeep ? at % kSimtK : at / BM][kADeep ? at / kSimtK : at % BM] = ra[i];
        }
#pragma unroll
        for (int i = 0; i < kBOf; ++i) {
            const int at = tid + i * 128;
            sb[buf][kBDeep ? at % kSimtK : at / kSimtN][kBDeep ? at / kSimtK : at % kSimtN] = rb[i];
        }
    };
    float acc[TM][8];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.0f;
    const int tm = tid / 16 * TM, tn = tid % 16 * 4;              // columns tn .. tn + 3 and 64 + tn .. : no bank conflicts
    fetch(0);
    put(0);
    __syncthreads();
    int buf = 0;
    for (long long k0 = 0; k0 < depth; k0 += kSimtK) {
        const bool more = k0 + kSimtK < depth;
        if (more) fetch(k0 + kSimtK);
#pragma unroll
        for (int k = 0; k < kSimtK; ++k) {
            float fa[TM], fb[8];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = sa[buf][k][tm + i];
#pragma unroll
            for (int j = 0; j < 4; ++j) { fb[j] = sb[buf][k][tn + j]; fb[4 + j] = sb[buf][k][64 + tn + j]; }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(fa[i], fb[j], acc[i][j]);
        }
        if (more) put(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (m0 + tm + i >= m_count) break;
        T* row = out + (m0 + tm + i) * ld_out;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int n = n0 + tn + (j < 4 ? j : 60 + j);
            if (n < n_count) row[n] = seq_from_float<T>(acc[i][j]);
        }
    }
}

}  // namespace tdx
