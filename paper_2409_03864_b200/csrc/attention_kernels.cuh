// Linear attention with a decay per head:  S[t] = l S[t-1] + k[t]^T v[t],  out[t] = q[t] S[t].
//
// A chunk of 64 rows with the state S0 in front of it is three products of matrices:
//   out[i] = sum over j <= i of l^(i-j) (q[i] . k[j]) v[j]  +  l^(i+1) q[i] S0,      S1 = l^n S0 + sum_j l^(n-1-j) k[j]^T v[j]
// so the rows of a sequence cost 2 * 64 (dim_k + dim_v) + 4 dim_k dim_v operations each instead of a walk over the state.
//
// The gradients are the same sum with the roles exchanged, dq with (dout, v, k) and S^T, dv and dk from the last row to the first with
// (k, q, dout) and (v, dout, q) and the gradient of the state, so one kernel serves all four ("q", "k", "v" below are roles).
//
// This file: mma.sync, for fp32 (three bf16 pieces of every operand) and for bf16 rows that the copy engine cannot read.  A chunk is a chain
// of products, each waiting for the one in front, with 8 warps an SM (4 where fp32 operands of more than 64 take the shared memory): that
// latency bounds it, not the bytes.  So sequences are cut into many segments.
#pragma once
#include "seq_common.cuh"

namespace tdx {

struct AttnParams {
    long long batch, max_len, rows;
    int heads, q_share, k_share, v_share;   // heads that share one of q, k, v
    int d1, d2;                             // dims of q and k, and of v and out
    const void *q, *k, *v;
    long long ld_q, ld_k, ld_v;
    void* out;
    long long ld_out;
    int out_f32;                            // out is fp32 for every head (its heads are summed afterwards)
    int wide;                               // rows of out are 32-byte aligned
    int vec;                                // fp32: rows of q, k and v are read 16 bytes at a time
    float scale_in, scale_out;              // on k^T v and on out
    int back;                               // from the last row to the first
    const float* log_decay;
    const int* offsets;
    const int* slots;
    long long n_slots, state_stride;
    const float* state_in;                  // the state before the first row that is worked on (for `back`: behind the last)
    float* state_out;
    int state_vec;                          // attn_umma_kernel: states are read and written 16 bytes at a time along d2
    int s1, s2;                             // strides of a state's d1 and d2
    long long seg, dense;                   // rows of a segment; segments of a dense sequence
    float* carry;                           // [slot][head][slice][KD][kAttnV]: what a piece of a segment adds to the state
    long long sub, sub_dense;               // rows of a piece of a segment (all of them but in attn_umma_kernel), and pieces of a dense sequence
    int all_pieces;                         // attn_umma_kernel: the last segment's pieces are wanted too, for state_out
    int every;                              // sequences of one segment have slots in carry too
    int carry_turned;                       // attn_umma_kernel: carry was written by a sum with d1 and d2 exchanged
    int slices;                             // of kAttnV columns of v
    int* status;
};

// What the pieces of sequences add to the state has slots in `carry`, by which the blocks of the pass over the states are numbered.  Where a
// batch has more sequences than its rows have segments, sequences of one segment have no slots, so that their number goes by the rows.
// Packed (rows are int): sequence b, from `row` on, has its slots from this number on.  Behind a sequence with slots it is floor(len / sub) + 1 more at
// least, which is no less than ceil(len / sub): with `every` since b is, else since it has more than seg rows.
__host__ __device__ __forceinline__ long long attn_slots_before(int row, long long b, int sub, int seg, bool every) {
    return row / sub + (every || b < row / seg ? b : row / seg);
}
__device__ __forceinline__ long long attn_first_slot(const AttnParams& p, long long b) {
    return p.offsets == nullptr ? b * p.sub_dense : attn_slots_before(__ldg(p.offsets + b), b, static_cast<int>(p.sub), static_cast<int>(p.seg), p.every);
}
// The piece of a slot: of the last sequence whose slots begin at or before it (those without begin where the next ones do).
__device__ __forceinline__ SeqPiece attn_slot_piece(const AttnParams& p, long long slot) {
    if (p.offsets == nullptr) return seq_piece(nullptr, p.batch, p.sub_dense, p.sub, slot);
    SeqPiece r;
    r.b = 0;
    for (long long hi = p.batch - 1; r.b < hi;) {
        const long long mid = (r.b + hi + 1) / 2;
        if (attn_first_slot(p, mid) <= slot) r.b = mid;
        else hi = mid - 1;
    }
    const long long index = slot - attn_first_slot(p, r.b);
    r.index = index < 0 || index > kNoPiece ? kNoPiece : static_cast<int>(index);
    return r;
}

constexpr int kAttnC = 64;                  // rows of a chunk
constexpr int kAttnV = 64;                  // columns of v that a block works on
constexpr int kAttnThreads = 128;

__device__ __forceinline__ void attn_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void attn_ldm(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void attn_ldm_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t attn_pair(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ float attn_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float attn_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
// a pair of fp32 values as N bf16 pairs whose sums they are: 8 significant bits each, 3 hold all 24
template <int N>
__device__ __forceinline__ void attn_split(float lo, float hi, uint32_t (&piece)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        piece[i] = attn_pair(lo, hi);
        if (i + 1 < N) { lo -= attn_lo(piece[i]); hi -= attn_hi(piece[i]); }
    }
}
// d += a b over all pairs of pieces that reach 2^-24 of the product.  EXACT: the products of 16 terms are summed on their own and then
// added to d in fp32.  The tensor cores cut off what a term has below the sum's last bit instead of rounding, always towards zero: over
// thousands of rows a sum held there is 3e-6 too small, added up this way it is 2e-7 off.
template <bool EXACT, int NA, int NB>
__device__ __forceinline__ void attn_mma_pieces(float (&d)[4], const uint32_t (&a)[NA][4], const uint32_t (&b0)[NB], const uint32_t (&b1)[NB]) {
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)                            // small terms first
#pragma unroll
        for (int j = NB - 1; j >= 0; --j)
            if (i + j < (NA > NB ? NA : NB)) attn_mma(EXACT ? t : d, a[i], b0[j], b1[j]);
    if (EXACT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] += t[i];
    }
}

template <typename T, int KD>
struct AttnTiles {
    static constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;
    static constexpr int kPitchK = KD * 2 + 16, kPitchV = kAttnV * 2 + 16;      // 16 bytes more than a row: ldmatrix without bank conflicts
    static constexpr int kK = kAttnC * kPitchK, kV = kAttnC * kPitchV, kS = KD * kPitchV;   // one piece
    static constexpr int kState = kPieces * (2 * kK + kV), kBytes = kState + kPieces * kS;
};

// `count` rows of width d of a matrix into the pieces' tiles of WIDTH columns; rows behind the last and columns behind d become zero
template <typename T, int WIDTH>
__device__ __forceinline__ void attn_load(uint8_t* tile, const T* base, long long ld, int step, int count, int d, bool vec) {
    constexpr int kPieces = sizeof(T) == 4 ? 3 : 1, kPitch = WIDTH * 2 + 16, kPiece = kAttnC * kPitch;
    if (sizeof(T) == 4 && vec) {
        constexpr int kPerRow = WIDTH / 4;
#pragma unroll 4
        for (int i = threadIdx.x; i < kAttnC * kPerRow; i += kAttnThreads) {
            const int row = i / kPerRow, c = i % kPerRow * 4;
            const float4 v = row < count && c < d ? __ldg(reinterpret_cast<const float4*>(base + row * step * ld + c)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            uint32_t lo[kPieces], hi[kPieces];
            attn_split(v.x, v.y, lo);
            attn_split(v.z, v.w, hi);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *reinterpret_cast<uint2*>(tile + p * kPiece + row * kPitch + c * 2) = make_uint2(lo[p], hi[p]);
        }
    } else {
        for (int i = threadIdx.x; i < kAttnC * WIDTH / 2; i += kAttnThreads) {
            const int row = i / (WIDTH / 2), c = i % (WIDTH / 2) * 2;
            const T* from = base + row * step * ld + c;
            const float lo = row < count && c < d ? seq_to_float(from[0]) : 0.0f, hi = row < count && c + 1 < d ? seq_to_float(from[1]) : 0.0f;
            uint32_t v[kPieces];
            attn_split(lo, hi, v);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *reinterpret_cast<uint32_t*>(tile + p * kPiece + row * kPitch + c * 2) = v[p];
        }
    }
}

// One block: a segment of a sequence, a head, 64 columns of v.  Four warps: for the outputs a warp has 16 rows of the chunk, for the
// state KD / 4 of its rows, in registers over all chunks; the other blocks of the head's columns do q k^T again (a third of the
// work at dim 128), which leaves registers for two blocks an SM.  STATE: only what the segment adds to the state, for the segments behind it.
// UP: bf16 pieces of the decayed keys that go into the state, 3 where the state is an output and keeps 24 bits, else 2.  The weights of a
// chunk's rows have two pieces (PP; fp32 three): what is rounded once on the way to a bf16 output is the state that its row reads.
template <typename T, int KD, bool STATE, int UP>
__global__ void __launch_bounds__(kAttnThreads) attn_kernel(const __grid_constant__ AttnParams p) {
    typedef AttnTiles<T, KD> Tiles;
    constexpr int NP = Tiles::kPieces, PP = NP == 3 ? 3 : 2, MT = KD / 64, NT = kAttnV / 8, PK = Tiles::kPitchK, PV = Tiles::kPitchV;
    extern __shared__ __align__(16) uint8_t attn_smem[];
    __shared__ float power[kAttnC + 1];                          // l^n
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem = static_cast<uint32_t>(__cvta_generic_to_shared(attn_smem));
    seq_grid_wait();
    const int slice = static_cast<int>(blockIdx.x % p.slices);
    const long long rest = blockIdx.x / p.slices;
    const int head = static_cast<int>(rest % p.heads);
    const long long number = rest / p.heads;
    if (!STATE && head == 0 && slice == 0) seq_check(p.offsets, number, p.batch, p.max_len, p.rows, p.status);
    const SeqPiece piece = STATE ? attn_slot_piece(p, number) : seq_piece(p.offsets, p.batch, p.dense, p.seg, number);
    const SeqRange r = seq_range(p.offsets, piece.b, p.max_len, p.rows, p.status);
    const long long start = piece.index * p.seg;
    const long long slot = !STATE && (p.state_in != nullptr || p.state_out != nullptr) ? state_slot(p.slots, piece.b, p.n_slots, p.status) : -1;
    const long long state_at = slot * p.state_stride + static_cast<long long>(head) * p.d1 * p.d2;
    const bool ends = start + p.seg >= r.len;
    if (start >= r.len && !(piece.index == 0 && !STATE)) return;
    if (STATE && ends) return;                                   // no segment behind it
    const int count = static_cast<int>(ends ? r.len - start : p.seg);
    const double log_l = static_cast<double>(__ldg(p.log_decay + head));
    if (tid <= kAttnC) power[tid] = tid == 0 ? 1.0f : static_cast<float>(exp(log_l * tid));
    // the state that `back` starts with stands behind the last row already: it decays once less
    const int less = p.back && piece.index == 0 ? 1 : 0;

    // this thread's part of the state: rows m (+ 8), columns n (+ 1)
    float st[MT][NT][4];
    const int m_first = warp * (KD / 4) + lane / 4, n_first = lane % 4 * 2;
    const long long carry_size = static_cast<long long>(KD) * kAttnV;
    const long long carry_step = static_cast<long long>(p.heads) * p.slices * carry_size;
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = m_first + a * 16 + (i >> 1) * 8, n = slice * kAttnV + n_first + b * 8 + (i & 1);
                st[a][b][i] = !STATE && p.state_in != nullptr && slot >= 0 && m < p.d1 && n < p.d2 ? __ldg(p.state_in + state_at + m * p.s1 + n * p.s2) : 0.0f;
            }
    if (!STATE && piece.index > 0) {
        const float far = static_cast<float>(exp(log_l * static_cast<double>(p.seg))), first = p.back ? static_cast<float>(exp(log_l * static_cast<double>(p.seg - 1))) : far;
        const float* from = p.carry + ((attn_first_slot(p, piece.b) * p.heads + head) * p.slices + slice) * carry_size;
        for (int s = 0; s < piece.index; ++s, from += carry_step) {
            const float f = s == 0 ? first : far;
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int b = 0; b < NT; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float2 v = *reinterpret_cast<const float2*>(from + (m_first + a * 16 + h * 8) * kAttnV + n_first + b * 8);
                        st[a][b][2 * h] = fmaf(st[a][b][2 * h], f, v.x);
                        st[a][b][2 * h + 1] = fmaf(st[a][b][2 * h + 1], f, v.y);
                    }
        }
    }

    const int step = p.back ? -1 : 1;
    const long long row0 = r.first + (p.back ? r.len - 1 - start : start);
    const T* q = static_cast<const T*>(p.q) + head / p.q_share * p.d1;
    const T* k = static_cast<const T*>(p.k) + head / p.k_share * p.d1;
    const T* v = static_cast<const T*>(p.v) + head / p.v_share * p.d2 + slice * kAttnV;
    const int d2 = min(p.d2 - slice * kAttnV, kAttnV);
    const int chunks = (count + kAttnC - 1) / kAttnC;
    auto load = [&](int c) {
        const int n = min(kAttnC, count - c * kAttnC);
        const long long row = row0 + static_cast<long long>(step) * c * kAttnC;
        if (!STATE) attn_load<T, KD>(attn_smem, q + row * p.ld_q, p.ld_q, step, n, p.d1, p.vec);
        attn_load<T, KD>(attn_smem + NP * Tiles::kK, k + row * p.ld_k, p.ld_k, step, n, p.d1, p.vec);
        attn_load<T, kAttnV>(attn_smem + NP * 2 * Tiles::kK, v + row * p.ld_v, p.ld_v, step, n, d2, p.vec);
    };
    constexpr uint32_t kStateAt = Tiles::kState;
    const uint32_t tq = smem, tk = tq + NP * Tiles::kK, tv = tk + NP * Tiles::kK;
    if (chunks > 0) load(0);
    for (int c = 0; c < chunks; ++c) {
        const int n = min(kAttnC, count - c * kAttnC), shift = c == 0 ? less : 0;
        if (!STATE) {
            // the state in front of the chunk for all warps; rounded to bf16 for the product with q (fp32: all 24 bits in three pieces)
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int b = 0; b < NT; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t piece_of[NP];
                        attn_split(st[a][b][2 * h], st[a][b][2 * h + 1], piece_of);
#pragma unroll
                        for (int i = 0; i < NP; ++i)
                            *reinterpret_cast<uint32_t*>(attn_smem + kStateAt + i * Tiles::kS + (m_first + a * 16 + h * 8) * PV + (n_first + b * 8) * 2) = piece_of[i];
                    }
        }
        __syncthreads();
        if (!STATE) {
            float o[NT][4], s[2 * (kAttnC / 16)][4];
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[b][i] = 0.0f;
#pragma unroll
            for (int b = 0; b < kAttnC / 8; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[b][i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < KD / 16; ++kk) {
                uint32_t fq[NP][4];
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    attn_ldm(fq[i], tq + i * Tiles::kK + (warp * 16 + lane % 16) * PK + kk * 32 + lane / 16 * 16);
#pragma unroll
                for (int b = 0; b < NT / 2; ++b) {               // q S0
                    uint32_t b0[NP], b1[NP], b2[NP], b3[NP];
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        uint32_t f[4];
                        attn_ldm_t(f, smem + kStateAt + i * Tiles::kS + (kk * 16 + lane % 16) * PV + b * 32 + lane / 16 * 16);
                        b0[i] = f[0]; b1[i] = f[1]; b2[i] = f[2]; b3[i] = f[3];
                    }
                    attn_mma_pieces<NP == 3>(o[2 * b], fq, b0, b1);
                    attn_mma_pieces<NP == 3>(o[2 * b + 1], fq, b2, b3);
                }
#pragma unroll
                for (int b = 0; b < kAttnC / 16; ++b) {          // q k^T up to the diagonal
                    if (b <= warp) {
                        uint32_t b0[NP], b1[NP], b2[NP], b3[NP];
#pragma unroll
                        for (int i = 0; i < NP; ++i) {
                            uint32_t f[4];
                            attn_ldm(f, tk + i * Tiles::kK + (b * 16 + lane % 8 + lane / 16 * 8) * PK + kk * 32 + (lane >> 3 & 1) * 16);
                            b0[i] = f[0]; b1[i] = f[1]; b2[i] = f[2]; b3[i] = f[3];
                        }
                        attn_mma_pieces<NP == 3>(s[2 * b], fq, b0, b1);
                        attn_mma_pieces<NP == 3>(s[2 * b + 1], fq, b2, b3);
                    }
                }
            }
            const int i0 = warp * 16 + lane / 4;
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const float f0 = power[i0 + 1 - shift], f1 = power[i0 + 9 - shift];
                o[b][0] *= f0; o[b][1] *= f0; o[b][2] *= f1; o[b][3] *= f1;
            }
#pragma unroll
            for (int kk = 0; kk < kAttnC / 16; ++kk) {           // the weights, then their product with v
                if (kk <= warp) {
                    uint32_t fp[PP][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int back = i0 + (i >> 1) * 8 - (kk * 16 + h * 8 + n_first + (i & 1));
                            w[i] = back >= 0 ? s[2 * kk + h][i] * (power[max(back, 0)] * p.scale_in) : 0.0f;
                        }
                        uint32_t lo[PP], hi[PP];
                        attn_split(w[0], w[1], lo);
                        attn_split(w[2], w[3], hi);
#pragma unroll
                        for (int i = 0; i < PP; ++i) { fp[i][2 * h] = lo[i]; fp[i][2 * h + 1] = hi[i]; }
                    }
#pragma unroll
                    for (int b = 0; b < NT / 2; ++b) {
                        uint32_t b0[NP], b1[NP], b2[NP], b3[NP];
#pragma unroll
                        for (int i = 0; i < NP; ++i) {
                            uint32_t f[4];
                            attn_ldm_t(f, tv + i * Tiles::kV + (kk * 16 + lane % 16) * PV + b * 32 + lane / 16 * 16);
                            b0[i] = f[0]; b1[i] = f[1]; b2[i] = f[2]; b3[i] = f[3];
                        }
                        attn_mma_pieces<NP == 3>(o[2 * b], fp, b0, b1);
                        attn_mma_pieces<NP == 3>(o[2 * b + 1], fp, b2, b3);
                    }
                }
            }
            // out
            const long long row = row0 + static_cast<long long>(step) * c * kAttnC;
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = i0 + (i >> 1) * 8, col = n_first + b * 8 + (i & 1);
                    if (at < n && col < d2) {
                        const long long to = (row + step * at) * p.ld_out + static_cast<long long>(head) * p.d2 + slice * kAttnV + col;
                        if (p.out_f32) static_cast<float*>(p.out)[to] = o[b][i] * p.scale_out;
                        else static_cast<T*>(p.out)[to] = seq_from_float<T>(o[b][i] * p.scale_out);
                    }
                }
        }
        // the state behind the chunk
        const float all = power[n - shift];
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) st[a][b][i] *= all;
#pragma unroll
        for (int kk = 0; kk < kAttnC / 16; ++kk) {
            if (kk * 16 >= n) break;
            float w[4];                                          // of this thread's four rows of the 16
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int left = n - 1 - (kk * 16 + (i >> 1) * 8 + n_first + (i & 1));
                w[i] = left >= 0 ? power[max(left, 0)] * p.scale_in : 0.0f;
            }
            uint32_t fk[MT][UP][4];
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                uint32_t f[NP][4];
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    attn_ldm_t(f[i], tk + i * Tiles::kK + (kk * 16 + lane % 8 + lane / 16 * 8) * PK + (warp * (KD / 4) + a * 16 + (lane >> 3 & 1) * 8) * 2);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float lo = 0.0f, hi = 0.0f;
#pragma unroll
                    for (int i = NP - 1; i >= 0; --i) { lo += attn_lo(f[i][j]); hi += attn_hi(f[i][j]); }
                    uint32_t up[UP];
                    attn_split(lo * w[(j >> 1) * 2], hi * w[(j >> 1) * 2 + 1], up);
#pragma unroll
                    for (int i = 0; i < UP; ++i) fk[a][i][j] = up[i];
                }
            }
#pragma unroll
            for (int b = 0; b < NT / 2; ++b) {
                uint32_t b0[NP], b1[NP], b2[NP], b3[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    uint32_t f[4];
                    attn_ldm_t(f, tv + i * Tiles::kV + (kk * 16 + lane % 16) * PV + b * 32 + lane / 16 * 16);
                    b0[i] = f[0]; b1[i] = f[1]; b2[i] = f[2]; b3[i] = f[3];
                }
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    attn_mma_pieces<UP == 3>(st[a][2 * b], fk[a], b0, b1);
                    attn_mma_pieces<UP == 3>(st[a][2 * b + 1], fk[a], b2, b3);
                }
            }
        }
        __syncthreads();
        if (c + 1 < chunks) load(c + 1);
    }
    if (STATE) {
        float* to = p.carry + ((number * p.heads + head) * p.slices + slice) * carry_size;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(to + (m_first + a * 16 + h * 8) * kAttnV + n_first + b * 8) = make_float2(st[a][b][2 * h], st[a][b][2 * h + 1]);
    } else if (ends && p.state_out != nullptr && slot >= 0) {
        // the gradient of the state in front of the first row has one more decay than that of the state behind it
        const float f = p.back && r.len > 0 ? static_cast<float>(exp(log_l)) : 1.0f;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = m_first + a * 16 + (i >> 1) * 8, n = slice * kAttnV + n_first + b * 8 + (i & 1);
                    if (m < p.d1 && n < p.d2) p.state_out[state_at + m * p.s1 + n * p.s2] = st[a][b][i] * f;
                }
    }
}

// Gradients of shared heads: the sum over the heads that share one, in their order.  Rows of no sequence stay as they were.
template <typename T>
__global__ void __launch_bounds__(256) attn_share_kernel(long long batch, long long max_len, long long rows, const int* offsets, int own_heads, int share, int d,
                                                         const float* __restrict__ each, T* out, long long ld_out) {
    seq_grid_wait();
    const long long width = static_cast<long long>(own_heads) * d;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows * width; i += gridDim.x * 256ll) {
        const long long row = i / width;
        const int in = static_cast<int>(i - row * width), h = in / d, c = in - h * d;
        if (offsets != nullptr && !seq_has_row(offsets, batch, max_len, rows, row)) continue;
        const float* from = each + (row * own_heads + h) * share * d + c;
        float v = 0.0f;
        for (int s = 0; s < share; ++s) v += from[s * d];
        out[row * ld_out + in] = seq_from_float<T>(v);
    }
}

// One token: a block has one row of the batch and one head.  Threads lie along dim_v, VEC values each, and in groups along dim_k; the
// state goes through registers once, which is what bounds it (8 dim_k dim_v bytes a head).  128 rows, 32 heads of 64 x 64: 24.5 us for 128 MB
// (5.2 of the copy's 6.6 TB/s).
constexpr int kAttnStepThreads = 128;
template <typename T, int VEC>
__global__ void __launch_bounds__(kAttnStepThreads) attn_step_kernel(const __grid_constant__ AttnParams p) {
    __shared__ float part[kAttnStepThreads * VEC];
    seq_grid_wait();
    const int head = static_cast<int>(blockIdx.x % p.heads);
    const long long b = blockIdx.x / p.heads;
    const int across = (p.d2 + VEC - 1) / VEC, groups = max(1, kAttnStepThreads / across), tid = threadIdx.x;
    T* out = static_cast<T*>(p.out) + b * p.ld_out + static_cast<long long>(head) * p.d2;
    const long long slot = state_slot(p.slots, b, p.n_slots, p.status);
    if (slot < 0) {
        for (int c = tid; c < p.d2; c += kAttnStepThreads) out[c] = seq_from_float<T>(0.0f);
        return;
    }
    const long long at = slot * p.state_stride + static_cast<long long>(head) * p.d1 * p.d2;
    const float decay = expf(__ldg(p.log_decay + head));
    const T* q = static_cast<const T*>(p.q) + b * p.ld_q + head / p.q_share * p.d1;
    const T* k = static_cast<const T*>(p.k) + b * p.ld_k + head / p.k_share * p.d1;
    const T* v = static_cast<const T*>(p.v) + b * p.ld_v + head / p.v_share * p.d2;
    const int group = tid / across, c = (tid - group * across) * VEC;
    float sum[VEC], value[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        sum[i] = 0.0f;
        value[i] = group < groups ? seq_to_float(v[c + i]) : 0.0f;
    }
    if (group < groups) {
#pragma unroll 8
        for (int m = group; m < p.d1; m += groups) {
            SeqVec<float, VEC> s;
            s.bits = *reinterpret_cast<const typename SeqVec<float, VEC>::bits_t*>(p.state_in + at + static_cast<long long>(m) * p.d2 + c);
            const float key = seq_to_float(k[m]), query = seq_to_float(q[m]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s.v[i] = fmaf(key, value[i], decay * s.v[i]);
                sum[i] = fmaf(query, s.v[i], sum[i]);
            }
            *reinterpret_cast<typename SeqVec<float, VEC>::bits_t*>(p.state_out + at + static_cast<long long>(m) * p.d2 + c) = s.bits;
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (group < groups) part[group * across * VEC + c + i] = sum[i];
    __syncthreads();
    for (int j = tid; j < p.d2; j += kAttnStepThreads) {
        float t = 0.0f;
        for (int g = 0; g < groups; ++g) t += part[g * across * VEC + j];
        out[j] = seq_from_float<T>(t * p.scale_out);
    }
}

}  // namespace tdx
