// The sums of attention_kernels.cuh on tcgen05, for bf16 rows that the copy engine can read: chunks of 128 rows, one block a segment
// and head, the state in registers.
//
//   warp 0        copies: k and v of a chunk into one of two sets of tiles while the other is worked on, q as soon as the last one is used
//   warp 1        products: W = q k^T;  O1 = q S0;  O2 = P v;  U = K~^T v
//   warps 2 - 5   P = W l^(i-j) below the diagonal, bf16, back into tensor memory, from where it is a product's operand;
//                 out = l^(i+1) O1 + O2
//   warps 6 - 13  K~ = l^(n-1-j) k in bf16 pieces (the first in place of k); S1 = l^n S0 + U in fp32 registers, 64 a thread; S1 as bf16 for
//                 the next chunk's O1
//
// A chunk of 128 x 128 takes about 5,500 cycles of an SM's share of the memory bandwidth and about 2,600 cycles of products, so one
// chunk at a time with its operands fetched ahead is enough.  U starts from zero in every chunk: the tensor cores cut sums off instead of
// rounding them, which over a whole sequence shows in the state (3e-6), over 128 rows it does not.
// Rows of the tile behind the chunk's last one belong to other rows of the sequence or to other sequences: their weights are selected
// to zero, not multiplied, and their rows of v are set to zero in shared memory.
#pragma once
#include "attention_kernels.cuh"
#include "bounded_wait.cuh"

namespace tdx {

constexpr int kAttnRows = 128;                                   // rows of a chunk here
constexpr int kAttnTile = 128 * 256;                             // bytes of 128 rows of 128 bf16, as two halves of 64 columns
constexpr int kAttnHalf = kAttnTile / 2;
constexpr int kAttnUmmaThreads = 14 * 32;
enum : uint32_t { kAttnTmemW = 0, kAttnTmemO1 = 128, kAttnTmemO2 = 256, kAttnTmemU = 384 };

// D[tmem] (+)= A[tmem] * B[smem desc]: A's rows are lanes, its columns bf16 pairs
__device__ __forceinline__ void attn_umma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void attn_tmem_st_x16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void attn_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <bool STATE, int UP>
struct AttnUmma {
    static constexpr int kSets = STATE || UP == 2 ? 2 : 1;        // of k and v
    static constexpr int kQ = 0, kState = STATE ? 0 : kAttnTile, kKv = STATE ? 0 : 2 * kAttnTile, kLow = kKv + kSets * 2 * kAttnTile;
    static constexpr int kBytes = kLow + (UP - 1) * kAttnTile;
};

template <bool STATE, int UP>
__global__ void __launch_bounds__(kAttnUmmaThreads, 1)
    attn_umma_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ AttnParams p) {
    typedef AttnUmma<STATE, UP> Lay;
    extern __shared__ uint8_t attn_raw[];
    __shared__ __align__(8) uint64_t full_q, free_q, full_kv[2], free_kv[2], bar_w, bar_p, bar_k, bar_o, bar_u, bar_state, bar_o_free;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ float power[kAttnRows + 1], weight[2 * kAttnRows];  // l^n; weight[128 + n] = scale_in l^n, 0 for negative n
    volatile int* abort_flag = &s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* const smem = attn_raw + ((1024u - (ptx::smem_u32(attn_raw) & 1023u)) & 1023u);

    if (tid == 0) {
        ptx::mbar_init(&full_q, 1); ptx::mbar_init(&free_q, 1);
        for (int i = 0; i < 2; ++i) { ptx::mbar_init(&full_kv[i], 1); ptx::mbar_init(&free_kv[i], 1); }
        ptx::mbar_init(&bar_w, 1); ptx::mbar_init(&bar_p, 4); ptx::mbar_init(&bar_k, 8); ptx::mbar_init(&bar_o, 1); ptx::mbar_init(&bar_u, 1);
        ptx::mbar_init(&bar_state, 8); ptx::mbar_init(&bar_o_free, 4);
        s_abort = 0;
        ptx::fence_barrier_init();
        if (!STATE) ptx::tma_prefetch_desc(&tm_q);
        ptx::tma_prefetch_desc(&tm_k);
        ptx::tma_prefetch_desc(&tm_v);
    }
    seq_grid_wait();
    const int head = static_cast<int>(blockIdx.x % p.heads);
    const long long number = blockIdx.x / p.heads;
    if (!STATE && head == 0) seq_check(p.offsets, number, p.batch, p.max_len, p.rows, p.status);
    const SeqPiece piece = seq_piece(p.offsets, p.batch, p.dense, p.seg, number);
    const SeqRange r = seq_range(p.offsets, piece.b, p.max_len, p.rows, p.status);
    const long long start = piece.index * p.seg;
    const long long slot = !STATE && (p.state_in != nullptr || p.state_out != nullptr) ? state_slot(p.slots, piece.b, p.n_slots, p.status) : -1;
    const long long state_at = slot * p.state_stride + static_cast<long long>(head) * p.d1 * p.d2;
    const bool ends = start + p.seg >= r.len;
    if (start >= r.len && !(piece.index == 0 && !STATE)) return;
    if (STATE && ends) return;
    const int count = static_cast<int>(ends ? r.len - start : p.seg);
    const int chunks = (count + kAttnRows - 1) / kAttnRows;
    const int less = p.back && piece.index == 0 ? 1 : 0;         // see attn_kernel
    const double log_l = static_cast<double>(__ldg(p.log_decay + head));
    if (tid <= kAttnRows) power[tid] = tid == 0 ? 1.0f : static_cast<float>(exp(log_l * tid));
    if (tid < kAttnRows) {
        weight[tid] = 0.0f;
        weight[kAttnRows + tid] = (tid == 0 ? 1.0f : static_cast<float>(exp(log_l * tid))) * p.scale_in;
    }
    // rows of K~ that stand for columns of k behind d1 are never written again
    if (p.d1 <= 64) {
        for (int s = 0; s < Lay::kSets; ++s)
            for (int i = tid; i < kAttnHalf / 16; i += kAttnUmmaThreads) *reinterpret_cast<uint4*>(smem + Lay::kKv + s * 2 * kAttnTile + kAttnHalf + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        for (int s = 0; s < UP - 1; ++s)
            for (int i = tid; i < kAttnHalf / 16; i += kAttnUmmaThreads) *reinterpret_cast<uint4*>(smem + Lay::kLow + s * kAttnTile + kAttnHalf + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        ptx::fence_proxy_async_smem();
    }
    if (warp == 1) {
        __syncwarp();
        ptx::tmem_alloc(&s_tmem, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    // chunk c has the rows first .. first + n - 1 in their own order, whatever the direction is
    const long long row0 = r.first + (p.back ? r.len - start : start);
    auto rows_of = [&](int c) { return min(kAttnRows, count - c * kAttnRows); };
    auto first_of = [&](int c) { return p.back ? row0 - static_cast<long long>(c) * kAttnRows - rows_of(c) : row0 + static_cast<long long>(c) * kAttnRows; };
    const int steps1 = (p.d1 + 15) / 16, halves1 = (p.d1 + 63) / 64, halves2 = (p.d2 + 63) / 64, n2 = (p.d2 + 15) / 16 * 16;

    if (warp == 0) {
        if (ptx::elect_one()) {
            const int hq = head / p.q_share, hk = head / p.k_share, hv = head / p.v_share;
            bool ok = true;
            for (int c = 0; ok && c < chunks; ++c) {
                const int row = static_cast<int>(first_of(c)), set = c % Lay::kSets, use = c / Lay::kSets;
                if (!STATE) {
                    if (c > 0 && !wait_bounded(&free_q, (c - 1) & 1, abort_flag, p.status, kTimeoutProducer)) { ok = false; break; }
                    ptx::mbar_arrive_expect_tx(&full_q, halves1 * kAttnHalf);
                    for (int h = 0; h < halves1; ++h) ptx::tma_load_3d(smem + Lay::kQ + h * kAttnHalf, &tm_q, &full_q, h * 64, hq, row);
                }
                if (use > 0 && !wait_bounded(&free_kv[set], (use - 1) & 1, abort_flag, p.status, kTimeoutProducer)) { ok = false; break; }
                uint8_t* kv = smem + Lay::kKv + set * 2 * kAttnTile;
                ptx::mbar_arrive_expect_tx(&full_kv[set], (halves1 + halves2) * kAttnHalf);
                for (int h = 0; h < halves1; ++h) ptx::tma_load_3d(kv + h * kAttnHalf, &tm_k, &full_kv[set], h * 64, hk, row);
                for (int h = 0; h < halves2; ++h) ptx::tma_load_3d(kv + kAttnTile + h * kAttnHalf, &tm_v, &full_kv[set], h * 64, hv, row);
            }
            if (!ok) {
                // let copies that are still in flight land before the block goes away
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        }
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t base = ptx::smem_u32(smem);
            // K-major operands: 16 of the reduction are 32 bytes further in a 128-byte row, 64 are a half tile; others: 16 rows of 128 bytes
            auto k_major = [&](uint32_t at, int step) { return ptx::make_smem_desc_sw128(at + (step >> 2) * kAttnHalf + (step & 3) * 32, 16u, 1024u); };
            auto mn_major = [&](uint32_t at, int step) { return ptx::make_smem_desc_sw128(at + step * 2048, kAttnHalf, 1024u); };
            const uint32_t idesc_w = ptx::make_idesc_bf16_f32(128, 128, 0, 0), idesc_o = ptx::make_idesc_bf16_f32(128, n2, 0, 1),
                           idesc_u = ptx::make_idesc_bf16_f32(128, n2, 1, 1);
            bool ok = true;
            auto wait = [&](uint64_t* bar, int use) { return ok = ok && wait_bounded(bar, use & 1, abort_flag, p.status, kTimeoutMma); };
            for (int c = 0; ok && c < chunks; ++c) {
                const int set = c % Lay::kSets;
                const uint32_t k = base + Lay::kKv + set * 2 * kAttnTile, v = k + kAttnTile;
                if (!wait(&full_kv[set], c / Lay::kSets)) break;
                if (!STATE) {
                    // (W takes the place of P, which O2 of the chunk before has to be done with)
                    if (!wait(&full_q, c) || (c > 0 && !wait(&bar_o, c - 1))) break;
                    ptx::tc_fence_after_sync();
                    for (int s = 0; s < steps1; ++s) ptx::umma_bf16(tmem + kAttnTmemW, k_major(base + Lay::kQ, s), k_major(k, s), idesc_w, s > 0);
                    ptx::umma_commit(&bar_w);
                    if (!wait(&bar_state, c) || (c > 0 && !wait(&bar_o_free, c - 1))) break;
                    ptx::tc_fence_after_sync();
                    for (int s = 0; s < steps1; ++s) ptx::umma_bf16(tmem + kAttnTmemO1, k_major(base + Lay::kQ, s), mn_major(base + Lay::kState, s), idesc_o, s > 0);
                    ptx::umma_commit(&free_q);
                }
                if (!wait(&bar_k, c) || (!STATE && !wait(&bar_p, c))) break;
                ptx::tc_fence_after_sync();
                if (!STATE) {
                    for (int s = 0; s < 8; ++s) attn_umma_ta(tmem + kAttnTmemO2, tmem + kAttnTmemW + s * 8, mn_major(v, s), idesc_o, s > 0);
                    ptx::umma_commit(&bar_o);
                }
                for (int u = UP - 1; u >= 0; --u) {              // small terms first
                    const uint32_t from = u == 0 ? k : base + Lay::kLow + (u - 1) * kAttnTile;
                    for (int s = 0; s < 8; ++s) ptx::umma_bf16(tmem + kAttnTmemU, mn_major(from, s), mn_major(v, s), idesc_u, u < UP - 1 || s > 0);
                }
                ptx::umma_commit(&free_kv[set]);
                ptx::umma_commit(&bar_u);
            }
        }
    } else if (warp < 6) {
        if (!STATE) {
            const int quarter = warp & 3, i = quarter * 32 + lane;
            const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
            for (int c = 0; c < chunks; ++c) {
                const int n = rows_of(c), shift = c == 0 ? less : 0;
                if (!wait_bounded(&bar_w, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
                ptx::tc_fence_after_sync();
#pragma unroll 1
                for (int g = 0; g < 4; ++g) {
                    uint32_t packed[16];
                    if (p.back ? g < quarter : g > quarter) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) packed[j] = 0u;
                    } else {
                        uint32_t w[32];
                        ptx::tmem_ld_32x32b_x32(tmem + lanes + kAttnTmemW + g * 32, w);
                        ptx::tmem_ld_wait();
                        float f[32];
                        if (p.back) {
                            const float* at = weight + kAttnRows + g * 32 - i;
#pragma unroll
                            for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(w[j]) * at[j];
                            if (g == quarter || n < kAttnRows) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) f[j] = g * 32 + j >= i && g * 32 + j < n ? f[j] : 0.0f;
                            }
                        } else {
                            const float* at = weight + kAttnRows + i - g * 32;
#pragma unroll
                            for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(w[j]) * at[-j];
                            if (g == quarter) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) f[j] = g * 32 + j <= i ? f[j] : 0.0f;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) packed[j] = attn_pair(f[2 * j], f[2 * j + 1]);
                    }
                    // columns 16 g and up: nothing of W that is still to be read
                    attn_tmem_st_x16(tmem + lanes + kAttnTmemW + g * 16, packed);
                }
                attn_tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&bar_p);
                if (!wait_bounded(&bar_o, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
                ptx::tc_fence_after_sync();
                const float far = (i < n ? power[p.back ? n - i - shift : i + 1 - shift] : 0.0f) * p.scale_out;
                const long long to = (first_of(c) + i) * p.ld_out + static_cast<long long>(head) * p.d2;
#pragma unroll 1
                for (int g = 0; g * 32 < p.d2; ++g) {
                    uint32_t o1[32], o2[32];
                    ptx::tmem_ld_32x32b_x32(tmem + lanes + kAttnTmemO1 + g * 32, o1);
                    ptx::tmem_ld_32x32b_x32(tmem + lanes + kAttnTmemO2 + g * 32, o2);
                    ptx::tmem_ld_wait();
                    float f[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = fmaf(__uint_as_float(o1[j]), far, __uint_as_float(o2[j]) * p.scale_out);
                    if (i < n) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (g * 32 + j * 8 < p.d2) {
                                if (p.out_f32) {
                                    float4* at = reinterpret_cast<float4*>(static_cast<float*>(p.out) + to + g * 32 + j * 8);
                                    at[0] = make_float4(f[8 * j], f[8 * j + 1], f[8 * j + 2], f[8 * j + 3]);
                                    at[1] = make_float4(f[8 * j + 4], f[8 * j + 5], f[8 * j + 6], f[8 * j + 7]);
                                } else {
                                    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + to + g * 32 + j * 8) =
                                        make_uint4(attn_pair(f[8 * j], f[8 * j + 1]), attn_pair(f[8 * j + 2], f[8 * j + 3]), attn_pair(f[8 * j + 4], f[8 * j + 5]), attn_pair(f[8 * j + 6], f[8 * j + 7]));
                                }
                            }
                        }
                    }
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&bar_o_free);
            }
        }
    } else {
        // this thread's part of the state: row m, columns 64 side and up
        const int quarter = warp & 3, side = (warp - 6) >> 2, m = quarter * 32 + lane, worker = tid - 6 * 32;
        const bool mine = side < halves2;
        float st[64];
        const long long carry_size = kAttnRows * kAttnRows, carry_step = carry_size * p.heads;
        float* const carry = p.carry + (number * p.heads + head) * carry_size + static_cast<long long>(side) * 64 * kAttnRows + m;
#pragma unroll
        for (int j = 0; j < 64; ++j) {
            const int n = side * 64 + j;
            st[j] = !STATE && p.state_in != nullptr && slot >= 0 && m < p.d1 && n < p.d2 ? __ldg(p.state_in + state_at + static_cast<long long>(m) * p.s1 + static_cast<long long>(n) * p.s2) : 0.0f;
        }
        if (!STATE && piece.index > 0 && mine) {
            const float all = static_cast<float>(exp(log_l * static_cast<double>(p.seg))), first = p.back ? static_cast<float>(exp(log_l * static_cast<double>(p.seg - 1))) : all;
            for (int s = 0; s < piece.index; ++s) {
                const float* from = carry + (s - piece.index) * carry_step;
                const float f = s == 0 ? first : all;
#pragma unroll
                for (int j = 0; j < 64; ++j) st[j] = fmaf(st[j], f, from[j * kAttnRows]);
            }
        }
        // the state in front of a chunk, rounded to bf16 for its product with q
        auto publish = [&]() {
            if (mine) {
#pragma unroll
                for (int g = 0; g < 8; ++g)
                    *reinterpret_cast<uint4*>(smem + Lay::kState + side * kAttnHalf + m * 128 + ((g ^ (m & 7)) << 4)) =
                        make_uint4(attn_pair(st[8 * g], st[8 * g + 1]), attn_pair(st[8 * g + 2], st[8 * g + 3]), attn_pair(st[8 * g + 4], st[8 * g + 5]), attn_pair(st[8 * g + 6], st[8 * g + 7]));
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bar_state);
        };
        if (!STATE && chunks > 0) publish();
        for (int c = 0; c < chunks; ++c) {
            const int n = rows_of(c), shift = c == 0 ? less : 0, set = c % Lay::kSets;
            if (!wait_bounded(&full_kv[set], (c / Lay::kSets) & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            // q k^T has been read from k before it is overwritten
            if (!STATE && !wait_bounded(&bar_w, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            uint8_t* const k = smem + Lay::kKv + set * 2 * kAttnTile;
            for (int at = worker; at < halves1 * (kAttnHalf / 16); at += 256) {
                const int row = at / 8 % kAttnRows;
                const float w = weight[kAttnRows + (p.back ? row : n - 1 - row)];
                const uint4 v = *reinterpret_cast<const uint4*>(k + at * 16);
                const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                uint32_t out[UP][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t up[UP];
                    attn_split(attn_lo(in[j]) * w, attn_hi(in[j]) * w, up);
#pragma unroll
                    for (int u = 0; u < UP; ++u) out[u][j] = row < n ? up[u] : 0u;
                }
#pragma unroll
                for (int u = 0; u < UP; ++u)
                    *reinterpret_cast<uint4*>((u == 0 ? k : smem + Lay::kLow + (u - 1) * kAttnTile) + at * 16) = make_uint4(out[u][0], out[u][1], out[u][2], out[u][3]);
            }
            if (n < kAttnRows) {
                for (int h = 0; h < halves2; ++h)
                    for (int at = worker; at < (kAttnRows - n) * 8; at += 256) *reinterpret_cast<uint4*>(k + kAttnTile + h * kAttnHalf + n * 128 + at * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bar_k);
            if (!wait_bounded(&bar_u, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            ptx::tc_fence_after_sync();
            if (mine) {
                const float f = power[n - shift];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    uint32_t u[32];
                    ptx::tmem_ld_32x32b_x32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + kAttnTmemU + side * 64 + g * 32, u);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) st[g * 32 + j] = fmaf(st[g * 32 + j], f, __uint_as_float(u[j]));
                }
            }
            ptx::tc_fence_before_sync();
            // (without q the next chunk's products wait for bar_k, which comes after this read)
            if (!STATE && c + 1 < chunks) publish();
        }
        if (STATE) {
            if (mine) {
#pragma unroll
                for (int j = 0; j < 64; ++j) carry[j * kAttnRows] = st[j];
            }
        } else if (ends && p.state_out != nullptr && slot >= 0 && m < p.d1) {
            const float f = p.back && r.len > 0 ? static_cast<float>(exp(log_l)) : 1.0f;   // see attn_kernel
#pragma unroll
            for (int j = 0; j < 64; ++j)
                if (side * 64 + j < p.d2) p.state_out[state_at + static_cast<long long>(m) * p.s1 + static_cast<long long>(side * 64 + j) * p.s2] = st[j] * f;
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        __syncwarp();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace tdx
