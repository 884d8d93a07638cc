// The sums of attention_kernels.cuh on tcgen05, for bf16 rows that the copy engine can read: chunks of 128 rows, one block a segment
// and head, the state in registers.
//
//   warp 0         copies: k and v of a chunk into one of two sets of tiles while the other is worked on, q as soon as the last one is used
//   warp 1         products: W = q k^T;  O1 = q S0;  O2 = P v;  U = K~^T v
//   warps 4 - 11   P = W l^(i-j) below the diagonal in two bf16 pieces, back into tensor memory, from where they are a product's
//                  operands; then out = l^(i+1) O1 + O2
//   warps 12 - 15  K~ = l^(n-1-j) k in bf16 pieces, the first in place of k (warps 4 - 15 where there are no outputs)
//   warps 16 - 23  S1 = l^n S0 + U in fp32 registers, 64 a thread; S1 as bf16 for the next chunk's O1
//
// The roles are apart so that a chunk's K~ and W are made while the state and the output of the one in front of it are still worked on:
// with P and out in four warps and K~ and the state in the same eight a chunk of 128 x 128 took 7,700 cycles.  Registers move from
// the first four warps and the keys' to the state's.
// The second piece of P costs 8 % (forward and backward of 4 x 2048 rows, 16 heads of 128: 218 -> 236 us) and takes the larger of the two
// roundings on the way to the output out (P's and the state's): 1.4 times the error of a single rounding became 1.0 to 1.3 times.
//
// Measured, bf16, heads of 128: one prompt of 4096 rows with 32 heads 83 us (171 with the kernel on mma.sync), forward and backward of 4 x
// 2048 rows with 16 heads 236 us (577).  The schedulers issue in 38 to 40 % of the cycles and memory runs at 28 to 30 % of its rate: a chunk
// of 4 us is the chain W, P, O2, out and the chain of states from one chunk to the next.
// A chunk of 128 x 128 takes about 5,500 cycles of an SM's share of the memory bandwidth and about 3,100 cycles of products, so one
// chunk at a time with its operands fetched ahead is enough.  U starts from zero in every chunk: the tensor cores cut sums off instead of
// rounding them, which over a whole sequence shows in the state (3e-6), over 128 rows it does not.
// Rows of the tile behind the chunk's last one belong to other rows of the sequence or to other sequences: their weights are selected
// to zero, not multiplied, and their rows of v are set to zero in shared memory.
#pragma once
#include "attention_kernels.cuh"
#include "bounded_wait.cuh"

#include <limits.h>

namespace tdx {

constexpr int kAttnRows = 128;                                   // rows of a chunk here
constexpr int kAttnTile = 128 * 256;                             // bytes of 128 rows of 128 bf16, as two halves of 64 columns
constexpr int kAttnHalf = kAttnTile / 2;
constexpr int kAttnUmmaThreads = 24 * 32;
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
// 32 bytes in one access (a thread has a row of its own: half as many lines per byte to look up as with 16)
__device__ __forceinline__ void attn_store_32(void* to, const uint32_t* r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void attn_prefetch(const __nv_bfloat16* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// Registers of a warpgroup; 768 threads are launched with 80 each, and 128 * (40 + 2 * 88 + 56 + 2 * 104) of them are asked for,
// which is as many.
template <int N>
__device__ __forceinline__ void attn_fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void attn_more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void attn_tmem_ld_x16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void attn_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// d (+)= a b over `steps` of 16 of the reduction; A1, B1: descriptor units a step, A4, B4: four steps
template <uint64_t A1, uint64_t A4, uint64_t B1, uint64_t B4>
__device__ __forceinline__ void attn_products(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, int steps, uint32_t accumulate) {
#pragma unroll 1
    for (int s = 0; s < steps; s += 4, a += A4, b += B4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (s + j < steps) {
                ptx::umma_bf16(d, a + j * A1, b + j * B1, idesc, accumulate);
                accumulate = 1u;
            }
    }
}

// Tiles in shared memory: two of k and (where there is room) v, which are in use until a chunk's U, one of q, which is free after O1.  (Two of q
// and one of v, and W of the next chunk in front of U, took 5.2 us a chunk of 128 x 128 instead of 4.0.)
template <bool STATE, int UP>
struct AttnUmma {
    static constexpr int kQs = STATE ? 0 : 1, kVs = STATE || UP == 2 ? 2 : 1;
    static constexpr int kQ = 0, kState = kQ + kQs * kAttnTile, kK = kState + (STATE ? 0 : kAttnTile), kV = kK + 2 * kAttnTile, kLow = kV + kVs * kAttnTile;
    static constexpr int kBytes = kLow + (UP - 1) * kAttnTile;
};

template <bool STATE, bool BACK, int UP>
__global__ void __launch_bounds__(kAttnUmmaThreads, 1)
    attn_umma_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const __grid_constant__ AttnParams p) {
    typedef AttnUmma<STATE, UP> Lay;
    extern __shared__ uint8_t attn_raw[];
    __shared__ __align__(8) uint64_t full_q[2], free_q[2], full_k[2], free_k[2], full_v[2], free_v[2], bar_w[2], bar_p, bar_k, bar_o, bar_u, bar_state, bar_o_free;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_progress;
    __shared__ float power[kAttnRows + 1], weight[2 * kAttnRows];  // l^n; weight[128 + n] = scale_in l^n, 0 for negative n
    volatile int *abort_flag = &s_abort, *progress = &s_progress;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* const smem = attn_raw + ((1024u - (ptx::smem_u32(attn_raw) & 1023u)) & 1023u);

    if (tid == 0) {
        for (int i = 0; i < 2; ++i)
            for (uint64_t* bar : {&full_q[i], &free_q[i], &full_k[i], &free_k[i], &full_v[i], &free_v[i]}) ptx::mbar_init(bar, 1);
        ptx::mbar_init(&bar_w[0], 1); ptx::mbar_init(&bar_w[1], 1); ptx::mbar_init(&bar_p, 8); ptx::mbar_init(&bar_k, STATE ? 12 : 4); ptx::mbar_init(&bar_o, 1); ptx::mbar_init(&bar_u, 1);
        ptx::mbar_init(&bar_state, 8); ptx::mbar_init(&bar_o_free, 8);
        s_abort = s_progress = 0;
        ptx::fence_barrier_init();
        if (!STATE) ptx::tma_prefetch_desc(&tm_q);
        ptx::tma_prefetch_desc(&tm_k);
        ptx::tma_prefetch_desc(&tm_v);
    }
    seq_launch_dependents();
    seq_grid_wait();
    const int head = static_cast<int>(blockIdx.x % p.heads);
    const long long number = blockIdx.x / p.heads;
    if (!STATE && head == 0) seq_check(p.offsets, number, p.batch, p.max_len, p.rows, p.status);
    // segments, or for the pass over the states the shorter pieces that it cuts them into
    const long long seg = STATE ? p.sub : p.seg;
    const SeqPiece piece = STATE ? attn_slot_piece(p, number) : seq_piece(p.offsets, p.batch, p.dense, seg, number);
    const SeqRange r = seq_range(p.offsets, piece.b, p.max_len, p.rows, p.status);
    const long long start = piece.index * seg;
    const long long slot = !STATE && (p.state_in != nullptr || p.state_out != nullptr) ? state_slot(p.slots, piece.b, p.n_slots, p.status) : -1;
    const long long state_at = slot * p.state_stride + static_cast<long long>(head) * p.d1 * p.d2;
    const bool ends = start + seg >= r.len;
    if (start >= r.len && !(piece.index == 0 && !STATE)) return;
    // of a sequence that has no slots, or in the last segment: nobody asks for it
    if (STATE && ((!p.every && r.len <= p.seg) || (!p.all_pieces && start / p.seg == (r.len - 1) / p.seg))) return;
    const int count = static_cast<int>(ends ? r.len - start : seg);
    const int chunks = (count + kAttnRows - 1) / kAttnRows;
    const int less = BACK && piece.index == 0 ? 1 : 0;         // see attn_kernel
    const double log_l = static_cast<double>(__ldg(p.log_decay + head));
    const long long row0 = r.first + (BACK ? r.len - start : start);
    auto rows_of = [&](int c) { return min(kAttnRows, count - c * kAttnRows); };
    // Chunk c has the rows first_of(c) .. + rows_of(c) - 1 in their own order, whatever the direction is.
    auto first_of = [&](int c) { return BACK ? row0 - static_cast<long long>(c) * kAttnRows - rows_of(c) : row0 + static_cast<long long>(c) * kAttnRows; };
    const int steps1 = (p.d1 + 15) / 16, halves1 = (p.d1 + 63) / 64, halves2 = (p.d2 + 63) / 64, n2 = (p.d2 + 15) / 16 * 16;
    // copies of a chunk's tiles, by one thread
    const int hq = head / p.q_share, hk = head / p.k_share, hv = head / p.v_share;
    auto copy_k = [&](int c) {
        uint64_t* bar = &full_k[c & 1];
        ptx::mbar_arrive_expect_tx(bar, halves1 * kAttnHalf);
        for (int h = 0; h < halves1; ++h) ptx::tma_load_3d(smem + Lay::kK + (c & 1) * kAttnTile + h * kAttnHalf, &tm_k, bar, h * 64, hk, static_cast<int>(first_of(c)));
    };
    auto copy_q = [&](int c) {
        const int set = c % max(Lay::kQs, 1);
        ptx::mbar_arrive_expect_tx(&full_q[set], halves1 * kAttnHalf);
        for (int h = 0; h < halves1; ++h) ptx::tma_load_3d(smem + Lay::kQ + set * kAttnTile + h * kAttnHalf, &tm_q, &full_q[set], h * 64, hq, static_cast<int>(first_of(c)));
    };
    auto copy_v = [&](int c) {
        const int set = c % Lay::kVs;
        ptx::mbar_arrive_expect_tx(&full_v[set], halves2 * kAttnHalf);
        for (int h = 0; h < halves2; ++h) ptx::tma_load_3d(smem + Lay::kV + set * kAttnTile + h * kAttnHalf, &tm_v, &full_v[set], h * 64, hv, static_cast<int>(first_of(c)));
    };
    if (tid == 0 && chunks > 0) {                                // under way while the others make the tables
        copy_k(0);
        if (!STATE) copy_q(0);
        copy_v(0);
    }
    if (tid >= 32 && tid <= 32 + kAttnRows) {
        const int n = tid - 32;
        const float l = n == 0 ? 1.0f : static_cast<float>(exp(log_l * n));
        power[n] = l;
        if (n < kAttnRows) {
            weight[n] = 0.0f;
            weight[kAttnRows + n] = l * p.scale_in;
        }
    }
    // rows of K~ that stand for columns of k behind d1 are never written again
    if (p.d1 <= 64) {
        for (int s = 0; s < 2; ++s)
            for (int i = tid; i < kAttnHalf / 16; i += kAttnUmmaThreads) *reinterpret_cast<uint4*>(smem + Lay::kK + s * kAttnTile + kAttnHalf + i * 16) = make_uint4(0u, 0u, 0u, 0u);
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
    // Each barrier completes once a chunk (those of a set of tiles once a use of the set).  A wait goes by the parity, so it must not begin before the
    // completion in front of the one that it is for.  Most waiters wait for every completion; W runs a chunk ahead of the keys' warps and has
    // two barriers; the keys' warps wait for v only where the chunk is short, behind bar_u, which says that the v in front was there.
    if (warp < 4) {
        attn_fewer_registers<40>();
        if (warp == 0) {
            bool ok = true;
            auto wait = [&](uint64_t* bar, int use) { return ok = ok && (use < 0 || wait_bounded_idle(bar, use & 1, abort_flag, p.status, kTimeoutProducer)); };
            constexpr int kQs = Lay::kQs > 0 ? Lay::kQs : 1, kVs = Lay::kVs;
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                // in the order in which the tiles become free
                if (c > 0) {
                    if (!wait(&free_k[c & 1], c / 2 - 1)) break;
                    if (ptx::elect_one()) copy_k(c);
                    if (kVs == 2) {
                        if (!wait(&free_v[c & 1], c / 2 - 1)) break;
                        if (ptx::elect_one()) copy_v(c);
                    }
                    __syncwarp();
                }
                if (lane == 0) *progress = c + 1;
                if (c > 0) {
                    if (!STATE) {
                        if (!wait(&free_q[c % kQs], c / kQs - 1)) break;
                        if (ptx::elect_one()) copy_q(c);
                    }
                    if (kVs == 1) {
                        if (!wait(&free_v[0], c - 1)) break;
                        if (ptx::elect_one()) copy_v(c);
                    }
                    __syncwarp();
                }
            }
            if (lane == 0) *progress = INT_MAX;
            if (!ok) {
                // let copies that are still in flight land before the block goes away
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        } else if (warp == 2) {
            // The chunk after next on its way into L2 once chunk c's copies are asked for: the tiles alone leave a copy one chunk's time.  (Asked for
            // by the copy engine it would stand in front of the copies.)  The copies' warp says how far it is, at its end that it is done.
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + hq * p.d1;
            const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(p.k) + hk * p.d1;
            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + hv * p.d2;
#pragma unroll 1
            for (int c = 0; c + 2 < chunks; ++c) {
                for (int turn = 0; *progress <= c && turn < 1 << 24; ++turn) __nanosleep(100);
                const long long ahead = first_of(c + 2);
                const int n = rows_of(c + 2);
                for (int i = lane; i < n; i += 32) {
                    for (int h = 0; h < halves1; ++h) {
                        attn_prefetch(k + (ahead + i) * p.ld_k + h * 64);
                        if (!STATE) attn_prefetch(q + (ahead + i) * p.ld_q + h * 64);
                    }
                    for (int h = 0; h < halves2; ++h) attn_prefetch(v + (ahead + i) * p.ld_v + h * 64);
                }
            }
        } else if (warp == 1) {
            if (ptx::elect_one()) {
                const uint32_t base = ptx::smem_u32(smem);
                // Steps of 16 of the reduction, in 16-byte units: K-major operands are 32 bytes further in a 128-byte row, 64 of the reduction are a
                // half tile; the others 16 rows of 128 bytes further.  Loops stay loops: unrolled, the roles' code together did not fit
                // the instruction caches, and every step of this thread waited for its instructions.
                auto k_major = [&](uint32_t at) { return ptx::make_smem_desc_sw128(at, 16u, 1024u); };
                auto mn_major = [&](uint32_t at) { return ptx::make_smem_desc_sw128(at, kAttnHalf, 1024u); };
                constexpr uint64_t kK1 = 32 >> 4, kK4 = kAttnHalf >> 4, kMn1 = 2048 >> 4, kMn4 = 4 * kMn1;
                const uint32_t idesc_w = ptx::make_idesc_bf16_f32(128, 128, 0, 0), idesc_o = ptx::make_idesc_bf16_f32(128, n2, 0, 1),
                               idesc_u = ptx::make_idesc_bf16_f32(128, n2, 1, 1);
                bool ok = true;
                auto wait = [&](uint64_t* bar, int use) { return ok = ok && wait_bounded_idle(bar, use & 1, abort_flag, p.status, kTimeoutMma); };
                constexpr int kQs = Lay::kQs > 0 ? Lay::kQs : 1, kVs = Lay::kVs;
#pragma unroll 1
                for (int c = STATE ? 0 : -1; ok && c < chunks; ++c) {
                    const uint32_t k = base + Lay::kK + (c & 1) * kAttnTile, v = base + Lay::kV + (c & (kVs - 1)) * kAttnTile;
                    if (!STATE && c >= 0) {
                        // (the state in front of the chunk is there, and U has been read)
                        if (!wait(&bar_state, c) || (c > 0 && !wait(&bar_o_free, c - 1))) break;
                        ptx::tc_fence_after_sync();
                        attn_products<kK1, kK4, kMn1, kMn4>(tmem + kAttnTmemO1, k_major(base + Lay::kQ + c % kQs * kAttnTile), mn_major(base + Lay::kState), idesc_o, steps1, 0u);
                        ptx::umma_commit(&free_q[c % kQs]);
                        // (the keys' warps set the rows of v behind a short chunk to zero)
                        if (!wait(&full_v[c % kVs], c / kVs) || !wait(&bar_p, c) || (rows_of(c) < kAttnRows && !wait(&bar_k, c))) break;
                        ptx::tc_fence_after_sync();
                        const uint64_t of_v = mn_major(v);
#pragma unroll 1
                        for (int s = 0; s < 16; ++s)             // second pieces first
                            attn_umma_ta(tmem + kAttnTmemO2, tmem + kAttnTmemW + (s >> 2 & 1) * 64 + (s < 8 ? 32 : 0) + (s & 3) * 8, of_v + (s & 7) * kMn1, idesc_o, s > 0);
                        ptx::umma_commit(&bar_o);
                    }
                    if (c >= 0) {
                    if (STATE && (!wait(&full_k[c & 1], c / 2) || !wait(&full_v[c % kVs], c / kVs) || !wait(&bar_state, c))) break;
                    if (!wait(&bar_k, c)) break;
                    ptx::tc_fence_after_sync();
#pragma unroll 1
                    for (int u = UP - 1; u >= 0; --u)                // small terms first
                        attn_products<kMn1, kMn4, kMn1, kMn4>(tmem + kAttnTmemU, mn_major(u == 0 ? k : base + Lay::kLow + (u - 1) * kAttnTile), mn_major(v), idesc_u, 8, u < UP - 1);
                    ptx::umma_commit(&free_k[c & 1]);
                    ptx::umma_commit(&free_v[c % kVs]);
                    ptx::umma_commit(&bar_u);
                    }
                    if (!STATE && c + 1 < chunks) {
                        // the next chunk's W: its k and q are there, and O2 is done with P, whose place W takes
                        const int next = c + 1;
                        if (!wait(&full_k[next & 1], next / 2) || !wait(&full_q[next % kQs], next / kQs) || (c >= 0 && !wait(&bar_o, c))) break;
                        ptx::tc_fence_after_sync();
                        attn_products<kK1, kK4, kK1, kK4>(tmem + kAttnTmemW, k_major(base + Lay::kQ + next % kQs * kAttnTile), k_major(base + Lay::kK + (next & 1) * kAttnTile), idesc_w, steps1, 0u);
                        ptx::umma_commit(&bar_w[next & 1]);
                    }
                }
            }
        }
    } else if (!STATE && warp < 12) {
        attn_more_registers<88>();
        {
            // two warps a quarter of the rows: 64 columns each
            const int quarter = warp & 3, part = (warp - 4) >> 2, i = quarter * 32 + lane;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
            for (int c = 0; c < chunks; ++c) {
                const int n = rows_of(c), shift = c == 0 ? less : 0;
                if (!wait_bounded_idle(&bar_w[c & 1], c >> 1 & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
                ptx::tc_fence_after_sync();
                uint32_t low[16];                                // the second pieces of this warp's first group
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int g = part * 2 + h;
                    uint32_t pieces[16][2];
#pragma unroll
                    for (int j = 0; j < 16; ++j) pieces[j][0] = pieces[j][1] = 0u;
                    if (BACK ? g >= quarter : g <= quarter) {    // on this side of the diagonal
                        uint32_t w[32];
                        ptx::tmem_ld_32x32b_x32(lanes + kAttnTmemW + g * 32, w);
                        const float* l = weight + kAttnRows + (BACK ? g * 32 - i : i - g * 32);
                        const bool cut = g == quarter || (BACK && n < kAttnRows);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float f[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int col = 2 * j + e;
                                f[e] = __uint_as_float(w[col]) * l[BACK ? col : -col];
                                if (cut) f[e] = (BACK ? g * 32 + col >= i && g * 32 + col < n : g * 32 + col <= i) ? f[e] : 0.0f;
                            }
                            attn_split(f[0], f[1], pieces[j]);
                        }
                    }
                    // P takes the place of W: first pieces of both groups that of the first one, second pieces that of the second
                    uint32_t high[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) high[j] = pieces[j][0];
                    attn_tmem_st_x16(lanes + kAttnTmemW + part * 64 + h * 16, high);
                    if (h == 1) attn_tmem_st_x16(lanes + kAttnTmemW + part * 64 + 32, low);
#pragma unroll
                    for (int j = 0; j < 16; ++j) low[j] = pieces[j][1];
                    if (h == 1) attn_tmem_st_x16(lanes + kAttnTmemW + part * 64 + 48, low);
                }
                attn_tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&bar_p);

                if (!wait_bounded_idle(&bar_o, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
                ptx::tc_fence_after_sync();
                const float far = (i < n ? power[BACK ? n - i - shift : i + 1 - shift] : 0.0f) * p.scale_out;
                const long long to_row = (first_of(c) + i) * p.ld_out + static_cast<long long>(head) * p.d2;
#pragma unroll 1
                for (int col = part * 64; col < min(part * 64 + 64, p.d2); col += 16) {
                    uint32_t o1[16], o2[16], out[8];
                    attn_tmem_ld_x16(lanes + kAttnTmemO1 + col, o1);
                    attn_tmem_ld_x16(lanes + kAttnTmemO2 + col, o2);
                    ptx::tmem_ld_wait();
                    float f[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) f[j] = fmaf(__uint_as_float(o1[j]), far, __uint_as_float(o2[j]) * p.scale_out);
                    if (i < n) {
                        if (p.out_f32) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (col + j * 4 < p.d2)
                                    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to_row + col + j * 4) = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) out[j] = attn_pair(f[2 * j], f[2 * j + 1]);
                            __nv_bfloat16* at = static_cast<__nv_bfloat16*>(p.out) + to_row + col;
                            if (p.wide) {
                                attn_store_32(at, out);
                            } else {
                                *reinterpret_cast<uint4*>(at) = make_uint4(out[0], out[1], out[2], out[3]);
                                if (col + 8 < p.d2) *reinterpret_cast<uint4*>(at + 8) = make_uint4(out[4], out[5], out[6], out[7]);
                            }
                        }
                    }
                    __syncwarp();
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&bar_o_free);
            }
        }
    } else if (warp < 16) {
        attn_fewer_registers<56>();
        constexpr int kWorkers = STATE ? 12 * 32 : 4 * 32;       // without outputs their warps make keys too
        const int worker = tid - (16 * 32 - kWorkers);
        for (int c = 0; c < chunks; ++c) {
            const int n = rows_of(c);
            if (!wait_bounded_idle(&full_k[c & 1], c >> 1 & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            // q k^T has been read from k before it is overwritten, and U of the chunk before from the other pieces
            if (!STATE && !wait_bounded_idle(&bar_w[c & 1], c >> 1 & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            if (c > 0 && !wait_bounded_idle(&bar_u, (c - 1) & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            // (behind bar_u: with U of the chunk before done, that chunk's v had landed, so this completion is the next one)
            if (n < kAttnRows && !wait_bounded_idle(&full_v[c % Lay::kVs], c / Lay::kVs & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            uint8_t* const k = smem + Lay::kK + (c & 1) * kAttnTile;
            // twice 16 bytes a thread at a time
            const int parts = halves1 * (kAttnHalf / 16);
#pragma unroll 1
            for (int first = worker; first < parts; first += 2 * kWorkers) {
                uint4 in[2];
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    in[q] = first + q * kWorkers < parts ? *reinterpret_cast<const uint4*>(k + (first + q * kWorkers) * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int at = first + q * kWorkers, row = at / 8 % kAttnRows;
                    // (rows that the chunk does not have: zero, not their weight, which may have grown beyond fp32)
                    const float w = row < n ? weight[kAttnRows + (BACK ? row : n - 1 - row)] : 0.0f;
                    if (row >= n) in[q] = make_uint4(0u, 0u, 0u, 0u);
                    const f32x2 ww = pack2(w, w), minus = pack2(-1.0f, -1.0f);
                    const uint32_t pair[4] = {in[q].x, in[q].y, in[q].z, in[q].w};
                    uint32_t out[UP][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        f32x2 left = mul2(pack2(attn_lo(pair[j]), attn_hi(pair[j])), ww);
#pragma unroll
                        for (int u = 0; u < UP; ++u) {           // as in attn_split
                            float lo, hi;
                            unpack2(left, lo, hi);
                            out[u][j] = attn_pair(lo, hi);
                            if (u + 1 < UP) left = fma2(pack2(attn_lo(out[u][j]), attn_hi(out[u][j])), minus, left);
                        }
                    }
                    if (at < parts) {
#pragma unroll
                        for (int u = 0; u < UP; ++u)
                            *reinterpret_cast<uint4*>((u == 0 ? k : smem + Lay::kLow + (u - 1) * kAttnTile) + at * 16) = make_uint4(out[u][0], out[u][1], out[u][2], out[u][3]);
                    }
                }
            }
            if (n < kAttnRows) {
                for (int h = 0; h < halves2; ++h)
                    for (int at = worker; at < (kAttnRows - n) * 8; at += kWorkers) *reinterpret_cast<uint4*>(smem + Lay::kV + c % Lay::kVs * kAttnTile + h * kAttnHalf + n * 128 + at * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bar_k);
        }
    } else {
        attn_more_registers<104>();
        // this thread's part of the state: row m, columns 64 side and up
        const int quarter = warp & 3, side = (warp - 16) >> 2, m = quarter * 32 + lane;
        const bool mine = side < halves2;
        float st[64];
        // What the pieces in front of a row add to the state: [column][row], so that a warp's rows lie side by side, or (a sum with the roles
        // of the state's dimensions exchanged) [row][column].
        const long long carry_size = kAttnRows * kAttnRows, carry_step = carry_size * p.heads;
#pragma unroll
        for (int j = 0; j < 64; ++j) st[j] = 0.0f;
        if (!STATE && p.state_in != nullptr && slot >= 0 && m < p.d1) {
            const float* from = p.state_in + state_at + static_cast<long long>(m) * p.s1 + static_cast<long long>(side) * 64 * p.s2;
            const int there = p.d2 - side * 64;
            if (p.state_vec) {
#pragma unroll
                for (int j = 0; j < 64; j += 4)
                    if (j < there) {
                        const float4 v = __ldg(reinterpret_cast<const float4*>(from + j));
                        st[j] = v.x; st[j + 1] = v.y; st[j + 2] = v.z; st[j + 3] = v.w;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < 64; ++j) {
                    if (j < there) st[j] = __ldg(from);
                    from += p.s2;
                }
            }
        }
        if (!STATE && piece.index > 0 && mine) {
            const int pieces = piece.index * static_cast<int>(p.seg / p.sub);
            const float* from = p.carry + (attn_first_slot(p, piece.b) * p.heads + head) * carry_size +
                                (p.carry_turned ? static_cast<long long>(m) * kAttnRows + side * 64 : static_cast<long long>(side) * 64 * kAttnRows + m);
            const float all = static_cast<float>(exp(log_l * static_cast<double>(p.sub))), first = BACK ? static_cast<float>(exp(log_l * static_cast<double>(p.sub - 1))) : all;
#pragma unroll 1
            for (int s = 0; s < pieces; ++s, from += carry_step) {
                const float f = s == 0 ? first : all;
                if (BACK && p.carry_turned) {
#pragma unroll
                    for (int j = 0; j < 64; j += 4) {
                        const float4 v = *reinterpret_cast<const float4*>(from + j);
                        st[j] = fmaf(st[j], f, v.x);
                        st[j + 1] = fmaf(st[j + 1], f, v.y);
                        st[j + 2] = fmaf(st[j + 2], f, v.z);
                        st[j + 3] = fmaf(st[j + 3], f, v.w);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 64; ++j) st[j] = fmaf(st[j], f, from[j * kAttnRows]);
                }
            }
        }
        // the state in front of a chunk, rounded to bf16 for its product with q
        auto publish = [&]() {
            if (!STATE && mine) {
#pragma unroll
                for (int g = 0; g < 8; ++g)
                    *reinterpret_cast<uint4*>(smem + Lay::kState + side * kAttnHalf + m * 128 + ((g ^ (m & 7)) << 4)) =
                        make_uint4(attn_pair(st[8 * g], st[8 * g + 1]), attn_pair(st[8 * g + 2], st[8 * g + 3]), attn_pair(st[8 * g + 4], st[8 * g + 5]), attn_pair(st[8 * g + 6], st[8 * g + 7]));
            }
            if (!STATE) ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bar_state);
        };
        if (chunks > 0) publish();
        for (int c = 0; c < chunks; ++c) {
            const int n = rows_of(c), shift = c == 0 ? less : 0;
            if (!wait_bounded_idle(&bar_u, c & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            ptx::tc_fence_after_sync();
            if (mine) {
                const float f = power[n - shift];
                const uint32_t at = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + kAttnTmemU + side * 64;
                uint32_t u[2][16];
                attn_tmem_ld_x16(at, u[0]);
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    ptx::tmem_ld_wait();
                    if (g < 3) attn_tmem_ld_x16(at + (g + 1) * 16, u[(g + 1) & 1]);
#pragma unroll
                    for (int j = 0; j < 16; ++j) st[g * 16 + j] = fmaf(st[g * 16 + j], f, __uint_as_float(u[g & 1][j]));
                }
            }
            ptx::tc_fence_before_sync();
            if (c + 1 < chunks) publish();
        }
        if (STATE) {
            if (mine) {
                float* to = p.carry + (number * p.heads + head) * carry_size + static_cast<long long>(side) * 64 * kAttnRows + m;
#pragma unroll
                for (int j = 0; j < 64; ++j) to[j * kAttnRows] = st[j];
            }
        } else if (UP == 3 && r.len <= p.seg && p.state_out != nullptr && slot >= 0 && m < p.d1) {
            const float f = BACK && r.len > 0 ? static_cast<float>(exp(log_l)) : 1.0f;   // see attn_kernel
            float* to = p.state_out + state_at + static_cast<long long>(m) * p.s1 + static_cast<long long>(side) * 64 * p.s2;
            const int there = p.d2 - side * 64;
            if (p.state_vec) {
#pragma unroll
                for (int j = 0; j < 64; j += 4)
                    if (j < there) *reinterpret_cast<float4*>(to + j) = make_float4(st[j] * f, st[j + 1] * f, st[j + 2] * f, st[j + 3] * f);
            } else {
#pragma unroll
                for (int j = 0; j < 64; ++j) {
                    if (j < there) *to = st[j] * f;
                    to += p.s2;
                }
            }
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

// The states behind sequences that have slots, from what their pieces add (made of three pieces of the keys): a block has 32 x 32 of
// one head's state, its rows side by side while it adds, its columns for the states in and out.  Where only sequences of more than a segment
// have slots, number i is the one that begins in the i-th `seg` rows: no two of them can.
__global__ void __launch_bounds__(256) attn_state_kernel(const __grid_constant__ AttnParams p) {
    __shared__ float tile[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n0 = blockIdx.x % 4 * 32, m0 = blockIdx.x / 4 % 4 * 32;
    const int head = static_cast<int>(blockIdx.x / 16 % p.heads);
    long long b = blockIdx.x / 16 / p.heads;
    seq_grid_wait();
    if (m0 >= p.d1 || n0 >= p.d2) return;
    if (!p.every) {
        const long long number = b;
        b = 0;
        for (long long hi = p.batch - 1; b < hi;) {
            const long long mid = (b + hi + 1) / 2;
            if (__ldg(p.offsets + mid) / p.seg <= number) b = mid;
            else hi = mid - 1;
        }
        if (__ldg(p.offsets + b) / p.seg != number) return;
    }
    const SeqRange r = seq_range(p.offsets, b, p.max_len, p.rows, p.status);
    if (!p.every && r.len <= p.seg) return;
    const long long slot = state_slot(p.slots, b, p.n_slots, p.status);
    if (slot < 0) return;
    const long long at = slot * p.state_stride + static_cast<long long>(head) * p.d1 * p.d2;
    const double log_l = static_cast<double>(__ldg(p.log_decay + head));
    const long long pieces = (r.len + p.sub - 1) / p.sub, last = r.len - (pieces - 1) * p.sub;
    const float* carry = p.carry + (attn_first_slot(p, b) * p.heads + head) * kAttnRows * kAttnRows;
    for (int i = warp; i < 32; i += 8)
        tile[i][lane] = p.state_in != nullptr && m0 + i < p.d1 && n0 + lane < p.d2 ? __ldg(p.state_in + at + static_cast<long long>(m0 + i) * p.s1 + static_cast<long long>(n0 + lane) * p.s2) : 0.0f;
    __syncthreads();
    float st[4];
    for (int i = 0; i < 4; ++i) st[i] = tile[lane][warp + i * 8];
    const float all = static_cast<float>(exp(log_l * static_cast<double>(p.sub)));
    for (long long s = 0; s < pieces; ++s) {
        const long long rows = s + 1 < pieces ? p.sub : last, left = p.back && s == 0 ? rows - 1 : rows;   // see attn_kernel
        const float f = left == 0 ? 1.0f : left == p.sub ? all : static_cast<float>(exp(log_l * static_cast<double>(left)));
#pragma unroll
        for (int i = 0; i < 4; ++i) st[i] = fmaf(st[i], f, carry[s * p.heads * kAttnRows * kAttnRows + (n0 + warp + i * 8) * kAttnRows + m0 + lane]);
    }
    __syncthreads();
    const float f = p.back && r.len > 0 ? static_cast<float>(exp(log_l)) : 1.0f;
    for (int i = 0; i < 4; ++i) tile[lane][warp + i * 8] = st[i] * f;
    __syncthreads();
    for (int i = warp; i < 32; i += 8)
        if (m0 + i < p.d1 && n0 + lane < p.d2) p.state_out[at + static_cast<long long>(m0 + i) * p.s1 + static_cast<long long>(n0 + lane) * p.s2] = tile[i][lane];
}

}  // namespace tdx
