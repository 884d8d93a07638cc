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

#include <type_traits>

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
    // tensor-core kernel: tiles of 128 * halves output features and bt rows (dw: bt columns)
    int halves, bt, box;             // box: rows of one copy of the activations
    int stages, tmem_cols;
    int buffers;                     // accumulators of a tile: 2, or 1 where one takes all 512 columns
    int features;                    // of the output's feature dimension: N, K, or (dw) N
    int feature_tiles;
    int blocks;                      // of 64 of the reduction (forward, dx)
    int column_tiles;                // dw
};

// The range of an expert's rows; one that leaves [0, rows] or descends is reported and empty.
__device__ __forceinline__ SeqRange grouped_range(const GroupedParams& p, int e) { return seq_range(p.offsets, e, p.rows, p.rows, p.status); }

// ---------------------------------------------------------------- CUDA cores
constexpr int kSimtThreads = 256;
constexpr int kSimtColumns = 64;
constexpr int kSimtGroups = 4;                                  // of 64 threads
constexpr int kSimtEach = 8;                                    // of the reduction for each group
constexpr int kSimtK = kSimtGroups * kSimtEach;

// One tile of BM x 64 outputs, 32 of the reduction at a time through shared memory; the next 32 are on their way while these are
// multiplied.  What bounds it is the scheduler and shared memory: 8 x 8 outputs a thread take two 16-byte reads of each operand for 64
// multiply-adds, and pairs of columns take one instruction for two.  A tile has 64 such threads, and products of a few thousand rows and
// columns have two or three tiles an SM; so four groups of threads take eight of the reduction each, and their sums are added up at the
// end, always in the same order.  1501 x 1000 x 520 in five experts, forward and both gradients: 174 us (27 TFLOP/s of the CUDA cores'
// 74); addresses made anew for every 32: 183 us; one column an instruction: 222 us; 8 x 4 outputs a thread and one group: 247 us.  BM = 16 serves experts of few rows, where a
// tile of 64 would be mostly empty.  VEC = 4 moves 16 bytes at a time.
// In shared memory the groups of four columns of a line k are exchanged by k / 4 (exclusive or), so that operands whose contiguous
// dimension is the reduction are written to different banks.
template <typename T, int PASS, int BM, int VEC>
__global__ void __launch_bounds__(kSimtThreads, 2) grouped_simt_kernel(const __grid_constant__ GroupedParams p) {
    constexpr int BN = kSimtColumns, kSide = BM == 64 ? 8 : 16;   // threads of a group along the columns
    constexpr int TM = BM == 64 ? 8 : 4, TN = BN / kSide, kTile = kSimtK * (BM + BN);
    static_assert(BM / TM * kSide == kSimtThreads / kSimtGroups, "a group covers a tile");
    static_assert(TM * TN * (kSimtThreads / 2) <= 2 * kTile, "two groups' sums fit");
    __shared__ __align__(16) float shared[2 * kTile];
    const T* a = static_cast<const T*>(p.a);
    const T* b = static_cast<const T*>(p.b);
    T* out = static_cast<T*>(p.out);
    const int tid = threadIdx.x;
    seq_grid_wait();
    int m_count, n_count, m0, n0;
    long long depth;
    if (PASS == kGroupedDw) {
        const int tiles_n = (p.K + BN - 1) / BN, tiles_m = (p.N + BM - 1) / BM;
        const long long item = blockIdx.x, per = static_cast<long long>(tiles_n) * tiles_m;
        const int e = static_cast<int>(item / per), in = static_cast<int>(item - e * per);
        const SeqRange r = grouped_range(p, e);
        m0 = in / tiles_n * BM; n0 = in % tiles_n * BN;
        m_count = p.N; n_count = p.K; depth = r.len;
        a += r.first * p.ld_a; b += r.first * p.ld_b; out += static_cast<long long>(e) * p.N * p.K;
    } else {
        n_count = PASS == kGroupedForward ? p.N : p.K;
        const int tiles_n = (n_count + BN - 1) / BN;
        const long long number = blockIdx.x / tiles_n;
        n0 = static_cast<int>(blockIdx.x - number * tiles_n) * BN;
        if (n0 == 0) seq_check(p.offsets, number, p.experts, p.rows, p.rows, p.status);
        const SeqPiece piece = seq_piece(p.offsets, p.experts, 1, BM, number);
        const SeqRange r = grouped_range(p, static_cast<int>(piece.b));
        if (static_cast<long long>(piece.index) * BM >= r.len) return;
        m0 = piece.index * BM; m_count = r.len; depth = PASS == kGroupedForward ? p.K : p.N;
        a += r.first * p.ld_a; b += piece.b * static_cast<long long>(p.N) * p.K; out += r.first * p.ld_out;
    }
    const long long ld_b = PASS == kGroupedDw ? p.ld_b : p.K, ld_out = PASS == kGroupedDw ? p.K : p.ld_out;
    constexpr bool kADeep = PASS != kGroupedDw, kBDeep = PASS == kGroupedForward;   // the reduction is the contiguous dimension
    constexpr int kAOf = (BM * kSimtK / VEC + kSimtThreads - 1) / kSimtThreads, kBOf = BN * kSimtK / VEC / kSimtThreads;
    SeqVec<T, VEC> ra[kAOf], rb[kBOf];
    // VEC elements of an operand, number `at` of what the block copies: line or column c, line k of the reduction
    auto place = [&](auto deep, int width, int at, int* c, int* k) {
        if (decltype(deep)::value) { *c = at / (kSimtK / VEC); *k = at % (kSimtK / VEC) * VEC; }
        else { *c = at % (width / VEC) * VEC; *k = at / (width / VEC); }
    };
    // the thread's first, from where its others are a fixed distance apart
    auto start = [&](auto deep, int width, const T* from, long long ld, int first) {
        int c, k;
        place(deep, width, tid, &c, &k);
        return from + (decltype(deep)::value ? (static_cast<long long>(first) + c) * ld + k : k * ld + first + c);
    };
    auto get = [&](auto deep, int width, int i, const T* from, long long ld, int count, long long left, SeqVec<T, VEC>* r) {
        int c, k;
        place(deep, width, tid + i * kSimtThreads, &c, &k);
#pragma unroll
        for (int v = 0; v < VEC; ++v) r->v[v] = seq_from_float<T>(0.0f);
        const int apart = kSimtThreads / ((decltype(deep)::value ? kSimtK : width) / VEC);
        if (c < count && k < left) *r = seq_load<T, VEC>(from + i * apart * ld);
    };
    auto put = [&](auto deep, int width, int at, float* to, const SeqVec<T, VEC>& r) {
        int c, k;
        place(deep, width, at, &c, &k);
        const int mask = width / 4 < 8 ? width / 4 - 1 : 7;
        float f[VEC];
        seq_unpack<T, VEC>(r, f);
        float* at_k = to + k * width + (((c / 4) ^ (k / 4 & mask)) * 4 + c % 4);
        if (decltype(deep)::value) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) at_k[i * width] = f[i];       // VEC of four start at a multiple of four: one k / 4
        } else {
            seq_store<float, VEC>(at_k, f);
        }
    };
    typedef typename std::conditional<kADeep, SeqYes, SeqNo>::type ADeep;
    typedef typename std::conditional<kBDeep, SeqYes, SeqNo>::type BDeep;
    const T* next_a = start(ADeep(), BM, a, p.ld_a, m0);
    const T* next_b = start(BDeep(), BN, b, ld_b, n0);
    auto fetch = [&](long long left) {
#pragma unroll
        for (int i = 0; i < kAOf; ++i)
            if (BM * kSimtK / VEC >= kSimtThreads || tid < BM * kSimtK / VEC) get(ADeep(), BM, i, next_a, p.ld_a, m_count - m0, left, &ra[i]);
#pragma unroll
        for (int i = 0; i < kBOf; ++i) get(BDeep(), BN, i, next_b, ld_b, n_count - n0, left, &rb[i]);
        next_a += kADeep ? kSimtK : kSimtK * p.ld_a;
        next_b += kBDeep ? kSimtK : kSimtK * ld_b;
    };
    auto keep = [&](int buf) {
        float* sa = shared + buf * kTile;
#pragma unroll
        for (int i = 0; i < kAOf; ++i)
            if (BM * kSimtK / VEC >= kSimtThreads || tid < BM * kSimtK / VEC) put(ADeep(), BM, tid + i * kSimtThreads, sa, ra[i]);
#pragma unroll
        for (int i = 0; i < kBOf; ++i) put(BDeep(), BN, tid + i * kSimtThreads, sa + kSimtK * BM, rb[i]);
    };
    f32x2 acc[TM][TN / 2];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN / 2; ++j) acc[i][j] = 0;
    // rows tm .. tm + 3 and 32 + tm .., columns tn .. tn + 3 and 32 + tn ..: neighbours read neighbours
    const int group = tid / (kSimtThreads / kSimtGroups), in_group = tid % (kSimtThreads / kSimtGroups);
    const int tm = in_group / kSide * 4, tn = in_group % kSide * 4;
    constexpr int kAMask = BM / 4 < 8 ? BM / 4 - 1 : 7;
    fetch(depth);
    keep(0);
    __syncthreads();
    int buf = 0;
    for (long long k0 = 0; k0 < depth; k0 += kSimtK) {
        const bool more = k0 + kSimtK < depth;
        if (more) fetch(depth - k0 - kSimtK);
        const float* sa = shared + buf * kTile + group * kSimtEach * BM;
        const float* sb = shared + buf * kTile + kSimtK * BM + group * kSimtEach * BN;
#pragma unroll
        for (int k = 0; k < kSimtEach; ++k) {
            const int turn = group * (kSimtEach / 4) + k / 4;
            float fa[TM];
            f32x2 fb[TN / 2];
#pragma unroll
            for (int i = 0; i < TM; i += 4) *reinterpret_cast<float4*>(fa + i) = *reinterpret_cast<const float4*>(sa + k * BM + ((tm / 4 + i * 2) ^ (turn & kAMask)) * 4);
#pragma unroll
            for (int j = 0; j < TN; j += 4) *reinterpret_cast<ulonglong2*>(fb + j / 2) = *reinterpret_cast<const ulonglong2*>(sb + k * BN + ((tn / 4 + j * 2) ^ (turn & 7)) * 4);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const f32x2 twice = pack2(fa[i], fa[i]);
#pragma unroll
                for (int j = 0; j < TN / 2; ++j) acc[i][j] = fma2(twice, fb[j], acc[i][j]);
            }
        }
        if (more) keep(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }
    // groups 2 and 3 give their sums to 0 and 1, and 1 gives its to 0
#pragma unroll
    for (int half = kSimtGroups / 2; half > 0; half /= 2) {
        f32x2* mine = reinterpret_cast<f32x2*>(shared) + tid % (half * (kSimtThreads / kSimtGroups));
        constexpr int kOne = kSimtThreads / kSimtGroups;
        if (group >= half && group < 2 * half) {
#pragma unroll
            for (int i = 0; i < TM * TN / 2; ++i) mine[i * half * kOne] = acc[i * 2 / TN][i % (TN / 2)];
        }
        __syncthreads();
        if (group < half) {
#pragma unroll
            for (int i = 0; i < TM * TN / 2; ++i) acc[i * 2 / TN][i % (TN / 2)] = add2(acc[i * 2 / TN][i % (TN / 2)], mine[i * half * kOne]);
        }
        __syncthreads();
    }
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int m = tm + i % 4 + i / 4 * 32;
        if (m >= m_count - m0) continue;
        T* row = out + (m0 + m) * ld_out;
#pragma unroll
        for (int j = 0; j < TN; j += VEC) {
            float sums[TN];
            unpack2(acc[i][j / 2], sums[j / 2 * 2], sums[j / 2 * 2 + 1]);
            if (VEC == 4) unpack2(acc[i][j / 2 + 1], sums[j / 2 * 2 + 2], sums[j / 2 * 2 + 3]);
            const int n = tn + j % 4 + j / 4 * 32;
            float f[VEC];
#pragma unroll
            for (int v = 0; v < VEC; ++v) f[v] = sums[j + v];
            if (n < n_count - n0) seq_store<T, VEC>(row + n0 + n, f);
        }
    }
}

// ---------------------------------------------------------------- tensor cores
// Persistent, one block an SM: warp 0 copies 128-byte-swizzled tiles of 64 of the reduction into a ring of stages (TMA), warp 1 issues the
// tcgen05 products, eight warps turn accumulators into bf16.  The features are the product's M (128 or two times 128) and the rows of an
// expert its N: an expert's last tile then costs what its rows need, in steps of 16, instead of a whole tile of 128, and a few rows cost
// 32 columns of a product that streams the weights.  Tiles of up to 256 of tensor memory's 512 columns hold their accumulators twice, so that
// an epilogue runs under the next tile's products.  Tiles of 256 x 256 take all columns: their products wait for the epilogue in front,
// about 5 us a tile beside 12 for every 1024 of the reduction (16 x 512 rows, 4096 features, four rounds of tiles: 72, 120, 220, 424 us at 1024,
// 2048, 4096, 8192), and are still the fastest for many rows (grouped_gemm.cu).
// Measured: 8 x 2048 rows, 4096 x 4096: 377 us (1458 of the 1664 TFLOP/s of a library's product); 8192 rows unevenly over 16 experts, 4096 x
// 2048: 144 to 157 (875 to 955), bound by the epilogues between products and then by the last round of tiles; 128 rows over 32 experts, 2048 x
// 2048: 42 us, which is the weights' 269 MB at the copy rate.
// dw sums over an expert's rows: both operands are read with the rows as the reduction, and rows of the last block that belong to the
// next expert are set to zero in shared memory in front of the product (a factor of zero in one operand would leave NaN and infinity).
constexpr int kGroupedMostExperts = 1024;                        // whose tile counts are kept in shared memory
constexpr int kGroupedSorted = 128;                              // experts that are sorted by their rows, each against all others
constexpr int kGroupedThreads = 320;
constexpr int kGroupedEpilogueWarps = 8;
constexpr int kGroupedStagePitch = 80;                           // bytes of a staged row of 32 bf16
constexpr int kGroupedStageWarp = 3 * 1024;                      // a warp's part: 32 such rows, or 2 KB for the copy engine
constexpr int kGroupedStaging = kGroupedEpilogueWarps * kGroupedStageWarp;
constexpr int kGroupedMostStages = 10;

struct GroupedTile {
    long long row;                   // first row of the tile (dw: of the expert)
    int expert, count;               // rows of the tile (dw: of the expert)
    int feature, column;             // first feature, and (dw) first column
    int blocks;                      // of 64 of the reduction
};

// The last entry of an ascending table that is at most `v`.
__device__ __forceinline__ int grouped_search(const int* table, int count, int v) {
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (table[mid] <= v) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// `first`: forward and dx: whole tiles of rows of the experts in front of each, added up, and behind them the experts with rows left over,
// most of them first, and their number; dw: the experts, most rows first.
template <int PASS>
__device__ __forceinline__ bool grouped_tile(const GroupedParams& p, const int* first, long long item, GroupedTile* t) {
    if (PASS == kGroupedDw) {
        const int per = p.feature_tiles * p.column_tiles;
        if (item >= static_cast<long long>(per) * p.experts) return false;
        const int place = static_cast<int>(item / per), in = static_cast<int>(item - static_cast<long long>(place) * per);
        t->expert = first[place];
        t->feature = in / p.column_tiles * (128 * p.halves);
        t->column = in % p.column_tiles * p.bt;
        const int lo = __ldg(p.offsets + t->expert), hi = __ldg(p.offsets + t->expert + 1);
        t->row = lo;
        t->count = seq_accepted(lo, hi, p.rows, p.rows) ? hi - lo : 0;
        t->blocks = (t->count + 63) / 64;
        return true;
    }
    // Whole tiles come first and those with what is left of an expert's rows behind them, large ones first, so that the last round, which
    // not all blocks have a tile for, is one of small tiles.  An expert's tiles of rows lie side by side for each tile of features, so that
    // its weights are read together.
    const int* rest = first + p.experts + 1;
    const long long whole = static_cast<long long>(first[p.experts]) * p.feature_tiles;
    int e, f, r;
    if (item < whole) {
        e = grouped_search(first, p.experts, static_cast<int>(item / p.feature_tiles));
        const int tiles = first[e + 1] - first[e], in = static_cast<int>(item - static_cast<long long>(first[e]) * p.feature_tiles);
        f = in / tiles;
        r = in - f * tiles;
    } else {
        const long long behind = item - whole;
        if (behind >= static_cast<long long>(rest[p.experts]) * p.feature_tiles) return false;
        const int place = static_cast<int>(behind / p.feature_tiles);
        e = rest[place];
        f = static_cast<int>(behind - static_cast<long long>(place) * p.feature_tiles);
        r = first[e + 1] - first[e];
    }
    const int from = __ldg(p.offsets + e), to = __ldg(p.offsets + e + 1);
    t->expert = e;
    t->row = from + static_cast<long long>(r) * p.bt;
    t->count = min(p.bt, to - from - r * p.bt);
    t->feature = f * (128 * p.halves);
    t->column = 0;
    t->blocks = p.blocks;
    return true;
}

template <int PASS>
__global__ void __launch_bounds__(kGroupedThreads, 1) grouped_umma_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                                                                          const __grid_constant__ CUtensorMap tm_out,
                                                                          const __grid_constant__ GroupedParams p) {
    extern __shared__ uint8_t grouped_smem[];
    __shared__ __align__(8) uint64_t full_bar[kGroupedMostStages], empty_bar[kGroupedMostStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    volatile int* abort_flag = &s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t a_bytes = static_cast<uint32_t>(p.halves) * 16384u, stage_bytes = a_bytes + static_cast<uint32_t>(p.bt) * 128u;
    uint8_t* const ring = grouped_smem + ((1024u - (ptx::smem_u32(grouped_smem) & 1023u)) & 1023u);
    uint8_t* const staging = ring + static_cast<size_t>(p.stages) * stage_bytes;
    int* const first = reinterpret_cast<int*>(staging + kGroupedStaging);

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(&full_bar[s], 1);
            ptx::mbar_init(&empty_bar[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&tfull_bar[b], 1);
            ptx::mbar_init(&tempty_bar[b], kGroupedEpilogueWarps);
        }
        s_abort = 0;
        ptx::fence_barrier_init();
        ptx::tma_prefetch_desc(&tm_a);
        ptx::tma_prefetch_desc(&tm_b);
        ptx::tma_prefetch_desc(&tm_out);
    }
    if (warp == 1) {
        ptx::tmem_alloc(&s_tmem, static_cast<uint32_t>(p.tmem_cols));
        ptx::tmem_relinquish();
    }
    ptx::grid_dependency_wait();
    if (warp == 0) {
        // where an expert stands among those with more rows (left over)
        auto rows_of = [&](int e) {
            const int lo = __ldg(p.offsets + e), hi = __ldg(p.offsets + e + 1), n = seq_accepted(lo, hi, p.rows, p.rows) ? hi - lo : 0;
            return PASS == kGroupedDw ? n : n % p.bt;
        };
        auto place_of = [&](int e, int n) {
            int place = 0;
            for (int o = 0; o < p.experts; ++o) {
                const int m = rows_of(o);
                place += m > n || (m == n && o < e);
            }
            return place;
        };
        // (narrow tiles cost the weights that they read, whatever their rows are)
        const bool sorted = p.experts <= kGroupedSorted && (PASS == kGroupedDw || p.bt > 64);
        if (PASS == kGroupedDw) {
            for (int e = lane; e < p.experts; e += 32) {
                const int n = grouped_range(p, e).len;
                first[sorted ? place_of(e, n) : e] = e;
            }
        } else {
            int* const rest = first + p.experts + 1;
            int whole = 0, count = 0;
            if (lane == 0) first[0] = 0;
            for (int e0 = 0; e0 < p.experts; e0 += 32) {
                const int e = e0 + lane, n = e < p.experts ? grouped_range(p, e).len : 0, left = n % p.bt;
                int w = n / p.bt;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int up = __shfl_up_sync(0xffffffffu, w, d);
                    if (lane >= d) w += up;
                }
                const uint32_t there = __ballot_sync(0xffffffffu, left > 0);
                if (e < p.experts) first[e + 1] = whole + w;
                if (left > 0) rest[sorted ? place_of(e, left) : count + __popc(there & ((1u << lane) - 1u))] = e;
                __syncwarp();
                whole += __shfl_sync(0xffffffffu, w, 31);
                count += __popc(there);
            }
            if (lane == 0) rest[p.experts] = count;
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    // A block's tiles: rounds go through the blocks forwards and backwards in turn, so that with tiles from large to small all blocks
    // get about as much (8192 rows unevenly over 16 experts, 4096 x 2048: 154 -> 147 us with large ones first; taking tiles from a counter
    // is no faster and needs a workspace).  Narrow tiles cost the same all of them.
    auto tile_of = [&](int local, GroupedTile* t) {
        const unsigned at = (local & 1) != 0 && p.bt > 64 ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
        return grouped_tile<PASS>(p, first, static_cast<long long>(local) * gridDim.x + at, t);
    };

    if (warp == 0) {
        if (ptx::elect_one()) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            GroupedTile t;
            for (int local = 0; ok && tile_of(local, &t); ++local) {
                const int boxes = PASS == kGroupedDw ? p.bt / 64 : (t.count + p.box - 1) / p.box;
                const uint32_t bytes = a_bytes + static_cast<uint32_t>(boxes) * (PASS == kGroupedDw ? 8192u : static_cast<uint32_t>(p.box) * 128u);
                for (int kb = 0; kb < t.blocks; ++kb) {
                    if (!wait_bounded(&empty_bar[stage], phase ^ 1u, abort_flag, p.status, kTimeoutProducer)) {
                        ok = false;
                        break;
                    }
                    uint64_t* bar = &full_bar[stage];
                    ptx::mbar_arrive_expect_tx(bar, bytes);
                    uint8_t* a = ring + static_cast<size_t>(stage) * stage_bytes;
                    uint8_t* b = a + a_bytes;
                    const int at = kb * 64, row = static_cast<int>(t.row);
                    if (PASS == kGroupedForward) {
                        for (int h = 0; h < p.halves; ++h) ptx::tma_load_3d(a + h * 16384, &tm_a, bar, at, t.feature + h * 128, t.expert);
                    } else if (PASS == kGroupedDx) {
                        for (int i = 0; i < 2 * p.halves; ++i) ptx::tma_load_3d(a + i * 8192, &tm_a, bar, t.feature + i * 64, at, t.expert);
                    } else {
                        for (int i = 0; i < 2 * p.halves; ++i) ptx::tma_load_2d(a + i * 8192, &tm_a, bar, t.feature + i * 64, row + at);
                    }
                    if (PASS == kGroupedDw) {
                        for (int i = 0; i < boxes; ++i) ptx::tma_load_2d(b + i * 8192, &tm_b, bar, t.column + i * 64, row + at);
                    } else {
                        for (int i = 0; i < boxes; ++i) ptx::tma_load_2d(b + i * p.box * 128, &tm_b, bar, at, row + i * p.box);
                    }
                    if (++stage == p.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok) {
                // let copies that are still in flight land before the block goes away
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        }
    } else if (warp == 1) {
        constexpr bool kATurned = PASS != kGroupedForward, kBTurned = PASS == kGroupedDw;   // the reduction is not the contiguous dimension
        const uint64_t a_desc0 = ptx::make_smem_desc_sw128(ptx::smem_u32(ring), kATurned ? 8192u : 16u, 1024u);
        const uint64_t b_desc0 = ptx::make_smem_desc_sw128(ptx::smem_u32(ring) + a_bytes, kBTurned ? 8192u : 16u, 1024u);
        constexpr uint64_t a_k16 = (kATurned ? 2048u : 32u) >> 4, b_k16 = (kBTurned ? 2048u : 32u) >> 4;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        GroupedTile t;
        for (int local = 0; ok && tile_of(local, &t); ++local) {
            const int buf = local % p.buffers, use = local / p.buffers;
            if (!wait_bounded(&tempty_bar[buf], (use & 1) ^ 1u, abort_flag, p.status, kTimeoutMma)) break;
            ptx::tc_fence_after_sync();
            const int n = PASS == kGroupedDw ? p.bt : (t.count + 15) / 16 * 16;
            const uint32_t idesc = ptx::make_idesc_bf16_f32(128, n, kATurned, kBTurned);
            const uint32_t d = tmem + static_cast<uint32_t>(buf * p.halves * p.bt);
            for (int kb = 0; kb < t.blocks; ++kb) {
                if (!wait_bounded(&full_bar[stage], phase, abort_flag, p.status, kTimeoutMma)) {
                    ok = false;
                    break;
                }
                int steps = 4;
                if (PASS == kGroupedDw && kb + 1 == t.blocks) {
                    // the rows behind the expert's last one, up to the end of the last step of 16
                    const int left = t.count - kb * 64;
                    steps = (left + 15) / 16;
                    uint8_t* base = ring + static_cast<size_t>(stage) * stage_bytes;
                    const int rows = steps * 16 - left, tiles = 2 * p.halves + p.bt / 64;
                    for (int i = lane; i < tiles * rows * 8; i += 32) {
                        const int tile = i / (rows * 8), in = i - tile * rows * 8;
                        *reinterpret_cast<uint4*>(base + tile * 8192 + (left + in / 8) * 128 + in % 8 * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(stage) * stage_bytes) >> 4;
                    for (int h = 0; h < p.halves; ++h) {
                        for (int j = 0; j < steps; ++j)
                            ptx::umma_bf16(d + static_cast<uint32_t>(h * p.bt), a_desc0 + at + h * (16384u >> 4) + j * a_k16, b_desc0 + at + j * b_k16, idesc,
                                           kb > 0 || j > 0 ? 1u : 0u);
                    }
                    ptx::umma_commit(&empty_bar[stage]);
                    if (kb + 1 == t.blocks) ptx::umma_commit(&tfull_bar[buf]);
                }
                __syncwarp();
                if (++stage == p.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (t.blocks == 0 && ptx::elect_one()) ptx::mbar_arrive(&tfull_bar[buf]);
            __syncwarp();
        }
    } else {
        const int ew = warp - 2, quarter = warp & 3, half = p.halves == 2 ? ew >> 2 : 0;
        const int c_first = p.halves == 2 ? 0 : (ew >> 2) * 32, c_step = p.halves == 2 ? 32 : 64;
        uint8_t* const mine = staging + ew * kGroupedStageWarp;
        __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(p.out);
        GroupedTile t;
        for (int local = 0; tile_of(local, &t); ++local) {
            const int buf = local % p.buffers, use = local / p.buffers;
            if (!wait_bounded(&tfull_bar[buf], use & 1, abort_flag, p.status, kTimeoutEpilogue)) break;
            ptx::tc_fence_after_sync();
            const int feature = t.feature + half * 128 + quarter * 32;
            const int columns = PASS == kGroupedDw ? min(p.bt, p.K - t.column) : t.count;
            const uint32_t from = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>((buf * p.halves + half) * p.bt);
            uint32_t r[32];
            if (c_first < columns) ptx::tmem_ld_32x32b_x32(from + c_first, r);
            for (int c0 = c_first; c0 < columns; c0 += c_step) {
                ptx::tmem_ld_wait();
                if (PASS != kGroupedDw && t.count == p.bt) {
                    // A whole tile leaves through the copy engine in blocks of 16 rows x 32 features (64-byte swizzle), two of them taking turns: stores
                    // from registers took 13 of the 124 us of 16 x 512 rows, 4096 x 2048, and the accumulators wait for them.  (It would also
                    // write the rows behind a tile that is not whole.)
                    uint32_t half_pairs[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        half_pairs[j] = *reinterpret_cast<uint32_t*>(&h);
                    }
                    if (c0 + c_step < columns) ptx::tmem_ld_32x32b_x32(from + c0 + c_step, r);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (lane == 0) ptx::tma_store_wait_read<1>();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t pair = half_pairs[b * 8 + j / 2];
                            *reinterpret_cast<uint16_t*>(mine + b * 1024 + j * 64 + (((lane >> 3) ^ (j >> 1 & 3)) << 4) + (lane & 7) * 2) = static_cast<uint16_t>(j & 1 ? pair >> 16 : pair);
                        }
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0 && feature < p.features) {
                            ptx::tma_store_2d(&tm_out, mine + b * 1024, feature, static_cast<int>(t.row) + c0 + b * 16);
                            ptx::tma_store_commit();
                        }
                    }
                    continue;
                }
                if (PASS != kGroupedDw && lane == 0) ptx::tma_store_wait_read<0>();   // of a whole tile in front of this one
                __syncwarp();
                if (PASS == kGroupedDw) {
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        pk[j] = t.blocks > 0 ? *reinterpret_cast<uint32_t*>(&h) : 0u;     // an expert without rows
                    }
                    if (c0 + c_step < columns) ptx::tmem_ld_32x32b_x32(from + c0 + c_step, r);
                    if (lane == 0) ptx::tma_store_wait_read<0>();
                    __syncwarp();
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *reinterpret_cast<uint4*>(mine + lane * 64 + ((g ^ (lane >> 1 & 3)) << 4)) = make_uint4(pk[4 * g], pk[4 * g + 1], pk[4 * g + 2], pk[4 * g + 3]);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && feature < p.N) {
                        ptx::tma_store_3d(&tm_out, mine, t.column + c0, feature, t.expert);
                        ptx::tma_store_commit();
                    }
                    continue;
                } else {
                    // a lane has a feature, an output row wants them side by side
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        *reinterpret_cast<__nv_bfloat16*>(mine + j * kGroupedStagePitch + lane * 2) = __float2bfloat16_rn(__uint_as_float(r[j]));
                }
                // the next columns are on their way while these are written
                if (c0 + c_step < columns) ptx::tmem_ld_32x32b_x32(from + c0 + c_step, r);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = lane / 4 + i * 8, part = lane % 4 * 8;
                    const uint4 v = *reinterpret_cast<const uint4*>(mine + row * kGroupedStagePitch + part * 2);
                    if (c0 + row < t.count && feature + part < p.features)
                        *reinterpret_cast<uint4*>(out + (t.row + c0 + row) * p.ld_out + feature + part) = v;
                }
                __syncwarp();
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&tempty_bar[buf]);
        }
        if (lane == 0) ptx::tma_store_wait_all<0>();             // shared memory stays until it has been read
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        __syncwarp();
        ptx::tmem_dealloc(tmem, static_cast<uint32_t>(p.tmem_cols));
    }
}

}  // namespace tdx
