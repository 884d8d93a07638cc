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
    // tensor-core kernels
    int steps, groups;               // of K: steps of 128, groups
    int per;                         // steps of a warp's range
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
    const float range = hi - lo, fifteenth = isinf(range) ? hi / 15.0f - lo / 15.0f : range / 15.0f;      // the range may overflow
    const T stored = seq_from_float<T>(zeros ? fifteenth : fmaxf(hi, -lo) / 7.0f);
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
// mask and a multiplication make bf16 pairs of the exact (q[j] - zero) / 64 and (q[j + 4] - zero) / 64 (see w4_pair).  The products of
// a group are summed in fp32 by the tensor cores and enter the result times the group's scale, so weights are never rounded.
//
// bf16: a column of B is a row of x.  fp32: each value of x is cut into three bf16 pieces (8 + 8 + 8 significant bits, no
// remainder), three neighbouring columns, so that the products are those of the full fp32 value.  A warp cuts the 128 k it is
// about to use once, through shared memory.
//
// Two kernels.  Up to 8 rows of x (fp32: 2), small enough for shared memory: w4_staged_kernel, a block has 16 or 32 rows of W, its
// warps take ranges of K, and x is laid out in shared memory once, in the order in which it is used.  Else w4_direct_kernel.
// Either way the warps' sums are joined in shared memory in the order of the warps.
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Nibbles j and j + 4 of a word as a bf16 pair (q - zero) / 64.  The bits of a bf16 below 0x0100 are a fixed-point number (subnormals
// and the first binade): q at bits 0 .. 3 of a half is q * 2^-133, at bits 4 .. 7 it is 16 q * 2^-133, so a mask alone gives
// a number, one multiplication by 2^127 or 2^123 with the zero as addend makes it (q - zero) / 64 exactly, and a shift is needed
// for every second pair only.  offset: the pair -zero / 64.  (In assembly: through __nv_bfloat162 the compiler takes the pairs
// apart and puts them together again, which tripled the integer instructions.)
constexpr float kW4Scale = 64.0f;
__device__ __forceinline__ uint32_t w4_pair(uint32_t word, int j, uint32_t offset) {
    const uint32_t bits = (j < 2 ? word : word >> 8) & (j & 1 ? 0x00F000F0u : 0x000F000Fu);
    uint32_t v;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v) : "r"(bits), "r"(j & 1 ? 0x7D007D00u : 0x7F007F00u), "r"(offset));
    return v;
}
__device__ __forceinline__ uint32_t w4_offset(int zero) {
    const float v = static_cast<float>(zero) * (-1.0f / kW4Scale);
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(v));
    return r;
}
// The three bf16 pieces of an fp32 value, by truncation, as the upper halves of words; what is not finite is all in the first.
__device__ __forceinline__ void w4_pieces(float v, uint32_t (&piece)[3]) {
    const uint32_t bits = __float_as_uint(v);
    const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
    const float r1 = finite ? v - __uint_as_float(bits & 0xffff0000u) : 0.0f;
    const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
    piece[0] = finite ? bits : bits | (bits & 0x007fffffu ? 0x00400000u : 0u);
    piece[1] = __float_as_uint(r1);
    piece[2] = __float_as_uint(r2);
}

__device__ __forceinline__ uint32_t w4_piece(float v, int piece) {
    uint32_t p[3];
    w4_pieces(v, p);
    return p[piece == 0 ? 0 : piece == 1 ? 1 : 2];
}

template <typename T> struct W4Columns;
template <> struct W4Columns<__nv_bfloat16> { static constexpr int kRows = 8, kPieces = 1; };   // rows of x in 8 columns
template <> struct W4Columns<float> { static constexpr int kRows = 2, kPieces = 3; };

constexpr int kW4Step = 128;         // k of a step
constexpr int kW4Rows = 16;          // rows of W of a warp

// Shared memory: the ring of weights (and, when it is no longer needed, the warps' sums), x, scales.
template <typename T>
__host__ __device__ inline size_t w4_x_bytes(long long steps, long long rows_of_x) {
    return static_cast<size_t>(steps) * rows_of_x * W4Columns<T>::kPieces * kW4Step * 2;
}
// pairs (scale, offset) between two rows of W: an odd number, so that eight rows start in different banks
__host__ __device__ constexpr int w4_scale_pitch(int groups) { return groups | 1; }
constexpr size_t kW4RingBytes = 4 * 2 * 16;      // of a thread (kW4Depth steps); a warp's sums are never longer than its part

// 16 bytes of x in shared memory: eight neighbouring k (an octet) of a row of x (of one piece of it) as pairs (j, j + 4).  Octet o of
// a step belongs to thread t = lane % 4, which meets it with its word `word` of the step:
//   o = (word / WORDS) * 4 * WORDS + t * WORDS + word % WORDS;  place: [step][word][row of x][piece][t].
template <typename T> struct W4Octet;
template <> struct W4Octet<__nv_bfloat16> {
    uint4 q;
    __device__ __forceinline__ void load(const __nv_bfloat16* from, bool there) {
        q = make_uint4(0u, 0u, 0u, 0u);
        if (there) q = __ldg(reinterpret_cast<const uint4*>(from));
    }
    __device__ __forceinline__ void store(uint4* to) const {
        *to = make_uint4(__byte_perm(q.x, q.z, 0x5410), __byte_perm(q.x, q.z, 0x7632), __byte_perm(q.y, q.w, 0x5410), __byte_perm(q.y, q.w, 0x7632));
    }
};
template <> struct W4Octet<float> {
    float4 lo, hi;
    __device__ __forceinline__ void load(const float* from, bool there) {
        lo = hi = make_float4(0.f, 0.f, 0.f, 0.f);
        if (there) {
            lo = __ldg(reinterpret_cast<const float4*>(from));
            hi = __ldg(reinterpret_cast<const float4*>(from) + 1);
        }
    }
    __device__ __forceinline__ void store(uint4* to) const {
        const float l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w};
        uint32_t pairs[3][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t p[3], q[3];
            w4_pieces(l[j], p);
            w4_pieces(h[j], q);
#pragma unroll
            for (int c = 0; c < 3; ++c) pairs[c][j] = __byte_perm(p[c], q[c], 0x7632);
        }
#pragma unroll
        for (int c = 0; c < 3; ++c) to[4 * c] = make_uint4(pairs[c][0], pairs[c][1], pairs[c][2], pairs[c][3]);
    }
};
template <typename T, int WORDS>
__device__ __forceinline__ void w4_lay_out(uint4* step_x, int o, int row, int rows_of_x, const W4Octet<T>& octet) {
    const int unit = o / (4 * WORDS), in = o % (4 * WORDS), t = in / WORDS, word = unit * WORDS + in % WORDS;
    octet.store(step_x + ((word * rows_of_x + row) * W4Columns<T>::kPieces) * 4 + t);
}

// A thread's weights of a step (two rows, 16 bytes each) travel through shared memory by asynchronous copies, kW4Depth steps
// ahead, into a place that only this thread uses: a loop that prefetched into registers waited for its newest loads (about
// twice the time for 8192 x 8192 weights in the form of that time), and a ring costs no registers and little code.
// Whole calls in bf16: 7.0 us for one token and 4096 x 4096 weights (4.6 in a graph; the host's part bounds it), 13.4 us for
// 8192 x 8192 (2.6 TB/s; start-up, layout of x and the join are about half of it).
constexpr int kW4Depth = 4;
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int BYTES>
__device__ __forceinline__ void async_copy(void* to, const void* from) {
    const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
// ring: this thread's place of depth 0, row g; row g + 8 and the next depth follow `threads` and 2 * threads places behind
template <int WORDS>
struct W4Reader {
    static constexpr int kUnits = 4 / WORDS, kGroup = 32 * WORDS;      // kUnits: groups of a step
    const uint8_t *w0, *w1;
    uint4* ring;
    int threads, left;                                                 // left: groups from here to the end of the row
    __device__ __forceinline__ void place(const W4Params& p, long long row, int step, int g, int t) {
        const long long pitch = p.K / 2, at = t * (4 * WORDS) + static_cast<long long>(step) * (kW4Step / 2);
        w0 = p.weight + min(row + g, p.N - 1) * pitch + at;
        w1 = p.weight + min(row + g + 8, p.N - 1) * pitch + at;
        left = p.groups - step * kUnits;
    }
    __device__ __forceinline__ void fetch(int depth) {                 // and moves on by a step
        uint4* to = ring + depth * 2 * threads;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            if (kUnits == 1 || u < left) {                             // groups past the end are skipped by w4_multiply
                async_copy<4 * WORDS>(reinterpret_cast<uint32_t*>(to) + u * WORDS, w0 + u * (kGroup / 2));
                async_copy<4 * WORDS>(reinterpret_cast<uint32_t*>(to + threads) + u * WORDS, w1 + u * (kGroup / 2));
            }
        }
        w0 += kW4Step / 2;
        w1 += kW4Step / 2;
        left -= kUnits;
    }
};
// Scales and zeros of `rows` rows, groups first .. first + count - 1, for w4_multiply: pairs (scale, offset) [row][group], rows
// `pitch` pairs apart
template <typename T>
__device__ __forceinline__ void w4_lay_out_scales(const W4Params& p, float2* to, int pitch, long long n0, int rows, int first, int count, int tid, int threads) {
    for (int r = tid / 32; r < rows; r += threads / 32) {
        const long long at = min(n0 + r, p.N - 1) * p.groups + first;
        for (int i = tid % 32; i < count; i += 32) {
            const float s = seq_to_float(static_cast<const T*>(p.scales)[at + i]);
            const uint32_t o = p.zeros ? w4_offset(p.zeros[at + i]) : 0xBE00BE00u;         // - 8 / 64
            to[r * pitch + i] = make_float2(s, __uint_as_float(o));
        }
    }
}
// acc += the step's products.  q0, q1: the weights of rows g and g + 8; x: the step's x in shared memory; at: this thread's place
// in it for each tile; word_x: 16-byte pieces of x per word; scales: of rows g and g + 8 from the step's first group on; units:
// groups that the step has.
template <int WORDS, int TILES>
__device__ __forceinline__ void w4_multiply(const uint4& q0, const uint4& q1, const uint4* x, const int (&at)[TILES], int word_x, const float2* scales0,
                                            const float2* scales1, int units, float (&acc)[TILES][4]) {
    const uint32_t w0[4] = {q0.x, q0.y, q0.z, q0.w}, w1[4] = {q1.x, q1.y, q1.z, q1.w};
#pragma unroll
    for (int u = 0; u < 4 / WORDS; ++u) {
        if (WORDS < 4 && u >= units) break;
        const float2 s0 = scales0[u], s1 = scales1[u];
        const uint32_t o0 = __float_as_uint(s0.y), o1 = __float_as_uint(s1.y);
        float sum[TILES][4];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[i][j] = 0.0f;
#pragma unroll
        for (int v = 0; v < WORDS; ++v) {
            uint32_t a0[4], a1[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a0[j] = w4_pair(w0[u * WORDS + v], j, o0);
                a1[j] = w4_pair(w1[u * WORDS + v], j, o1);
            }
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const uint4 b = x[(u * WORDS + v) * word_x + at[i]];
                mma_bf16(sum[i], a0[0], a1[0], a0[1], a1[1], b.x, b.y);
                mma_bf16(sum[i], a0[2], a1[2], a0[3], a1[3], b.z, b.w);
            }
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            acc[i][0] = fmaf(s0.x, sum[i][0], acc[i][0]);
            acc[i][1] = fmaf(s0.x, sum[i][1], acc[i][1]);
            acc[i][2] = fmaf(s1.x, sum[i][2], acc[i][2]);
            acc[i][3] = fmaf(s1.x, sum[i][3], acc[i][3]);
        }
    }
}
// This thread's place in a word of x for each tile.  Columns without a row of x (or, for fp32, without a piece) repeat another
// one: a column's sums depend on nothing else, and those are not written.
template <typename T, int TILES>
__device__ __forceinline__ void w4_columns(int rows_of_x, int g, int t, int (&at)[TILES]) {
    constexpr int kX = W4Columns<T>::kRows, kP = W4Columns<T>::kPieces;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int row = min(i * kX + (kP == 1 ? g : min(g / 3, 1)), rows_of_x - 1);
        at[i] = (row * kP + (kP == 1 ? 0 : g % 3)) * 4 + t;
    }
}
template <int TILES>
__device__ __forceinline__ void w4_keep_sums(float* sums, int g, int t, const float (&acc)[TILES][4]) {
    constexpr int kSumRow = TILES * 8 + 1;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        float* to = sums + g * kSumRow + i * 8 + 2 * t;
        to[0] = acc[i][0];
        to[1] = acc[i][1];
        to[8 * kSumRow] = acc[i][2];
        to[8 * kSumRow + 1] = acc[i][3];
    }
}

// WORDS = group / 32 words of weights per thread, row and group; BLOCKS: sets of 16 rows of W that a block goes
// through, so that x is laid out for them once and their loads follow each other without a gap.
template <typename T, int WORDS, int BLOCKS>
__global__ void __launch_bounds__(512) w4_staged_kernel(const __grid_constant__ W4Params p) {
    constexpr int kUnits = 4 / WORDS, kX = W4Columns<T>::kRows, kP = W4Columns<T>::kPieces, kOctets = kW4Step / 8;
    extern __shared__ __align__(16) unsigned char w4_smem[];
    seq_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = blockDim.x, g = lane >> 2, t = lane & 3;
    const long long n0 = blockIdx.x * static_cast<long long>(kW4Rows * BLOCKS);
    const int rows_of_x = static_cast<int>(p.M), first = min(p.steps, warp * p.per), count = min(p.steps, first + p.per) - first;
    const int word_x = rows_of_x * kP * 4, pitch = w4_scale_pitch(p.groups);
    uint4* ring = reinterpret_cast<uint4*>(w4_smem);
    uint4* xs = ring + kW4Depth * 2 * threads;
    float2* scales = reinterpret_cast<float2*>(xs + p.steps * 4 * word_x);
    float* sums = reinterpret_cast<float*>(w4_smem);                   // in place of the ring, at the end
    W4Reader<WORDS> reader;
    reader.place(p, n0, first, g, t);
    reader.ring = ring + threadIdx.x;
    reader.threads = threads;
    seq_grid_wait();
    int ahead = 0, ahead_block = 0;                                    // step and block of the next fetch
    auto fetch = [&](int depth) {
        if (ahead == count && ++ahead_block < BLOCKS) {
            ahead = 0;
            reader.place(p, n0 + ahead_block * kW4Rows, first, g, t);
        }
        if (ahead < count) {
            reader.fetch(depth);
            ++ahead;
        }
        async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < kW4Depth; ++i) fetch(i);
    const int octets = p.steps * kOctets;
#pragma unroll 1
    for (int row = 0; row < rows_of_x; ++row) {
        const T* from = static_cast<const T*>(p.x) + row * p.ld_x;
        for (int o = threadIdx.x; o < octets; o += threads) {
            W4Octet<T> octet;
            octet.load(from + o * 8, o * 8LL < p.K);
            w4_lay_out<T, WORDS>(xs + o / kOctets * (4 * word_x), o % kOctets, row, rows_of_x, octet);
        }
    }
    w4_lay_out_scales<T>(p, scales, pitch, n0, kW4Rows * BLOCKS, 0, p.groups, threadIdx.x, threads);
    int at[1];
    w4_columns<T, 1>(rows_of_x, g, t, at);
    float acc[BLOCKS][1][4];
    __syncthreads();
    int depth = 0;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][0][j] = 0.0f;
        const uint4* x = xs + first * (4 * word_x);
        const float2 *s0 = scales + (b * kW4Rows + g) * pitch + first * kUnits, *s1 = s0 + 8 * pitch;
        int left = p.groups - first * kUnits;
#pragma unroll 1
        for (int step = 0; step < count; ++step) {
            async_wait<kW4Depth - 1>();
            const uint4* from = reader.ring + depth * 2 * threads;
            const uint4 q0 = from[0], q1 = from[threads];
            w4_multiply<WORDS, 1>(q0, q1, x, at, word_x, s0, s1, left, acc[b]);
            fetch(depth);
            depth = depth + 1 == kW4Depth ? 0 : depth + 1;
            x += 4 * word_x;
            s0 += kUnits;
            s1 += kUnits;
            left -= kUnits;
        }
    }
    async_wait<0>();
    __syncthreads();
    constexpr int kSumRow = 9, kSumWarp = kW4Rows * kSumRow;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) w4_keep_sums<1>(sums + (warp * BLOCKS + b) * kSumWarp, g, t, acc[b]);
    __syncthreads();
    constexpr int kRowsOfW = kW4Rows * BLOCKS;
    for (int o = threadIdx.x; o < kRowsOfW * rows_of_x; o += threads) {
        const int row = o % kRowsOfW, in = o / kRowsOfW;
        const long long n = n0 + row;
        if (n < p.N) {
            const float* from = sums + row * kSumRow + in % kX * kP;
            float s = 0.0f;
#pragma unroll
            for (int c = kP - 1; c >= 0; --c)                          // the small pieces first
                for (int r = 0; r < threads / 32; ++r) s += from[r * (BLOCKS * kSumWarp) + c];
            static_cast<T*>(p.y)[in * p.ld_y + n] = seq_from_float<T>(s * kW4Scale);
        }
    }
}

// Every thread reads the x that it needs itself, 16 bytes at a time (x is read by every block, and comes from L1 and
// L2).  TILES: tiles of 8 columns.
template <typename T, int WORDS, int TILES>
__global__ void __launch_bounds__(256) w4_direct_kernel(const __grid_constant__ W4Params p) {
    constexpr int kWarps = 8, kGroup = 32 * WORDS, kPer = 8 * WORDS;   // kPer: weights of a thread, row and group
    constexpr int kAhead = 8 / WORDS;                                  // groups in flight: 32 bytes a row
    __shared__ float red[kWarps][16][TILES * 8 + 1];
    seq_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const long long n0 = blockIdx.x * 16LL, m0 = static_cast<long long>(blockIdx.y) * W4Columns<T>::kRows * TILES;
    const int groups = p.groups;
    const long long pitch = p.K / 2;
    const long long r0 = min(n0 + g, p.N - 1), r1 = min(n0 + g + 8, p.N - 1);
    const uint8_t* wp0 = p.weight + r0 * pitch + t * (4 * WORDS);
    const uint8_t* wp1 = p.weight + r1 * pitch + t * (4 * WORDS);
    const T* sp0 = static_cast<const T*>(p.scales) + r0 * groups;
    const T* sp1 = static_cast<const T*>(p.scales) + r1 * groups;
    const uint8_t* zp0 = p.zeros ? p.zeros + r0 * groups : nullptr;
    const uint8_t* zp1 = p.zeros ? p.zeros + r1 * groups : nullptr;
    // This thread's column of each tile.  Columns without a row of x (or, for fp32, without a piece) repeat another one: a column's
    // sums depend on nothing else, and those are not written.
    const T* xp[TILES];
    const int piece = W4Columns<T>::kPieces == 1 ? 0 : g % 3;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const long long m = m0 + i * W4Columns<T>::kRows + (W4Columns<T>::kPieces == 1 ? g : min(g / 3, 1));
        xp[i] = static_cast<const T*>(p.x) + min(m, p.M - 1) * p.ld_x + t * kPer;
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
            const uint32_t o0 = w4_offset(z0[slot]), o1 = w4_offset(z1[slot]);
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
                    uint32_t b[4];                                     // pairs (x[j], x[j + 4])
                    const T* x = xp[i] + static_cast<long long>(grp) * kGroup + w * 8;
                    if (sizeof(T) == 2) {
                        const uint4 v = __ldg(reinterpret_cast<const uint4*>(x));
                        b[0] = __byte_perm(v.x, v.z, 0x5410);
                        b[1] = __byte_perm(v.x, v.z, 0x7632);
                        b[2] = __byte_perm(v.y, v.w, 0x5410);
                        b[3] = __byte_perm(v.y, v.w, 0x7632);
                    } else {
                        const float4 lo = __ldg(reinterpret_cast<const float4*>(x)), hi = __ldg(reinterpret_cast<const float4*>(x) + 1);
                        b[0] = __byte_perm(w4_piece(lo.x, piece), w4_piece(hi.x, piece), 0x7632);
                        b[1] = __byte_perm(w4_piece(lo.y, piece), w4_piece(hi.y, piece), 0x7632);
                        b[2] = __byte_perm(w4_piece(lo.z, piece), w4_piece(hi.z, piece), 0x7632);
                        b[3] = __byte_perm(w4_piece(lo.w, piece), w4_piece(hi.w, piece), 0x7632);
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
        static_cast<T*>(p.y)[m * p.ld_y + n] = seq_from_float<T>(s * kW4Scale);
    }
}

}  // namespace tdx
