// What the kernels of the sequence operators (causal convolution, selective scan, 4-bit products) share: element
// conversion, the elementwise functions, packed fp32 pairs, and the rows and state slots of a sequence.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace tdx {

// recorded in the device status word (see kStatusBounds in simt_kernels.cuh): a sequence offset or a state slot that
// lies outside the caller's tensors; that sequence or state is skipped
enum : int { kStatusSequence = 16 };

// compile-time answers for generic lambdas
struct SeqYes { static constexpr bool value = true; };
struct SeqNo { static constexpr bool value = false; };

// ---------------------------------------------------------------- elements
__device__ __forceinline__ float seq_to_float(float v) { return v; }
__device__ __forceinline__ float seq_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T seq_from_float(float v);
template <>
__device__ __forceinline__ float seq_from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 seq_from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// VEC elements that move as one access: 16, 8, 4 or 2 bytes
template <int BYTES> struct SeqBits;
template <> struct SeqBits<16> { typedef uint4 type; };
template <> struct SeqBits<8> { typedef uint2 type; };
template <> struct SeqBits<4> { typedef uint32_t type; };
template <> struct SeqBits<2> { typedef uint16_t type; };
template <typename T, int VEC>
struct SeqVec {
    typedef typename SeqBits<VEC * sizeof(T)>::type bits_t;
    union { bits_t bits; T v[VEC]; };
    __device__ __forceinline__ SeqVec() {}
};
template <typename T, int VEC>
__device__ __forceinline__ SeqVec<T, VEC> seq_load(const T* p) {
    SeqVec<T, VEC> r;
    r.bits = __ldg(reinterpret_cast<const typename SeqVec<T, VEC>::bits_t*>(p));
    return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void seq_store(T* p, const float (&f)[VEC]) {
    SeqVec<T, VEC> r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = seq_from_float<T>(f[i]);
    *reinterpret_cast<typename SeqVec<T, VEC>::bits_t*>(p) = r.bits;
}
template <typename T, int VEC>
__device__ __forceinline__ void seq_unpack(const SeqVec<T, VEC>& r, float (&f)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = seq_to_float(r.v[i]);
}

// ---------------------------------------------------------------- elementwise functions
constexpr float kLog2e = 1.4426950408889634f;
// 2^x by the special-function unit (error about 2^-22 of the result; results under 2^-126 are 0)
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// exp(v).  fp32 activations get expf; behind bf16 ones (2^-9) the rounding of v * log2(e), up to |v| * 2^-24, does not show.
template <typename T>
__device__ __forceinline__ float seq_exp(float v) { return sizeof(T) == 4 ? expf(v) : fast_exp2(v * kLog2e); }
template <typename T>
__device__ __forceinline__ float sigmoid_f(float v) { return fast_rcp(1.0f + seq_exp<T>(-v)); }
// log(1 + exp(v)) = max(v, 0) + log1p(u), u = exp(-|v|) in (0, 1], and log1p(u) = 2 atanh(r / 2), r = 2 u / (2 + u) <= 2/3: no
// cancellation for any v, so the result keeps its relative accuracy where it is tiny.  2 atanh(r / 2) / r is a polynomial of
// degree 4 in r^2, fitted by least squares in relative error (7.6e-9 with these coefficients).
__device__ __forceinline__ float softplus_from_exp(float v, float u) {
    const float r = u * fast_rcp(fmaf(u, 0.5f, 1.0f)), q = r * r;
    float p = fmaf(q, 0.14080727f / 256.0f, 0.13982172f / 64.0f);
    p = fmaf(q, p, 0.20012326f / 16.0f);
    p = fmaf(q, p, 0.3333316f / 4.0f);
    p = fmaf(q, p, 1.0f);
    return fmaf(r, p, fmaxf(v, 0.0f));
}
template <typename T>
__device__ __forceinline__ float softplus_f(float v) { return softplus_from_exp(v, seq_exp<T>(-fabsf(v))); }
// the same with its derivative, the sigmoid of v, from the same exponential
template <typename T>
__device__ __forceinline__ float softplus_grad_f(float v, float& grad) {
    const float u = seq_exp<T>(-fabsf(v));
    grad = (v >= 0.0f ? 1.0f : u) * fast_rcp(1.0f + u);
    return softplus_from_exp(v, u);
}

// ---------------------------------------------------------------- pairs of fp32 (one instruction for two values)
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// ---------------------------------------------------------------- sequences
// Sequence b occupies rows [first, first + len).  Without offsets the batch is dense.  Offsets live on the device, so the
// kernels check them: a sequence that leaves [0, rows) or is longer than max_len is reported and treated as empty.
struct SeqRange { long long first; int len; };
__device__ __forceinline__ bool seq_accepted(int lo, int hi, long long max_len, long long rows) {
    return lo >= 0 && hi >= lo && hi <= rows && hi - lo <= max_len;
}
__device__ __forceinline__ SeqRange seq_range(const int* __restrict__ offsets, long long b, long long max_len, long long rows, int* status) {
    SeqRange r;
    if (offsets == nullptr) {
        r.first = b * max_len;
        r.len = static_cast<int>(max_len);
        return r;
    }
    const int lo = __ldg(offsets + b), hi = __ldg(offsets + b + 1);
    if (!seq_accepted(lo, hi, max_len, rows)) {
        atomicCAS(status, 0, kStatusSequence);
        r.first = 0;
        r.len = 0;
        return r;
    }
    r.first = lo;
    r.len = hi - lo;
    return r;
}
// Sequences are cut into pieces of `piece` rows, each worked on by a block (or a few).  A dense batch has `dense` pieces per
// sequence.  Packed ones share rows / piece + batch numbers: sequence b starts at number offsets[b] / piece + b, which leaves
// room for ceil(len / piece) of them and at least one, whatever the lengths are; the few numbers left over are pieces with no
// rows.  Number i belongs to the last sequence that starts at or before i.  No sequences have no pieces: there is no offset behind the first.
constexpr int kNoPiece = 1 << 29;
struct SeqPiece { long long b; int index; };
__host__ __device__ __forceinline__ long long seq_pieces(bool packed, long long batch, long long rows, long long dense, long long piece) {
    return !packed ? batch * dense : batch > 0 ? rows / piece + batch : 0;
}
__device__ __forceinline__ SeqPiece seq_piece(const int* __restrict__ offsets, long long batch, long long dense, long long piece, long long i) {
    SeqPiece r;
    if (offsets == nullptr) {
        r.b = i / dense;
        r.index = static_cast<int>(i - r.b * dense);
        return r;
    }
    long long lo = 0, hi = batch - 1;
    while (lo < hi) {
        const long long mid = (lo + hi + 1) / 2;
        if (__ldg(offsets + mid) / piece + mid <= i) lo = mid;
        else hi = mid - 1;
    }
    r.b = lo;
    const long long index = i - (__ldg(offsets + lo) / piece + lo);
    r.index = index < 0 || index > kNoPiece ? kNoPiece : static_cast<int>(index);   // in front of the first sequence: no rows
    return r;
}
// seq_piece relies on ascending offsets: where they do not ascend, some sequences are found by no piece.  So that they are reported
// all the same, one thread of the pieces 0 .. batch - 1 (there are at least as many) looks at the sequence of the piece's number.
__device__ __forceinline__ void seq_check(const int* __restrict__ offsets, long long number, long long batch, long long max_len, long long rows, int* status) {
    if (offsets != nullptr && threadIdx.x == 0 && number < batch) seq_range(offsets, number, max_len, rows, status);
}
// Whether a row belongs to a sequence that was worked on: the last one that starts at or before it.
__device__ __forceinline__ bool seq_has_row(const int* __restrict__ offsets, long long batch, long long max_len, long long rows, long long row) {
    long long lo = 0, hi = batch - 1;
    while (lo < hi) {
        const long long mid = (lo + hi + 1) / 2;
        if (__ldg(offsets + mid) <= row) lo = mid;
        else hi = mid - 1;
    }
    const int from = __ldg(offsets + lo), to = __ldg(offsets + lo + 1);
    return from <= row && row < to && seq_accepted(from, to, max_len, rows);
}
// Slot of sequence (or batch row) b in the state tensors; negative: it has no state.
__device__ __forceinline__ long long state_slot(const int* __restrict__ slots, long long b, long long n_slots, int* status) {
    const long long s = slots == nullptr ? b : __ldg(slots + b);
    if (s >= n_slots) {
        atomicCAS(status, 0, kStatusSequence);
        return -1;
    }
    return s;
}

__device__ __forceinline__ void seq_grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void seq_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace tdx
