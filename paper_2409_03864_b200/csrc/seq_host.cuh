// What the entry points of the sequence and layer operators share on the host: launches, argument checks, access widths.
// It goes by the names fail, count_launch, ceil_div and TDX_CUDA of the translation unit that includes it (host_state.cuh and
// host_config.cuh in tdx_api.cu, layer_host.cuh elsewhere).
#pragma once
#include <algorithm>
#include <atomic>
#include <climits>
#include <cstring>

namespace {

constexpr int64_t kSeqMaxLen = 1 << 30;

// Programmatic stream serialization: the launch overlaps the tail of the kernel in front of it in the stream; every kernel
// of this file waits for that kernel's end before it touches global memory.
template <typename... Params, typename... Given>
int launch_seq(void (*kernel)(Params...), int64_t grid_x, int64_t grid_y, int threads, size_t smem, cudaStream_t st, const Given&... given) {
    if (grid_x > INT_MAX || grid_y > 65535) return fail(TDX_ERR_UNSUPPORTED, "problem too large for one launch");
    cudaLaunchConfig_t lc;
    std::memset(&lc, 0, sizeof lc);
    lc.gridDim = dim3(static_cast<unsigned>(grid_x), static_cast<unsigned>(grid_y));
    lc.blockDim = dim3(static_cast<unsigned>(threads));
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    TDX_CUDA(cudaLaunchKernelEx(&lc, kernel, static_cast<Params>(given)...));
    count_launch();
    return TDX_OK;
}

// Lets a kernel have more than 48 KB of shared memory: `most` (as much as there is, for a kernel without static shared memory),
// remembered per device, so that later calls skip it.
template <typename Kernel>
int allow_smem(Kernel kernel, std::atomic<bool> (&known)[64], size_t bytes, int most = kSmemLimitDefault) {
    if (bytes <= 48 * 1024) return TDX_OK;
    int dev = 0;
    TDX_CUDA(cudaGetDevice(&dev));
    const bool listed = dev >= 0 && dev < 64;
    if (listed && known[dev].load(std::memory_order_acquire)) return TDX_OK;
    TDX_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    if (listed) known[dev].store(true, std::memory_order_release);
    return TDX_OK;
}

bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }
int64_t elem_bytes(int dtype) { return dtype == TDX_F32 ? 4 : 2; }

// A tensor argument: present where needed, aligned to its elements, rows at least as wide as they are used.
int check_tensor(const char* name, const void* p, bool needed, size_t align, int64_t ld = 0, int64_t width = 0) {
    if (p == nullptr) return needed ? fail(TDX_ERR_INVALID_ARG, "%s is NULL", name) : TDX_OK;
    if (misaligned(p, align)) return fail(TDX_ERR_ALIGNMENT, "%s is not aligned to its elements", name);
    if (ld > (1 << 24)) return fail(TDX_ERR_UNSUPPORTED, "ld_%s = %lld is above 2^24", name, (long long)ld);
    if (ld < width) return fail(TDX_ERR_INVALID_ARG, "ld_%s = %lld is less than the row's %lld elements", name, (long long)ld, (long long)width);
    return TDX_OK;
}
#define TDX_TRY(expr)        \
    do {                     \
        int rc_ = (expr);    \
        if (rc_) return rc_; \
    } while (0)

// The parts that a convolution and a scan share.  `step`: one row per sequence.
int check_sequences(int64_t batch, int64_t max_len, int64_t rows, int64_t channels, int dtype, const int32_t* offsets, bool step) {
    if (batch < 0 || channels < 0 || (!step && (max_len < 0 || rows < 0))) return fail(TDX_ERR_INVALID_ARG, "negative size");
    if (dtype != TDX_F32 && dtype != TDX_BF16) return fail(TDX_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (batch > INT_MAX || channels > INT_MAX) return fail(TDX_ERR_UNSUPPORTED, "batch or channels above 2^31 - 1");
    if (step) return TDX_OK;
    if (max_len > kSeqMaxLen) return fail(TDX_ERR_UNSUPPORTED, "sequences of more than 2^30 rows");
    if (offsets == nullptr) {
        if (rows != batch * max_len) return fail(TDX_ERR_INVALID_ARG, "rows = %lld is not batch * max_len", (long long)rows);
    } else {
        if (misaligned(offsets, 4)) return fail(TDX_ERR_ALIGNMENT, "seq_offsets is not aligned to its elements");
        if (rows > INT_MAX) return fail(TDX_ERR_UNSUPPORTED, "more than 2^31 - 1 packed rows");
    }
    return TDX_OK;
}
int check_states(bool used, int64_t batch, int64_t per_slot, int64_t* stride, const int32_t* slots, int64_t n_slots) {
    if (!used) return TDX_OK;
    if (misaligned(slots, 4)) return fail(TDX_ERR_ALIGNMENT, "slots is not aligned to its elements");
    if (n_slots < 0 || (slots == nullptr && n_slots < batch))
        return fail(TDX_ERR_INVALID_ARG, "n_slots = %lld does not hold the batch's states", (long long)n_slots);
    if (*stride == 0) *stride = per_slot;
    if (*stride < per_slot) return fail(TDX_ERR_INVALID_ARG, "state_stride is less than a state's %lld elements", (long long)per_slot);
    return TDX_OK;
}
int check_workspace(void* workspace, size_t have, size_t need) {
    if (need == 0) return TDX_OK;
    if (workspace == nullptr || have < need)
        return fail(TDX_ERR_WORKSPACE, "workspace of %llu bytes needed, %llu given", (unsigned long long)need, (unsigned long long)(workspace ? have : 0));
    if (misaligned(workspace, 256)) return fail(TDX_ERR_ALIGNMENT, "workspace is not 256-byte aligned");
    return TDX_OK;
}
size_t round_256(size_t bytes) { return (bytes + 255) / 256 * 256; }

int sm_count_or_default() {
    int dev = -1, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return kDefaultSmCount;
    }
    return n;
}

// Elements that every tensor of the call can be accessed by at once: the widest of `most`, ... , 1 that divides all bases
// and row strides.
struct Widest {
    int64_t bytes;
    explicit Widest(int64_t most) : bytes(most) {}
    void ptr(const void* p) { while (bytes > 1 && reinterpret_cast<uintptr_t>(p) % bytes) bytes /= 2; }
    void stride(int64_t elems, int64_t el) { while (bytes > 1 && (elems * el) % bytes) bytes /= 2; }
};

}  // namespace
