// Host side of the translation units beside tdx_api.cu: the names that seq_host.cuh goes by, and seq_host.cuh itself.
#pragma once
#include "tdx.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "layer_bridge.h"

namespace {

using tdx_host::count_launch;

int fail(int status, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return tdx_host::fail_text(status, buf);
}

#define TDX_CUDA(expr)                                                                                   \
    do {                                                                                                 \
        cudaError_t e_ = (expr);                                                                         \
        if (e_ != cudaSuccess) return fail(TDX_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_)); \
    } while (0)

constexpr int kSmemLimitDefault = 232448;  // 227 KiB opt-in limit of sm_100
constexpr int kDefaultSmCount = 148;
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

#include "seq_host.cuh"
