// What tdx_api.cu gives to the library's other translation units: errors, the device, the launch count, tensor maps.
#pragma once
#include <cuda.h>
#include <stddef.h>
#include <stdint.h>

namespace tdx_host {

struct Device { int sm_count, smem_optin; int* status; };

int fail_text(int status, const char* text);
void count_launch();
int get_device(Device* out);
// bf16 tensor, 128-byte (or 64-byte) swizzle, zero fill outside the tensor; maps are cached by their description
int bf16_map(const void* ptr, int rank, const uint64_t* dims, const uint64_t* strides_bytes, const uint32_t* box, CUtensorMap* out, int swizzle_bytes = 128);

}  // namespace tdx_host
