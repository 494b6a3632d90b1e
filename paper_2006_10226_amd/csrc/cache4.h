// Geometry of the 4-bit cache (include/qnn.h) for the kernels that write and
// read it.
#pragma once

#include "qnn_host.h"
#include "qnn_internal.h"

namespace qnn {

// Head dimension as stored.
__host__ __device__ constexpr int cache4_padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct Cache4Args {
    uint8_t *data;
    int32_t pages, shift;      // page size 1 << shift
    int32_t heads, dim;
    uint32_t page_bytes, head_bytes;
};

// QNN_OK and the kernel's form of a cache, or why it is refused.
qnn_status check_cache4(const qnn_cache4 &c, const char *what, Cache4Args *out);

// A record: the low byte is the zero point, the rest the scale's f32 bits.
__device__ __forceinline__ float rec_scale(uint32_t r) { return __builtin_bit_cast(float, r & 0xffffff00u); }
__device__ __forceinline__ float rec_zero(uint32_t r) { return (float)(r & 0xffu); }

}  // namespace qnn
