// The layout of the block summaries and the whole numbers that keys and queries are coded in, as include/ecoserve.h has them.
#pragma once

#include "common.h"

namespace eco {

constexpr int kNotFinite = 127;  // the exponent of a block that holds a NaN or an infinity

// Channels of one side of a record: head_dim, rounded up to half of the 64 bytes that a matrix instruction takes at a time.
__host__ __device__ inline int summary_channels(int D) { return (D + 31) / 32 * 32; }
inline size_t summary_code_bytes(const ecoserve_layout& L) {
  return (size_t)L.num_blocks * L.num_kv_heads * 2 * summary_channels(L.head_dim);
}

}  // namespace eco

#if defined(__HIPCC__)
namespace eco {

// The smallest e >= -126 with size <= 127 * 2^e, for finite size >= 0: size = 1.m * 2^(x - 127), and 127 * 2^e is 1.111111 (seven binary
// digits) times a power of two.
__device__ __forceinline__ int code_exponent(float size) {
  const uint32_t u = __float_as_uint(size);
  return max((int)(u >> 23) - 133 + ((u & 0x7fffffu) > 0x7e0000u ? 1 : 0), -126);
}

}  // namespace eco
#endif
