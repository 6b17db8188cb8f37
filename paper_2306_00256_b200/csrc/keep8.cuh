// Internal: blocks of 32 channels in 8 bits with one exponent.
#pragma once
#include "values.h"

namespace ceca {

constexpr int kBlock8 = 32;

__host__ __device__ constexpr int64_t blocks8(int64_t d) { return (d + kBlock8 - 1) / kBlock8; }
__host__ __device__ constexpr int64_t kept_row_bytes(int64_t d) { return (d + blocks8(d) + 15) / 16 * 16; }

#ifdef __CUDACC__
// The exponent byte of a block whose largest magnitude has these bits (the sign taken off; a NaN is above all): 255 for one that
// is not finite, at least 6, so that no scale below leaves the normal numbers.
__device__ __forceinline__ uint32_t exponent8(uint32_t top) { return max(top >> 23, 6u); }
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// What x is multiplied by before it is rounded (0 for a block of NaNs), and the step that a whole number stands for.
__device__ __forceinline__ float scale8(uint32_t e) { return e == 255u ? 0.f : __uint_as_float((260u - e) << 23); }
__device__ __forceinline__ float step8(uint32_t e) { return e == 255u ? NAN : __uint_as_float(e << 23) * 0.015625f; }
__device__ __forceinline__ int hold8(float x, float scale) {   // (in a block of NaNs x may be one: 0 all the same)
  return max(-127, min(127, __float2int_rn(x * scale)));
}
#endif

}  // namespace ceca
