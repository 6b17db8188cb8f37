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
// bytes `from` and from + 1 of w, two whole numbers: (x + 128) + 2^23, less 2^23 + 128
__device__ __forceinline__ Val<2> whole_numbers(uint32_t w, int from) {
  w ^= 0x80808080u;
  const Val<2> v = {__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | from)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | (from + 1)))};
  return add(v, all<2>(-8388736.f));
}
// four of them, of x: rounded to the nearest in the low bits of a sum with 1.5 2^23
__device__ __forceinline__ uint32_t hold_four(Val<2> x, Val<2> y, Val<2> by) {
  const auto low = [](float v) { return __float_as_uint(fminf(fmaxf(v, -127.f), 127.f) + 12582912.f); };
  x = mul(x, by);
  y = mul(y, by);
  return __byte_perm(__byte_perm(low(x.x), low(x.y), 0x0040), __byte_perm(low(y.x), low(y.y), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t greatest(uint32_t top, Val<2> x) { return max(top, max(magnitude(x.x), magnitude(x.y))); }
__device__ __forceinline__ uint32_t pack_bf16(Val<2> x) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ Val<2> unpack_bf16(uint32_t x) { return {__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)}; }
#endif

}  // namespace ceca
