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
// What x is multiplied by before it is rounded (0 for a block of NaNs), and the step that a whole number stands for: an infinity in a block of NaNs, whose
// whole numbers are 0.
__device__ __forceinline__ float scale8(uint32_t e) { return e == 255u ? 0.f : __uint_as_float((260u - e) << 23); }
__device__ __forceinline__ float step8(uint32_t e) { return __uint_as_float(e << 23) * 0.015625f; }
__device__ __forceinline__ int hold8(float x, float scale) {   // (in a block of NaNs x may be one: 0 all the same)
  return max(-127, min(127, __float2int_rn(x * scale)));
}
// bytes `from` and from + 1 of w, two whole numbers: (x + 128) + 2^23, less 2^23 + 128
__device__ __forceinline__ Val<2> whole_numbers(uint32_t w, int from) {
  w ^= 0x80808080u;
  const Val<2> v = {__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | from)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | (from + 1)))};
  return add(v, all<2>(-8388736.f));
}
// four of them, of x: rounded to the nearest in the low bits of a sum with 1.5 2^23.  `cut`: some are rounded to 128, which becomes 127.
__device__ __forceinline__ uint32_t hold_four(Val<2> x, Val<2> y, Val<2> by, bool cut) {
  x = mul(x, by);
  y = mul(y, by);
  if (cut) {
    const auto within = [](float v) { return fminf(fmaxf(v, -127.f), 127.f); };
    x = {within(x.x), within(x.y)};
    y = {within(y.x), within(y.y)};
  }
  x = add(x, all<2>(12582912.f));
  y = add(y, all<2>(12582912.f));
  return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040), __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
}
// Whether the largest of a block, of these bits, is held as more than 127: mantissas from 127.5 / 128 on.
__device__ __forceinline__ bool cut8(uint32_t top) { return (top & 0x7fffffu) >= 0x7f0000u; }
// The larger magnitude, as a number; a NaN if there is one.
__device__ __forceinline__ float greatest(float top, Val<2> x) {
  asm("{\n\t.reg .f32 a, b;\n\tabs.f32 a, %1;\n\tabs.f32 b, %2;\n\tmax.NaN.f32 %0, %0, a;\n\tmax.NaN.f32 %0, %0, b;\n\t}" : "+f"(top) : "f"(x.x), "f"(x.y));
  return top;
}
__device__ __forceinline__ uint32_t pack_bf16(Val<2> x) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ Val<2> unpack_bf16(uint32_t x) { return {__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)}; }
#endif

}  // namespace ceca
