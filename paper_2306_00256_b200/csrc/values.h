// Internal: fp32 and bf16 storage behind one set of loads and stores; arithmetic is fp32 throughout.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ceca.h"

namespace ceca {

using bf16 = __nv_bfloat16;

#ifdef __CUDACC__
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void narrow(float *p, float v) { *p = v; }
__device__ __forceinline__ void narrow(bf16 *p, float v) { *p = __float2bfloat16_rn(v); }

// C values in fp32; two are computed on together (f32x2).
template <int C> struct Val;
template <> struct Val<1> { float x; };
template <> struct Val<2> { float x, y; };
__device__ __forceinline__ uint64_t bits(Val<2> v) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
  return r;
}
__device__ __forceinline__ Val<2> halves(uint64_t r) {
  Val<2> v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ __forceinline__ Val<1> mul(Val<1> a, Val<1> b) { return {a.x * b.x}; }
__device__ __forceinline__ Val<1> add(Val<1> a, Val<1> b) { return {a.x + b.x}; }
__device__ __forceinline__ Val<1> sub(Val<1> a, Val<1> b) { return {a.x - b.x}; }
__device__ __forceinline__ Val<1> fma(Val<1> a, Val<1> b, Val<1> c) { return {fmaf(a.x, b.x, c.x)}; }
__device__ __forceinline__ Val<2> mul(Val<2> a, Val<2> b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return halves(r);
}
__device__ __forceinline__ Val<2> add(Val<2> a, Val<2> b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return halves(r);
}
__device__ __forceinline__ Val<2> fma(Val<2> a, Val<2> b, Val<2> c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return halves(r);
}
__device__ __forceinline__ Val<2> sub(Val<2> a, Val<2> b) { return fma(b, Val<2>{-1.f, -1.f}, a); }
template <int C> __device__ __forceinline__ Val<C> all(float v);
template <> __device__ __forceinline__ Val<1> all<1>(float v) { return {v}; }
template <> __device__ __forceinline__ Val<2> all<2>(float v) { return {v, v}; }
__device__ __forceinline__ Val<1> read(const float *p, Val<1>) { return {*p}; }
__device__ __forceinline__ Val<2> read(const float *p, Val<2>) {   // shared memory, 8-byte aligned
  const float2 v = *reinterpret_cast<const float2 *>(p);
  return {v.x, v.y};
}
__device__ __forceinline__ void write(float *p, Val<1> v) { *p = v.x; }
__device__ __forceinline__ void write(float *p, Val<2> v) { *reinterpret_cast<float2 *>(p) = make_float2(v.x, v.y); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
#endif

template <typename T> struct TypeOf;
template <> struct TypeOf<float> { static constexpr int32_t value = DSGD_F32; };
template <> struct TypeOf<bf16> { static constexpr int32_t value = DSGD_BF16; };

inline bool is_type(int32_t t) { return t == DSGD_F32 || t == DSGD_BF16; }
inline bool is_index(int32_t t) { return t == DSGD_I32 || t == DSGD_I64; }
inline int64_t type_bytes(int32_t t) { return t == DSGD_BF16 ? 2 : 4; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

#ifdef __CUDACC__
// A kernel that another one of the same call follows lets it begin early (follow_early); that one, launched with
// launch_after, does what does not depend on the first and then waits for its end (after_first).
__device__ __forceinline__ void follow_early() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_first() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename Args>
inline cudaError_t launch_after(void (*kernel)(const Args), const Args &p, dim3 grid, int threads, int bytes, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
#endif

}  // namespace ceca
