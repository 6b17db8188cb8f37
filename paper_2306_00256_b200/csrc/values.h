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
#endif

template <typename T> struct TypeOf;
template <> struct TypeOf<float> { static constexpr int32_t value = DSGD_F32; };
template <> struct TypeOf<bf16> { static constexpr int32_t value = DSGD_BF16; };

inline bool is_type(int32_t t) { return t == DSGD_F32 || t == DSGD_BF16; }
inline bool is_index(int32_t t) { return t == DSGD_I32 || t == DSGD_I64; }
inline int64_t type_bytes(int32_t t) { return t == DSGD_BF16 ? 2 : 4; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace ceca
