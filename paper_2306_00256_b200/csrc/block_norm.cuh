// Internal: the end of a block and the start of the next, and its gradient.
#pragma once
#include <cuda_runtime.h>

#include "ceca.h"
#include "keep8.cuh"
#include "values.h"

namespace ceca {

struct BlockArgs {
  dsgd_rows_t h, y, gate, h_out, u, du, dh_out, dh, dy, dgate;   // `at` is NULL where there is none
  const void *w_pre, *w_post, *scale;
  void *dw_pre, *dw_post, *dscale;
  int64_t w_pre_stride, w_post_stride, scale_stride, dw_pre_stride, dw_post_stride, dscale_stride;
  float *stats;
  uint8_t *h8, *y8, *gate8;     // forward: what is kept; the gradient finds it in h, y, gate
  int64_t t, d, row_bytes;      // of a kept row
  int32_t n, stream_type, act_type, weights_type, silu, kept, accumulate;
  float eps;
  float2 *means;                // workspace: of rows (the form for wide ones)
  float *parts, *scale_parts;   // sums over some rows: n x parts x 2 x d, n x scale_count
  int32_t part_count, scale_count;
  int64_t part_rows;
};

#ifdef __CUDACC__
__device__ __forceinline__ float load(const void *p, int32_t type, int64_t i) {
  return type == DSGD_BF16 ? widen(static_cast<const bf16 *>(p)[i]) : static_cast<const float *>(p)[i];
}
__device__ __forceinline__ void store(void *p, int32_t type, int64_t i, float v) {
  if (type == DSGD_BF16) narrow(static_cast<bf16 *>(p) + i, v);
  else narrow(static_cast<float *>(p) + i, v);
}
__device__ __forceinline__ int64_t place(const dsgd_rows_t &x, int64_t agent, int64_t row) { return agent * x.agent_stride + row * x.row_stride; }

// A gate's factor and its derivative.  The smaller of sigmoid and 1 - sigmoid comes from the exponential itself, so neither loses digits.
struct Gate {
  float g, slope;
};
__device__ __forceinline__ Gate gate_of(float a, bool silu) {
  const float e = ex2(-1.4426950408889634f * fabsf(a)), r = rcp(1.f + e), s = e * r;   // (fabsf keeps a NaN)
  const float sig = a < 0.f ? s : r, slope = s * r;
  return silu ? Gate{a * sig, fmaf(a, slope, sig)} : Gate{sig, slope};
}

// 1 / sqrt(sum / d + eps) of a sum of squares; one that overflowed is taken again by `again`, of the values times 2^-100.
template <typename Again> __device__ __forceinline__ float inverse_rms(float sum, int64_t d, float eps, Again again) {
  float unit = 1.f;
  if (sum == INFINITY) {
    unit = 0x1p-100f;
    sum = again(unit);
  }
  return unit / sqrtf(fmaf(eps * unit, unit, sum / (float)d));
}
#endif

}  // namespace ceca
