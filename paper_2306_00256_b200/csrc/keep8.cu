// Activations kept in 8 bits, and brought back.
#include <cuda_runtime.h>

#include <algorithm>

#include "ceca.h"
#include "keep8.cuh"
#include "tma.h"

namespace ceca {
namespace {

struct KeepArgs {
  dsgd_rows_t x;
  uint8_t *kept;
  int64_t t, d, rows, row_bytes;
  int32_t type;
};

// A warp takes a block of 32 channels at a time.
__global__ void __launch_bounds__(256) keep_kernel(const KeepArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t blocks = blocks8(p.d), stride = (int64_t)gridDim.x * 8;
  for (int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); b < p.rows * blocks; b += stride) {
    const int64_t row = b / blocks, k = b - row * blocks, c = k * kBlock8 + lane;
    const int64_t at = row / p.t * p.x.agent_stride + row % p.t * p.x.row_stride + c;
    float v = 0.f;
    if (c < p.d) v = p.type == DSGD_BF16 ? widen(static_cast<const bf16 *>(p.x.at)[at]) : static_cast<const float *>(p.x.at)[at];
    const uint32_t e = exponent8(__reduce_max_sync(0xffffffffu, magnitude(v)));
    uint8_t *to = p.kept + row * p.row_bytes;
    if (c < p.d) to[c] = (uint8_t)(int8_t)hold8(v, scale8(e));
    if (lane == 0) to[p.d + k] = (uint8_t)e;
    if (k == blocks - 1 && p.d + blocks + lane < p.row_bytes) to[p.d + blocks + lane] = 0;
  }
}

__global__ void __launch_bounds__(256) bring_kernel(const KeepArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t blocks = blocks8(p.d), stride = (int64_t)gridDim.x * 8;
  for (int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); b < p.rows * blocks; b += stride) {
    const int64_t row = b / blocks, k = b - row * blocks, c = k * kBlock8 + lane;
    if (c >= p.d) continue;
    const uint8_t *from = p.kept + row * p.row_bytes;
    const float v = (float)(int8_t)from[c] * step8(from[p.d + k]);
    const int64_t at = row / p.t * p.x.agent_stride + row % p.t * p.x.row_stride + c;
    if (p.type == DSGD_BF16) narrow(static_cast<bf16 *>(p.x.at) + at, v);
    else narrow(static_cast<float *>(p.x.at) + at, v);
  }
}

ceca_status_t keep8(dsgd_rows_t x, const void *kept, int32_t n, int64_t t, int64_t d, int32_t type, bool back, void *stream) {
  const int64_t most = ((int64_t)1 << 31) - 1024;
  if (n < 1 || n > 65535 || t < 0 || t >= most || d < 1 || d >= most || x.row_stride < d || x.agent_stride < 0 || (back && n > 1 && x.agent_stride < d) || !is_type(type))
    return CECA_ERR_INVALID_ARG;
  if (t == 0) return CECA_OK;
  if (!x.at || !kept) return CECA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(kept) & 15) return CECA_ERR_ALIGNMENT;
  KeepArgs p{x, static_cast<uint8_t *>(const_cast<void *>(kept)), t, d, n * t, kept_row_bytes(d), type};
  const int64_t work = p.rows * blocks8(d);
  const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(work, 8), (int64_t)sm_count() * 8);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (back) bring_kernel<<<grid, 256, 0, s>>>(p);
  else keep_kernel<<<grid, 256, 0, s>>>(p);
  return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

}  // namespace
}  // namespace ceca

extern "C" int64_t dsgd_kept_row_bytes(int64_t d) { return d < 1 ? 0 : ceca::kept_row_bytes(d); }

extern "C" ceca_status_t dsgd_keep8(dsgd_rows_t x, void *kept, int32_t n, int64_t t, int64_t d, int32_t type, void *stream) {
  return ceca::keep8(x, kept, n, t, d, type, false, stream);
}

extern "C" ceca_status_t dsgd_bring8(const void *kept, dsgd_rows_t x, int32_t n, int64_t t, int64_t d, int32_t type, void *stream) {
  return ceca::keep8(x, kept, n, t, d, type, true, stream);
}
