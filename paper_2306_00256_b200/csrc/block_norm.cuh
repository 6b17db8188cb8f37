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
  int64_t part_rows;            // (the form for wide rows; else a part takes every part_count-th row)
  int32_t stages, stage_bytes;  // of the ring in shared memory
  int32_t room[5];              // bytes of a row's place in a stage, by tensor
};

// Rows of up to kWidest channels are held in registers by a group of threads (a part of a warp, a warp, or a CTA), 8 or 16 channels each.  Of the same work, what a row costs besides
// (its sums, its addresses) is less with 16, as long as registers last: forward they do (8 x 4096 x 2048 bf16 125 us, 144 with 8 channels a thread), and
// the gradient has twice as much to hold (180 us with 8 channels, 216 with 16).  kWidest is what 512 threads hold.
constexpr int64_t kWidest = 8192;
struct Shape {
  int group, passes;   // threads of a group, eights of channels a thread
};
__host__ __device__ constexpr Shape shape_of(int64_t d) {
  return d <= 64 ? Shape{8, 1} : d <= 128 ? Shape{16, 1} : d <= 256 ? Shape{32, 1} : d <= 512 ? Shape{32, 2} : d <= 1024 ? Shape{64, 2} : d <= 2048 ? Shape{128, 2} : d <= 4096 ? Shape{256, 2} : Shape{512, 2};
}
__host__ __device__ constexpr Shape grad_shape_of(int64_t d) {
  return d <= 64 ? Shape{8, 1} : d <= 128 ? Shape{16, 1} : d <= 256 ? Shape{32, 1} : d <= 512 ? Shape{64, 1} : d <= 1024 ? Shape{128, 1} : d <= 2048 ? Shape{256, 1} : d <= 4096 ? Shape{512, 1} : Shape{512, 2};
}
// Groups of a CTA: rows that one warp, or a part of one, holds share one.
__host__ __device__ constexpr int groups_of(int group) { return group <= 32 ? 128 / group : 1; }
// CTAs an SM that the kernels are compiled for: 512 threads of 128 registers (forward, with 8 channels each, 768 of 80).
__host__ __device__ constexpr int resident_block(int group, int passes) { return (passes == 2 ? 512 : 768) / (group * groups_of(group)); }
__host__ __device__ constexpr int resident_grad(int group) { return 512 / (group * groups_of(group)); }
// Floats of the workspace that a part of the gradient's sums takes: those of both weights by channel, and the scale's, one of each group.
__host__ __device__ constexpr int64_t part_floats(int64_t d) { return 2 * d + groups_of(grad_shape_of(d).group); }
// Bytes of a group's weights that the gradient keeps in shared memory, for the registers' sake (8 x 4096 x 2047 bf16: 290 us, 367 with them in registers; fp32 stream
// of 2048 channels 260 and 277).  With 16 channels a thread there is no room for them beside the rows.
__host__ __device__ constexpr int aside_grad(int group, int passes) { return passes == 1 ? 64 * group : 0; }
// Whether a tensor's rows all start on 16-byte boundaries.
inline bool on_words(const dsgd_rows_t &x, int32_t type) {
  const int64_t n = 16 / type_bytes(type);
  return !x.at || ((reinterpret_cast<uintptr_t>(x.at) & 15) == 0 && x.agent_stride % n == 0 && x.row_stride % n == 0);
}
int64_t block_grad_parts(int64_t n, int64_t t, int64_t d);           // block_norm.cu: of the sums over rows, per agent
cudaError_t finish_block_grad(const BlockArgs &p, cudaStream_t s);   // block_norm.cu: joins them
// The kernels for rows in registers (block_rows.cuh), one translation unit for each pair of types of the stream and of the activations (mixed: fp32 and
// bf16), for rows that all start on 16-byte boundaries and for others.
cudaError_t block_rows_f32(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_rows_bf16(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_rows_mixed(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_odd_rows_f32(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_odd_rows_bf16(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_odd_rows_mixed(const BlockArgs &p, bool grad, cudaStream_t s);
cudaError_t block_odd_rows_any(const BlockArgs &p, bool grad, cudaStream_t s);   // any types

#ifdef __CUDACC__
__device__ __forceinline__ float load(const void *p, int32_t type, int64_t i) {
  return type == DSGD_BF16 ? widen(static_cast<const bf16 *>(p)[i]) : static_cast<const float *>(p)[i];
}
__device__ __forceinline__ void store(void *p, int32_t type, int64_t i, float v) {
  if (type == DSGD_BF16) narrow(static_cast<bf16 *>(p) + i, v);
  else narrow(static_cast<float *>(p) + i, v);
}
__device__ __forceinline__ int64_t place(const dsgd_rows_t &x, int64_t agent, int64_t row) { return agent * x.agent_stride + row * x.row_stride; }

// The gates' factors and their derivatives.  With e = exp(-a), 1 - sigmoid is e sigmoid: neither loses digits.  Below a = -87.3, where e would soon leave
// fp32, the sigmoid is held at 2^-126: its exponent is cut.  Silu's gate is cut itself, so that it is no larger where it is a factor (the type's lowest value
// would give -4, an infinity itself): silu and its derivative stay at -87.4 2^-126.  (Cut like that for both, rows read one by one are slower with
// sigmoids: 8 x 4096 x 2047 bf16 174 -> 181 us.)  A NaN goes through.
constexpr float kShut = -0x1.5d58ap+6f;   // -126 ln 2
struct Gates {
  Val<2> g, slope;
};
__device__ __forceinline__ float least(float x, float y) {   // a NaN if x is one
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float most(float x, float y) {   // a NaN if x is one
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ Gates gates_of(Val<2> a, bool silu) {
  if (silu) a = {most(a.x, kShut), most(a.y, kShut)};
  Val<2> t = mul(a, all<2>(-1.4426950408889634f));
  if (!silu) t = {least(t.x, 126.f), least(t.y, 126.f)};
  const Val<2> e = {ex2(t.x), ex2(t.y)}, b = add(e, all<2>(1.f));
  const Val<2> sig = {rcp(b.x), rcp(b.y)}, slope = mul(sig, mul(e, sig));
  if (silu) return {mul(a, sig), fma(a, slope, sig)};
  return {sig, slope};
}

// 1 / sqrt(sum / d + eps) of a sum of squares, and of one that overflowed and was taken again of the values times kLess (eps is nothing beside it).
constexpr float kLess = 0x1p-100f;
__device__ __forceinline__ float inverse_rms(float sum, float over_d, float eps) { return rsqrtf(fmaf(sum, over_d, eps)); }
__device__ __forceinline__ float inverse_rms_beyond(float sum, float over_d) { return kLess / sqrtf(sum * over_d); }
#endif

}  // namespace ceca
