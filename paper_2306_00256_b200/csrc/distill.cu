// Distillation from a teacher's top logits: loss per row, and its gradient with respect to the student's logits.
//
//   q = softmax(z / T),  p_j = exp(t_j / T - N),  loss = w (sum_j p_j (log p_j - log q_j) [+ p0 log(p0 / q0)])
//   dz = (w / T) (q - p) at the top's entries, (w / T) (q [- p0 q / q0]) elsewhere
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ceca.h"
#include "values.h"

namespace ceca {
namespace {

constexpr int kMaxTop = 4096;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct DistillArgs {
  const void *z, *idx, *t;
  const float *teacher_lse, *weight;
  float *loss;
  void *dz;
  int64_t v, k, ldz, ldi, ldt, lddz;
  float scale;     // log2(e) / T
  float inv_temp;  // 1 / T
};

__device__ __forceinline__ float block_sum(float x, float *red) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
  for (int w = 0; w < kWarps; ++w) x += red[w];
  __syncthreads();
  return x;
}

__device__ __forceinline__ float block_max(float x, float *red) {
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
  for (int w = 1; w < kWarps; ++w) x = fmaxf(x, red[w]);
  __syncthreads();
  return x;
}

template <typename TZ, typename TT, typename TI>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillArgs p) {
  extern __shared__ uint32_t member[];   // one bit per vocabulary entry: listed by the teacher
  __shared__ float red[kWarps];
  __shared__ int32_t entry[kMaxTop];
  __shared__ float prob[kMaxTop];
  const int64_t row = blockIdx.x;
  const TZ *z = static_cast<const TZ *>(p.z) + row * p.ldz;
  TZ *dz = p.dz ? static_cast<TZ *>(p.dz) + row * p.lddz : nullptr;
  const TI *idx = static_cast<const TI *>(p.idx) + row * p.ldi;
  const TT *t = static_cast<const TT *>(p.t) + row * p.ldt;
  const float w = p.weight ? p.weight[row] : 1.f;
  const bool tail = p.teacher_lse != nullptr;
  const int words = (int)((p.v + 31) / 32);
  for (int c = threadIdx.x; c < words; c += kThreads) member[c] = 0;

  float top = -INFINITY;
  int some = 0;
  for (int j = threadIdx.x; j < p.k; j += kThreads) {
    const int64_t at = idx[j];
    const float tj = widen(t[j]) * p.scale;
    const bool there = at >= 0 && at < p.v && !(tj == -INFINITY);
    entry[j] = there ? (int32_t)at : -1;
    prob[j] = tj;
    some |= there;
    if (there) top = fmaxf(top, tj);
  }
  some = __syncthreads_or(some);
  if (w == 0.f || !some) {
    if (threadIdx.x == 0 && p.loss) p.loss[row] = 0.f;
    if (dz)
      for (int64_t c = threadIdx.x; c < p.v; c += kThreads) narrow(dz + c, 0.f);
    return;
  }
  // log2 of p_j
  float norm;
  if (tail) {
    norm = p.teacher_lse[row] * 1.4426950408889634f;
  } else {
    top = block_max(top, red);
    float s = 0.f;
    for (int j = threadIdx.x; j < p.k; j += kThreads)
      if (entry[j] >= 0) s += exp2f(prob[j] - top);
    norm = top + log2f(block_sum(s, red));
  }
  float mass = 0.f;
  for (int j = threadIdx.x; j < p.k; j += kThreads)
    if (entry[j] >= 0) {
      atomicOr(member + (entry[j] >> 5), 1u << (entry[j] & 31));
      mass += exp2f(prob[j] - norm);
    }
  const float rest = tail ? fmaxf(0.f, 1.f - block_sum(mass, red)) : 0.f;
  __syncthreads();

  float m = -INFINITY;
  for (int64_t c = threadIdx.x; c < p.v; c += kThreads) m = fmaxf(m, widen(z[c]));
  m = block_max(m, red) * p.scale;
  if (m == -INFINITY) m = 0.f;
  float all = 0.f, out = 0.f;
  for (int64_t c = threadIdx.x; c < p.v; c += kThreads) {
    const float e = exp2f(fmaf(widen(z[c]), p.scale, -m));
    all += e;
    if (!(member[c >> 5] >> (c & 31) & 1)) out += e;
  }
  all = block_sum(all, red);
  out = block_sum(out, red);
  float part = 0.f;
  for (int j = threadIdx.x; j < p.k; j += kThreads)
    if (entry[j] >= 0) {
      const float lp = prob[j] - norm, pj = exp2f(lp);
      const float y = widen(z[entry[j]]);
      const float lq = y == -INFINITY ? y : fmaf(y, p.scale, -m) - log2f(all);
      if (pj > 0.f) part += pj * (lp - lq);
    }
  part = block_sum(part, red);
  if (threadIdx.x == 0 && p.loss) {
    if (rest > 0.f) part += rest * log2f(rest / (out / all));
    p.loss[row] = w * part * 0.6931471805599453f;
  }
  if (!dz) return;
  const float scale = w * p.inv_temp;
  const float inside = all > 0.f ? scale / all : 0.f;
  const float outside = tail && out > 0.f ? inside - scale * rest / out : inside;
  for (int64_t c = threadIdx.x; c < p.v; c += kThreads) {
    const float e = exp2f(fmaf(widen(z[c]), p.scale, -m));
    float g = e * outside;
    if (member[c >> 5] >> (c & 31) & 1) {
      float pc = 0.f;
      for (int j = 0; j < p.k; ++j)
        if (entry[j] == c) pc += exp2f(prob[j] - norm);
      g = e * inside - scale * pc;
    }
    narrow(dz + c, g);
  }
}

template <typename TZ, typename TT, typename TI>
cudaError_t launch(const DistillArgs &p, int64_t r, cudaStream_t s) {
  const size_t bytes = (size_t)((p.v + 31) / 32) * 4;
  cudaFuncSetAttribute(distill_kernel<TZ, TT, TI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  distill_kernel<TZ, TT, TI><<<(unsigned)r, kThreads, bytes, s>>>(p);
  return cudaGetLastError();
}

template <typename TZ, typename TT> cudaError_t launch_i(const DistillArgs &p, int32_t it, int64_t r, cudaStream_t s) {
  return it == DSGD_I64 ? launch<TZ, TT, int64_t>(p, r, s) : launch<TZ, TT, int32_t>(p, r, s);
}

ceca_status_t distill(const void *z, const void *idx, const void *t, const float *teacher_lse, const float *weight,
                      float *loss, void *dz, int64_t r, int64_t v, int64_t k, int64_t ldz, int64_t ldi, int64_t ldt,
                      int64_t lddz, int32_t logits_type, int32_t index_type, int32_t teacher_type, float temperature,
                      void *stream) {
  if (r < 0 || r >= ((int64_t)1 << 31) || v < 1 || v >= ((int64_t)1 << 31) || k < 0 || k > kMaxTop || ldz < v ||
      ldi < k || ldt < k || lddz < v || !is_type(logits_type) || !is_index(index_type) || !is_type(teacher_type) ||
      !(temperature > 0.f) || !std::isfinite(temperature))
    return CECA_ERR_INVALID_ARG;
  if (r == 0) return CECA_OK;
  if (!z || (k > 0 && (!idx || !t))) return CECA_ERR_INVALID_ARG;
  if (dz == z && lddz != ldz) return CECA_ERR_UNSUPPORTED;
  DistillArgs p{};
  p.z = z; p.idx = idx; p.t = t; p.teacher_lse = teacher_lse; p.weight = weight; p.loss = loss; p.dz = dz;
  p.v = v; p.k = k; p.ldz = ldz; p.ldi = ldi; p.ldt = ldt; p.lddz = lddz;
  p.scale = (float)(1.4426950408889634 / (double)temperature);
  p.inv_temp = (float)(1.0 / (double)temperature);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (logits_type == DSGD_F32)
    e = teacher_type == DSGD_F32 ? launch_i<float, float>(p, index_type, r, s) : launch_i<float, bf16>(p, index_type, r, s);
  else
    e = teacher_type == DSGD_F32 ? launch_i<bf16, float>(p, index_type, r, s) : launch_i<bf16, bf16>(p, index_type, r, s);
  return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

}  // namespace
}  // namespace ceca

extern "C" ceca_status_t dsgd_distill_loss(const void *z, const void *idx, const void *t, const float *teacher_lse,
                                           const float *weight, float *loss, int64_t r, int64_t v, int64_t k,
                                           int64_t ldz, int64_t ldi, int64_t ldt, int32_t logits_type,
                                           int32_t index_type, int32_t teacher_type, float temperature, void *stream) {
  if (r > 0 && !loss) return CECA_ERR_INVALID_ARG;
  return ceca::distill(z, idx, t, teacher_lse, weight, loss, nullptr, r, v, k, ldz, ldi, ldt, v, logits_type,
                       index_type, teacher_type, temperature, stream);
}

extern "C" ceca_status_t dsgd_distill_grad(const void *z, const void *idx, const void *t, const float *teacher_lse,
                                           const float *weight, float *loss, void *dz, int64_t r, int64_t v,
                                           int64_t k, int64_t ldz, int64_t ldi, int64_t ldt, int64_t lddz,
                                           int32_t logits_type, int32_t index_type, int32_t teacher_type,
                                           float temperature, void *stream) {
  if (r > 0 && !dz) return CECA_ERR_INVALID_ARG;
  return ceca::distill(z, idx, t, teacher_lse, weight, loss, dz, r, v, k, ldz, ldi, ldt, lddz, logits_type,
                       index_type, teacher_type, temperature, stream);
}
