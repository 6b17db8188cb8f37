// Gated linear recurrence over a sequence and its gradient.
//
//   a = sigmoid(f),  h_s = keep_s h_{s-1} + (1 - a_s) x_s          (keep = a, or 0 where a document begins)
//   l_s = dh_s + keep_{s+1} l_{s+1},  dx_s = (1 - a_s) l_s,  df_s = a_s (1 - a_s) l_s (p_s - x_s),  dh0 = keep_0 l_0
//
// with p_s the state before step s (0 where a document begins).  States are carried in fp32.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ceca.h"
#include "values.h"

namespace ceca {
namespace {

// Steps between two states that the forward call keeps for the gradient.
constexpr int kMarkSteps = 128;

struct RecurArgs {
  const void *x, *f, *dh;
  const float *h0, *dh_last;
  const uint8_t *starts;
  void *h, *dx, *df;
  float *h_last, *dh0;
  float *marks;
  int64_t b, t, d, n_marks;
  int64_t x_seq, x_step, f_seq, f_step, h_seq, h_step, dh_seq, dh_step, dx_seq, dx_step, df_seq, df_step;
};

// sigmoid(f) and sigmoid(-f), each to full relative accuracy: e = exp(-|f|) never overflows.
__device__ __forceinline__ void gates(float f, float *a, float *na) {
  const float e = __expf(-fabsf(f));
  const float r = __fdividef(1.f, 1.f + e);
  *a = f >= 0.f ? r : e * r;
  *na = f >= 0.f ? e * r : r;
}

template <typename T> __global__ void __launch_bounds__(128) recurrence_kernel(const RecurArgs p) {
  const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x, i = blockIdx.y;
  if (c >= p.d) return;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c;
  T *ho = static_cast<T *>(p.h) + i * p.h_seq + c;
  float h = p.h0 ? p.h0[i * p.d + c] : 0.f;
  for (int64_t s = 0; s < p.t; ++s) {
    if (p.marks && s % kMarkSteps == 0) p.marks[(i * p.n_marks + s / kMarkSteps) * p.d + c] = h;
    float a, na;
    gates(widen(f[s * p.f_step]), &a, &na);
    const float b = na * widen(x[s * p.x_step]);
    const bool fresh = p.starts && p.starts[i * p.t + s];
    h = fresh ? b : fmaf(a, h, b);
    narrow(ho + s * p.h_step, h);
  }
  if (p.h_last) p.h_last[i * p.d + c] = h;
}

template <typename T> __global__ void __launch_bounds__(128) recurrence_grad_kernel(const RecurArgs p) {
  const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x, i = blockIdx.y;
  if (c >= p.d) return;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c;
  const T *dh = static_cast<const T *>(p.dh) + i * p.dh_seq + c;
  T *dx = static_cast<T *>(p.dx) + i * p.dx_seq + c;
  T *df = static_cast<T *>(p.df) + i * p.df_seq + c;
  float carry = p.dh_last ? p.dh_last[i * p.d + c] : 0.f;   // keep_{s+1} l_{s+1}
  for (int64_t m = p.n_marks - 1; m >= 0; --m) {
    const int64_t s0 = m * kMarkSteps;
    const int len = (int)min((int64_t)kMarkSteps, p.t - s0);
    float before[kMarkSteps];
    float h = p.marks[(i * p.n_marks + m) * p.d + c];
    for (int j = 0; j < len; ++j) {
      float a, na;
      gates(widen(f[(s0 + j) * p.f_step]), &a, &na);
      const bool fresh = p.starts && p.starts[i * p.t + s0 + j];
      before[j] = fresh ? 0.f : h;
      const float b = na * widen(x[(s0 + j) * p.x_step]);
      h = fresh ? b : fmaf(a, h, b);
    }
    for (int j = len - 1; j >= 0; --j) {
      const int64_t s = s0 + j;
      float a, na;
      gates(widen(f[s * p.f_step]), &a, &na);
      const float xv = widen(x[s * p.x_step]);
      const float l = widen(dh[s * p.dh_step]) + carry;
      narrow(dx + s * p.dx_step, na * l);
      narrow(df + s * p.df_step, a * na * l * (before[j] - xv));
      carry = p.starts && p.starts[i * p.t + s] ? 0.f : a * l;
    }
  }
  if (p.dh0) p.dh0[i * p.d + c] = carry;
}

__global__ void __launch_bounds__(256) recurrence_empty_kernel(const float *from, float *to, int64_t count) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k < count) to[k] = from ? from[k] : 0.f;
}

ceca_status_t done() { return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA; }

// t = 0: the state goes through unchanged (in place it is there already).
ceca_status_t pass_through(const float *from, float *to, int64_t count, cudaStream_t s) {
  if (!to || to == from) return CECA_OK;
  recurrence_empty_kernel<<<(unsigned)ceil_div(count, 256), 256, 0, s>>>(from, to, count);
  return done();
}

bool sizes_ok(int64_t b, int64_t t, int64_t d, int32_t type) {
  return b >= 1 && b <= 65535 && d >= 1 && d < ((int64_t)1 << 31) && t >= 0 && t < ((int64_t)1 << 31) && is_type(type);
}

bool strides_ok(int64_t d, int64_t seq, int64_t step) { return seq >= 0 && step >= d; }

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" int64_t dsgd_recurrence_marks(int64_t t) { return t <= 0 ? 0 : ceil_div(t, kMarkSteps); }

extern "C" ceca_status_t dsgd_recurrence(const void *x, const void *f, const float *h0, const uint8_t *starts,
                                         void *h, float *h_last, float *marks, int64_t b, int64_t t, int64_t d,
                                         int64_t x_seq_stride, int64_t x_step_stride, int64_t f_seq_stride,
                                         int64_t f_step_stride, int64_t h_seq_stride, int64_t h_step_stride,
                                         int32_t type, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || !strides_ok(d, h_seq_stride, h_step_stride) ||
      (t > 0 && (!x || !f || !h || (b > 1 && h_seq_stride == 0))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(h0, h_last, b * d, s);
  RecurArgs p{};
  p.x = x; p.f = f; p.h0 = h0; p.starts = starts; p.h = h; p.h_last = h_last; p.marks = marks;
  p.b = b; p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.h_seq = h_seq_stride; p.h_step = h_step_stride;
  const dim3 grid((unsigned)ceil_div(d, 128), (unsigned)b);
  if (type == DSGD_F32) recurrence_kernel<float><<<grid, 128, 0, s>>>(p);
  else recurrence_kernel<bf16><<<grid, 128, 0, s>>>(p);
  return done();
}

extern "C" ceca_status_t dsgd_recurrence_grad(const void *x, const void *f, const void *dh, const float *marks,
                                              const uint8_t *starts, const float *dh_last, void *dx, void *df,
                                              float *dh0, int64_t b, int64_t t, int64_t d, int64_t x_seq_stride,
                                              int64_t x_step_stride, int64_t f_seq_stride, int64_t f_step_stride,
                                              int64_t dh_seq_stride, int64_t dh_step_stride, int64_t dx_seq_stride,
                                              int64_t dx_step_stride, int64_t df_seq_stride, int64_t df_step_stride,
                                              int32_t type, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || dh_seq_stride < 0 || dh_step_stride < 0 ||
      !strides_ok(d, dx_seq_stride, dx_step_stride) || !strides_ok(d, df_seq_stride, df_step_stride) ||
      (t > 0 && (!x || !f || !dh || !marks || !dx || !df || (b > 1 && (dx_seq_stride == 0 || df_seq_stride == 0)))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(dh_last, dh0, b * d, s);
  RecurArgs p{};
  p.x = x; p.f = f; p.dh = dh; p.marks = const_cast<float *>(marks); p.starts = starts; p.dh_last = dh_last;
  p.dx = dx; p.df = df; p.dh0 = dh0;
  p.b = b; p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.dh_seq = dh_seq_stride; p.dh_step = dh_step_stride; p.dx_seq = dx_seq_stride; p.dx_step = dx_step_stride;
  p.df_seq = df_seq_stride; p.df_step = df_step_stride;
  const dim3 grid((unsigned)ceil_div(d, 128), (unsigned)b);
  if (type == DSGD_F32) recurrence_grad_kernel<float><<<grid, 128, 0, s>>>(p);
  else recurrence_grad_kernel<bf16><<<grid, 128, 0, s>>>(p);
  return done();
}
