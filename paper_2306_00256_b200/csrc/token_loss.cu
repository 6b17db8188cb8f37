// Log-probabilities of tokens, and the policy and preference losses that are made of them, with their gradients.
//
//   l = log softmax(z / T)[token],  dz = (c / T) (one-hot - q),  c the derivative of the loss by l
//
// A row is summed without its token: with R = sum of 2^(z c - k) over the others and y the token's exponent in that frame, 1 - q = R / (R + 2^y)
// and l = -log(1 + R / 2^y) keep their digits where the model is sure, and the others' share of the gradient is (c / T) (1 - q) / R each.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "ceca.h"
#include "logits.cuh"
#include "tma.h"

namespace ceca {
namespace {

enum Loss : int32_t { kLogprob, kPolicy, kPreference };

// What the gradient needs of a row: the others' exponentials are 2^(z c - k) (of a far row 2^((z - k) c)), their entries -factor times that, the
// token's `own`.
struct alignas(16) RowOut {
  float k, factor, own;
  int32_t far;
};

struct TokenArgs {
  const void *z, *tokens, *bounds;
  const float *old_logp, *advantage, *ref_logp, *weight;
  float *loss, *logp;
  void *dz;
  int64_t r, v, ldz, lddz, pairs;
  float scale, temperature, low, high, kl, beta, smoothing;   // scale = log2(e) / T
  int32_t idx64, bounds64, average, what;
  RowOut *rows;        // workspace
  float *row_logp;     // preference
  double *slopes;      // of each sequence
};

__device__ __forceinline__ int64_t index_of(const void *p, int32_t wide, int64_t i) {
  return wide ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

// A row's sums: of the others R in frame k (or M), and the token's exponent y there.
struct RowSum {
  float k, rest, y;
  bool far;
};
struct Odds {
  float logp, other;   // log q, 1 - q of the token
};
__device__ __forceinline__ Odds odds_of(const RowSum &s) {
  if (s.rest == 0.f) return s.y == -INFINITY ? Odds{-INFINITY, 1.f} : Odds{s.y == s.y ? 0.f : s.y, s.y == s.y ? 0.f : s.y};
  const float a = s.y - log2f(s.rest);   // log2 of the token's odds against the others
  if (a > 0.f) {
    const float e = exp2f(-a);
    return {-log1pf(e), e / (1.f + e)};
  }
  const float e = exp2f(a);
  return {kLn2 * a - log1pf(e), 1.f / (1.f + e)};
}

// The loss of a row and its derivative by the token's log-probability, both times the weight.
__device__ __forceinline__ float2 policy(const TokenArgs &p, int64_t i, float w, float l) {
  const float adv = p.advantage[i], ratio = expf(l - p.old_logp[i]);
  const float plain = ratio * adv, clipped = fminf(fmaxf(ratio, p.low), p.high) * adv;
  const bool free = !(plain > clipped);   // (a NaN goes on)
  float loss = -(free ? plain : clipped), slope = free ? -plain : 0.f;
  if (p.ref_logp && p.kl != 0.f) {
    const float x = p.ref_logp[i] - l, e = expm1f(x);
    loss += p.kl * (e - x);
    slope -= p.kl * e;
  }
  return make_float2(w * loss, w * slope);
}
__device__ __forceinline__ RowOut row_out(const TokenArgs &p, const RowSum &s, const Odds &o, float slope) {
  const float by = slope / p.temperature, own = by * o.other;
  return {s.k, s.rest == 0.f ? 0.f : own / s.rest, own, s.far ? 1 : 0};
}

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ float cta_max(float x, float *part) {
  x = warp_max(x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  x = part[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) x = fmaxf(x, part[i]);
  return x;
}
__device__ __forceinline__ float cta_sum(float x, float *part) {
  x = warp_sum(x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) x += part[i];
  return x;
}

// A CTA reads a row twice: its maximum, its sum.
template <typename TZ> __global__ void __launch_bounds__(kThreads) sum_kernel(const TokenArgs p) {
  __shared__ float part[kWarps];
  for (int64_t i = blockIdx.x; i < p.r; i += gridDim.x) {
    const int64_t tok = index_of(p.tokens, p.idx64, i);
    const float w = p.what == kPolicy && p.weight ? p.weight[i] : 1.f;
    const bool live = tok >= 0 && tok < p.v && w != 0.f;
    if (!live) {
      if (threadIdx.x == 0) {
        if (p.what == kLogprob || (p.what == kPolicy && p.logp)) p.logp[i] = 0.f;
        if (p.what == kPolicy) p.loss[i] = 0.f;
        if (p.what == kPreference) p.row_logp[i] = 0.f;
        if (p.rows) p.rows[i] = {0.f, 0.f, 0.f, 0};
      }
      continue;
    }
    const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
    float m = -INFINITY;
    for (int64_t c = threadIdx.x; c < p.v; c += kThreads)
      if (c != tok) m = fmaxf(m, widen(z[c]));
    m = cta_max(m, part);
    RowSum s;
    s.far = !(fabsf(frame_of(m, p.scale)) < kFar);
    s.k = s.far ? m == -INFINITY ? widen(z[tok]) : m : frame_of(m, p.scale);
    const auto exponent = [&](float x) { return s.far ? (x - s.k) * p.scale : fmaf(x, p.scale, -s.k); };
    float sum = 0.f;
    for (int64_t c = threadIdx.x; c < p.v; c += kThreads)
      if (c != tok) sum += m == -INFINITY ? (widen(z[c]) == -INFINITY ? 0.f : NAN) : ex2(exponent(widen(z[c])));
    s.rest = cta_sum(sum, part);
    const float own = widen(z[tok]);
    s.y = own == -INFINITY ? own : own == INFINITY ? NAN : exponent(own);
    if (threadIdx.x) continue;
    const Odds o = odds_of(s);
    if (p.what == kLogprob) p.logp[i] = o.logp;
    if (p.what == kPolicy) {
      const float2 l = policy(p, i, w, o.logp);
      p.loss[i] = l.x;
      if (p.logp) p.logp[i] = o.logp;
      if (p.rows) p.rows[i] = row_out(p, s, o, l.y);
    }
    if (p.what == kPreference) {
      p.row_logp[i] = o.logp;
      if (p.rows) p.rows[i] = row_out(p, s, o, 1.f);   // the sequence's slope comes later
    }
  }
}

__device__ __forceinline__ int64_t bound(const TokenArgs &p, int64_t j) { return min(max(index_of(p.bounds, p.bounds64, j), (int64_t)0), p.r); }

// A CTA takes a pair: its sequences' sums in 64 bits, the loss, and each one's slope.
__global__ void __launch_bounds__(kThreads) pair_kernel(const TokenArgs p) {
  __shared__ double sums[2][kWarps];
  __shared__ int64_t counts[2][kWarps];
  const int warp = threadIdx.x >> 5;
  for (int64_t q = blockIdx.x; q < p.pairs; q += gridDim.x) {
    const float w = p.weight ? p.weight[q] : 1.f;
    __syncthreads();
    for (int k = 0; k < 2; ++k) {
      double s = 0.;
      int64_t n = 0;
      for (int64_t i = bound(p, 2 * q + k) + threadIdx.x; i < bound(p, 2 * q + k + 1); i += kThreads) {
        const int64_t tok = index_of(p.tokens, p.idx64, i);
        s += (double)p.row_logp[i];
        n += tok >= 0 && tok < p.v;
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        n += __shfl_xor_sync(0xffffffffu, n, o);
      }
      if ((threadIdx.x & 31) == 0) {
        sums[k][warp] = s;
        counts[k][warp] = n;
      }
    }
    __syncthreads();
    if (threadIdx.x) continue;
    double l[2], by[2];
    for (int k = 0; k < 2; ++k) {
      int64_t n = 0;
      l[k] = 0.;
      for (int i = 0; i < kWarps; ++i) {
        l[k] += sums[k][i];
        n += counts[k][i];
      }
      by[k] = p.average ? 1. / (double)max(n, (int64_t)1) : 1.;
      l[k] *= by[k];
      if (p.logp) p.logp[2 * q + k] = (float)l[k];
      if (p.ref_logp) l[k] -= (double)p.ref_logp[2 * q + k];
    }
    const double m = (double)p.beta * (l[0] - l[1]), e = exp(-fabs(m)), small = e / (1. + e);
    const double up = log1p(e) + fmax(-m, 0.), down = log1p(e) + fmax(m, 0.);   // -log sigmoid(m), -log sigmoid(-m)
    const double at_minus = m >= 0. ? small : 1. - small, at = m >= 0. ? 1. - small : small;   // sigmoid(-m), sigmoid(m)
    const double eps = (double)p.smoothing;
    if (p.loss) p.loss[q] = w == 0.f ? 0.f : (float)((double)w * ((1. - eps) * up + (eps > 0. ? eps * down : 0.)));
    if (p.slopes) {
      const double slope = w == 0.f ? 0. : (double)w * (double)p.beta * (eps * at - (1. - eps) * at_minus);
      p.slopes[2 * q] = slope * by[0];
      p.slopes[2 * q + 1] = -slope * by[1];
    }
  }
}

// The sequence that a row lies in, or -1.
__device__ __forceinline__ int64_t sequence_of(const TokenArgs &p, int64_t i) {
  if (p.pairs == 0) return -1;
  int64_t lo = 0, hi = 2 * p.pairs + 1;   // the first bound above i
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (index_of(p.bounds, p.bounds64, mid) > i) hi = mid;
    else lo = mid + 1;
  }
  return lo == 2 * p.pairs + 1 ? -1 : lo - 1;
}

template <typename TZ> __global__ void __launch_bounds__(kThreads) turn_kernel(const TokenArgs p) {
  for (int64_t i = blockIdx.x; i < p.r; i += gridDim.x) {
    RowOut o = p.rows[i];
    if (p.what == kPreference) {
      const int64_t j = sequence_of(p, i);
      const float slope = j < 0 ? 0.f : (float)p.slopes[j];
      o.factor = slope == 0.f ? 0.f : o.factor * slope;
      o.own = slope == 0.f ? 0.f : o.own * slope;
    }
    const int64_t tok = index_of(p.tokens, p.idx64, i);
    const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
    TZ *dz = static_cast<TZ *>(p.dz) + i * p.lddz;
    for (int64_t c = threadIdx.x; c < p.v; c += kThreads) {
      float g = 0.f;
      if (c == tok) g = o.own;
      else if (o.factor != 0.f) {
        const float x = widen(z[c]);
        g = -o.factor * ex2(o.far ? (x - o.k) * p.scale : fmaf(x, p.scale, -o.k));
      }
      narrow(dz + c, g);
    }
  }
}

constexpr int64_t kMost = ((int64_t)1 << 31) - 1024;
bool sizes_ok(int64_t r, int64_t v) { return r >= 0 && r < ((int64_t)1 << 28) && v >= 1 && v < kMost; }

bool common_ok(int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t logits_type, int32_t index_type, float temperature) {
  return sizes_ok(r, v) && ldz >= v && lddz >= v && is_type(logits_type) && is_index(index_type) && temperature > 0.f && std::isfinite(temperature);
}

TokenArgs common(const void *z, const void *tokens, void *dz, int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t index_type, float temperature,
                 void *workspace) {
  TokenArgs p{};
  p.z = z; p.tokens = tokens; p.dz = dz;
  p.r = r; p.v = v; p.ldz = ldz; p.lddz = lddz;
  p.scale = (float)(1.4426950408889634 / (double)temperature);
  p.temperature = temperature;
  p.idx64 = index_type == DSGD_I64;
  p.rows = dz ? static_cast<RowOut *>(workspace) : nullptr;
  p.slopes = reinterpret_cast<double *>(static_cast<RowOut *>(workspace) + r);
  return p;
}

bool workspace_ok(const void *workspace, size_t bytes, int64_t r, int64_t v, int64_t pairs) {
  return workspace && bytes >= dsgd_token_workspace_bytes(r, v, pairs) && !(reinterpret_cast<uintptr_t>(workspace) & 15);
}

ceca_status_t run(const TokenArgs &p, int32_t logits_type, cudaStream_t s) {
  const bool wide = logits_type == DSGD_F32;
  const unsigned grid = (unsigned)std::min<int64_t>(p.r, (int64_t)sm_count() * 8);
  if (p.r > 0) {
    if (wide) sum_kernel<float><<<grid, kThreads, 0, s>>>(p);
    else sum_kernel<bf16><<<grid, kThreads, 0, s>>>(p);
  }
  if (p.what == kPreference && p.pairs > 0) pair_kernel<<<(unsigned)std::min<int64_t>(p.pairs, 1024), kThreads, 0, s>>>(p);
  if (p.dz && p.r > 0) {
    if (wide) turn_kernel<float><<<grid, kThreads, 0, s>>>(p);
    else turn_kernel<bf16><<<grid, kThreads, 0, s>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

ceca_status_t policy_call(const void *z, const void *tokens, const float *old_logp, const float *advantage, const float *ref_logp, const float *weight,
                          float *loss, float *logp, void *dz, int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t logits_type,
                          int32_t index_type, float temperature, float clip_low, float clip_high, float kl, void *workspace, size_t workspace_bytes,
                          void *stream) {
  if (!common_ok(r, v, ldz, lddz, logits_type, index_type, temperature) || !(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) ||
      !std::isfinite(clip_high) || !(kl >= 0.f) || !std::isfinite(kl))
    return CECA_ERR_INVALID_ARG;
  if (r == 0) return CECA_OK;
  if (!z || !tokens || !old_logp || !advantage || !loss) return CECA_ERR_INVALID_ARG;
  if (dz == z && lddz != ldz) return CECA_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, r, v, 0)) return CECA_ERR_WORKSPACE;
  TokenArgs p = common(z, tokens, dz, r, v, ldz, lddz, index_type, temperature, workspace);
  p.what = kPolicy;
  p.old_logp = old_logp; p.advantage = advantage; p.ref_logp = ref_logp; p.weight = weight; p.loss = loss; p.logp = logp;
  p.low = 1.f - clip_low; p.high = 1.f + clip_high; p.kl = kl;
  return run(p, logits_type, static_cast<cudaStream_t>(stream));
}

ceca_status_t preference_call(const void *z, const void *tokens, const void *bounds, const float *ref_logp, const float *weight, float *loss,
                              float *logp, void *dz, int64_t pairs, int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t logits_type,
                              int32_t index_type, int32_t bounds_type, float temperature, float beta, float smoothing, int32_t average,
                              void *workspace, size_t workspace_bytes, void *stream) {
  if (!common_ok(r, v, ldz, lddz, logits_type, index_type, temperature) || !is_index(bounds_type) || pairs < 0 || pairs >= ((int64_t)1 << 27) ||
      !std::isfinite(beta) || !(smoothing >= 0.f && smoothing <= 1.f))
    return CECA_ERR_INVALID_ARG;
  if ((r > 0 && (!z || !tokens)) || (pairs > 0 && (!bounds || !loss))) return CECA_ERR_INVALID_ARG;
  if (r == 0 && pairs == 0) return CECA_OK;
  if (dz == z && dz && lddz != ldz) return CECA_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, r, v, pairs)) return CECA_ERR_WORKSPACE;
  TokenArgs p = common(z, tokens, dz, r, v, ldz, lddz, index_type, temperature, workspace);
  p.what = kPreference;
  p.row_logp = reinterpret_cast<float *>(p.slopes + 2 * pairs);
  p.bounds = bounds; p.bounds64 = bounds_type == DSGD_I64;
  p.ref_logp = ref_logp; p.weight = weight; p.loss = loss; p.logp = logp; p.pairs = pairs;
  p.beta = beta; p.smoothing = smoothing; p.average = average != 0;
  return run(p, logits_type, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" size_t dsgd_token_workspace_bytes(int64_t r, int64_t v, int64_t pairs) {
  if (!sizes_ok(r, v) || pairs < 0 || pairs >= ((int64_t)1 << 27)) return 0;
  return (sizeof(RowOut) + sizeof(float)) * (size_t)r + 2 * sizeof(double) * (size_t)pairs;
}

extern "C" ceca_status_t dsgd_token_logprob(const void *z, const void *tokens, float *logp, int64_t r, int64_t v, int64_t ldz, int32_t logits_type,
                                            int32_t index_type, float temperature, void *workspace, size_t workspace_bytes, void *stream) {
  if (!common_ok(r, v, ldz, v, logits_type, index_type, temperature)) return CECA_ERR_INVALID_ARG;
  if (r == 0) return CECA_OK;
  if (!z || !tokens || !logp) return CECA_ERR_INVALID_ARG;
  if (!workspace_ok(workspace, workspace_bytes, r, v, 0)) return CECA_ERR_WORKSPACE;
  TokenArgs p = common(z, tokens, nullptr, r, v, ldz, v, index_type, temperature, workspace);
  p.what = kLogprob;
  p.logp = logp;
  return run(p, logits_type, static_cast<cudaStream_t>(stream));
}

extern "C" ceca_status_t dsgd_policy_loss(const void *z, const void *tokens, const float *old_logp, const float *advantage, const float *ref_logp,
                                          const float *weight, float *loss, float *logp, int64_t r, int64_t v, int64_t ldz, int32_t logits_type,
                                          int32_t index_type, float temperature, float clip_low, float clip_high, float kl, void *workspace,
                                          size_t workspace_bytes, void *stream) {
  return policy_call(z, tokens, old_logp, advantage, ref_logp, weight, loss, logp, nullptr, r, v, ldz, v, logits_type, index_type, temperature,
                     clip_low, clip_high, kl, workspace, workspace_bytes, stream);
}

extern "C" ceca_status_t dsgd_policy_grad(const void *z, const void *tokens, const float *old_logp, const float *advantage, const float *ref_logp,
                                          const float *weight, float *loss, float *logp, void *dz, int64_t r, int64_t v, int64_t ldz,
                                          int64_t lddz, int32_t logits_type, int32_t index_type, float temperature, float clip_low, float clip_high,
                                          float kl, void *workspace, size_t workspace_bytes, void *stream) {
  if (r > 0 && !dz) return CECA_ERR_INVALID_ARG;
  return policy_call(z, tokens, old_logp, advantage, ref_logp, weight, loss, logp, dz, r, v, ldz, lddz, logits_type, index_type, temperature,
                     clip_low, clip_high, kl, workspace, workspace_bytes, stream);
}

extern "C" ceca_status_t dsgd_preference_loss(const void *z, const void *tokens, const void *bounds, const float *ref_logp, const float *weight,
                                              float *loss, float *logp, int64_t pairs, int64_t r, int64_t v, int64_t ldz, int32_t logits_type,
                                              int32_t index_type, int32_t bounds_type, float temperature, float beta, float smoothing,
                                              int32_t average, void *workspace, size_t workspace_bytes, void *stream) {
  return preference_call(z, tokens, bounds, ref_logp, weight, loss, logp, nullptr, pairs, r, v, ldz, v, logits_type, index_type, bounds_type,
                         temperature, beta, smoothing, average, workspace, workspace_bytes, stream);
}

extern "C" ceca_status_t dsgd_preference_grad(const void *z, const void *tokens, const void *bounds, const float *ref_logp, const float *weight,
                                              float *loss, float *logp, void *dz, int64_t pairs, int64_t r, int64_t v, int64_t ldz, int64_t lddz,
                                              int32_t logits_type, int32_t index_type, int32_t bounds_type, float temperature, float beta,
                                              float smoothing, int32_t average, void *workspace, size_t workspace_bytes, void *stream) {
  if (r > 0 && !dz) return CECA_ERR_INVALID_ARG;
  return preference_call(z, tokens, bounds, ref_logp, weight, loss, logp, dz, pairs, r, v, ldz, lddz, logits_type, index_type, bounds_type,
                         temperature, beta, smoothing, average, workspace, workspace_bytes, stream);
}
