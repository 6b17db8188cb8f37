// Distillation from a teacher's top logits: loss per row, and its gradient with respect to the student's logits.
//
//   q = softmax(z / T),  p_j = exp(t_j / T - N),  loss = w (sum_j p_j (log p_j - log q_j) [+ p0 log(p0 / q0)])
//   dz = (w / T) (q - p) at the top's entries, (w / T) (q [- p0 q / q0]) elsewhere
//
// One CTA takes a row (a cluster of them where there are few rows) in two passes over it.  The first keeps a running
// maximum and a running sum of exponentials per thread, over the entries outside the top: q0 must not come from a
// difference of sums that may be nearly equal.  A bitmap in shared memory says which entries are in the top; the few of
// them are gathered and summed apart.  The second pass writes w / T (1 / S [- p0 / S0]) exp(z / T - M) everywhere and
// the top's entries are then written over.  The second read of a row comes from L2: all rows in work together fill less
// than half of it.  Exponents are (z - M) log2(e) / T, the difference first: the sums stay right for logits of any size,
// masks of the type's lowest value among them.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "ceca.h"
#include "tma.h"
#include "values.h"

namespace ceca {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxTop = 4096;
constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int64_t kMaxBits = 1 << 20;   // of the bitmap; longer rows wrap around in it
constexpr int kDeep = 4;                // vectors a thread loads before it uses the first

struct DistillArgs {
  const void *z, *idx, *t;
  const float *teacher_lse, *weight;
  float *loss;
  void *dz;
  int64_t v, k, ldz, ldi, ldt, lddz;
  float scale;        // log2(e) / T
  float temperature;
  int32_t cluster;    // CTAs per row
  int32_t words;      // of the bitmap
};

// 16 bytes of logits.
template <typename T> struct Vec {
  static constexpr int N = 16 / sizeof(T), P = N / 2;
  uint4 w;
};
__device__ __forceinline__ uint32_t &word(uint4 &v, int i) { return (&v.x)[i]; }
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return (&v.x)[i]; }
__device__ __forceinline__ Val<2> pair(const Vec<float> &v, int i) { return {__uint_as_float(word(v.w, 2 * i)), __uint_as_float(word(v.w, 2 * i + 1))}; }
__device__ __forceinline__ Val<2> pair(const Vec<bf16> &v, int i) {   // a bf16 is the upper half of the fp32 of the same value
  const uint32_t x = word(v.w, i);
  return {__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)};
}
__device__ __forceinline__ void set_pair(Vec<float> &v, int i, Val<2> a) {
  word(v.w, 2 * i) = __float_as_uint(a.x);
  word(v.w, 2 * i + 1) = __float_as_uint(a.y);
}
__device__ __forceinline__ void set_pair(Vec<bf16> &v, int i, Val<2> a) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a.x, a.y);
  word(v.w, i) = *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> __device__ __forceinline__ Vec<T> all_least() {   // -infinity throughout
  const uint32_t x = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return {make_uint4(x, x, x, x)};
}
// The elements whose bit is set in `mask` become -infinity.
template <typename T> __device__ __forceinline__ void strike(Vec<T> &v, uint32_t mask) {
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e)
    if (mask >> e & 1) {
      if (sizeof(T) == 4) word(v.w, e) = 0xff800000u;
      else word(v.w, e / 2) = e % 2 ? (word(v.w, e / 2) & 0xffffu) | 0xff800000u : (word(v.w, e / 2) & 0xffff0000u) | 0xff80u;
    }
}
__device__ __forceinline__ float top_of(const Vec<float> &v) {
  return fmaxf(fmaxf(__uint_as_float(v.w.x), __uint_as_float(v.w.y)), fmaxf(__uint_as_float(v.w.z), __uint_as_float(v.w.w)));
}
__device__ __forceinline__ float top_of(const Vec<bf16> &v) {
  const auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
  const __nv_bfloat162 m = __hmax2(__hmax2(h(v.w.x), h(v.w.y)), __hmax2(h(v.w.z), h(v.w.w)));
  return fmaxf(__low2float(m), __high2float(m));
}

// A row as whole vectors on 16-byte boundaries: vector 0 begins `pad` elements before the row, and the last may end after
// it.  Slot s is element s - pad.
template <typename T> struct Row {
  const T *at0;   // where vector 0 begins
  int pad;
  int64_t slots, vectors;
  __device__ __forceinline__ Row(const T *row, int64_t v) {
    pad = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    at0 = row - pad;
    slots = v + pad;
    vectors = (slots + Vec<T>::N - 1) / Vec<T>::N;
  }
  __device__ __forceinline__ bool whole(int64_t j) const { return (j > 0 || pad == 0) && (j + 1) * Vec<T>::N <= slots; }
  // vector j, with -infinity for what is not of the row
  __device__ __forceinline__ Vec<T> load(int64_t j, bool last_use) const {
    Vec<T> v = all_least<T>();
    if (whole(j)) {
      const uint4 *p = reinterpret_cast<const uint4 *>(at0) + j;
      v.w = last_use ? __ldcs(p) : *p;
    } else if (j < vectors) {
      T *e = reinterpret_cast<T *>(&v.w);
      for (int i = 0; i < Vec<T>::N; ++i) {
        const int64_t s = j * Vec<T>::N + i;
        if (s >= pad && s < slots) e[i] = at0[s];
      }
    }
    return v;
  }
};

// Sums or maxima over the CTA of up to N values at once, each in one fixed order.
template <int N, bool MAX> __device__ __forceinline__ void over_block(float *x, float *red) {
  const int warps = blockDim.x >> 5;
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float y = __shfl_xor_sync(0xffffffffu, x[i], o);
      x[i] = MAX ? fmaxf(x[i], y) : x[i] + y;
    }
    if ((threadIdx.x & 31) == 0) red[i * kMaxWarps + (threadIdx.x >> 5)] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = red[i * kMaxWarps];
    for (int w = 1; w < warps; ++w) x[i] = MAX ? fmaxf(x[i], red[i * kMaxWarps + w]) : x[i] + red[i * kMaxWarps + w];
  }
}

// Shared memory behind the bitmap: k entries of each.
struct Entries {
  int32_t *at;    // the vocabulary entry, or -1
  float *t, *z;   // the teacher's logit / T, the student's logit
};

template <typename TZ, typename TT, typename TI, bool CLUSTER>
__global__ void __launch_bounds__(kMaxThreads, 2) distill_kernel(const DistillArgs p) {
  constexpr int N = Vec<TZ>::N, P = Vec<TZ>::P;
  extern __shared__ uint32_t bitmap[];
  __shared__ float red[4][4 * kMaxWarps];
  __shared__ float share[2];
  Entries en;
  en.at = reinterpret_cast<int32_t *>(bitmap + p.words);
  en.t = reinterpret_cast<float *>(en.at + p.k);
  en.z = en.t + p.k;
  const int ranks = CLUSTER ? p.cluster : 1;
  const int64_t row = CLUSTER ? blockIdx.x / ranks : blockIdx.x;
  const int rank = CLUSTER ? (int)(blockIdx.x - row * ranks) : 0;
  const TZ *z = static_cast<const TZ *>(p.z) + row * p.ldz;
  TZ *dz = p.dz ? static_cast<TZ *>(p.dz) + row * p.lddz : nullptr;
  const TI *idx = static_cast<const TI *>(p.idx) + row * p.ldi;
  const TT *t = static_cast<const TT *>(p.t) + row * p.ldt;
  const float w = p.weight ? p.weight[row] : 1.f;
  const bool tail = p.teacher_lse != nullptr;
  const Row<TZ> rz(z, p.v);
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
  // this CTA's vectors and slots
  const int64_t per = (rz.vectors + ranks - 1) / ranks;
  const int64_t v0 = rank * per, v1 = min(rz.vectors, v0 + per);
  const int64_t slot0 = v0 * N, slot1 = v1 * N;
  const bool wraps = slot1 - slot0 > kMaxBits;   // then a set bit only says that an entry may be there

  for (int c = threadIdx.x; c < p.words; c += blockDim.x) bitmap[c] = 0;
  __syncthreads();
  // the top: its entries, which of them are there, the bitmap
  int some = 0, twice = 0;
  float x[4] = {-INFINITY, -INFINITY, 0.f, 0.f};   // maxima of z and of t over the top
  for (int j = threadIdx.x; j < p.k; j += blockDim.x) {
    const int64_t at = idx[j];
    const float tj = widen(t[j]) / p.temperature;
    const bool there = w != 0.f && at >= 0 && at < p.v && !(tj == -INFINITY);
    en.at[j] = there ? (int32_t)at : -1;
    en.t[j] = tj;
    if (!there) continue;
    some = 1;
    const float zj = widen(z[at]);
    en.z[j] = zj;
    x[0] = fmaxf(x[0], zj);
    x[1] = fmaxf(x[1], tj);
    const int64_t slot = at + rz.pad;
    if (slot >= slot0 && slot < slot1) {
      const uint32_t b = (uint32_t)((slot - slot0) & (kMaxBits - 1));
      twice |= atomicOr(bitmap + (b >> 5), 1u << (b & 31)) >> (b & 31) & 1;
    }
  }
  some = __syncthreads_or(some);
  if (!some) {   // nothing to learn here, and nothing read
    if (threadIdx.x == 0 && rank == 0 && p.loss) p.loss[row] = 0.f;
    if (dz) {
      for (int64_t j = v0 + threadIdx.x; j < v1; j += blockDim.x) {
        if (together && rz.whole(j)) __stcs(reinterpret_cast<uint4 *>(dz - rz.pad) + j, make_uint4(0, 0, 0, 0));
        else
          for (int i = 0; i < N; ++i) {
            const int64_t s = j * N + i;
            if (s >= rz.pad && s < rz.slots) narrow(dz + s - rz.pad, 0.f);
          }
      }
    }
    return;
  }
  twice = __syncthreads_or(twice);

  // which of vector j's elements are in the top
  const auto in_top = [&](int64_t j) -> uint32_t {
    const uint32_t b = (uint32_t)((j * N - slot0) & (kMaxBits - 1));
    uint32_t m = bitmap[b >> 5] >> (b & 31) & ((1u << N) - 1);
    if (m && wraps) {
      uint32_t sure = 0;
      for (int e = 0; e < p.k; ++e) {
        const int64_t s = (int64_t)en.at[e] + rz.pad - j * N;
        if (en.at[e] >= 0 && s >= 0 && s < N) sure |= 1u << s;
      }
      m = sure;
    }
    return m;
  };

  // pass 1: maximum and sum over the entries outside the top
  float m = -INFINITY;
  Val<2> sum{0.f, 0.f};
  for (int64_t base = v0; base < v1; base += (int64_t)kDeep * blockDim.x) {
    Vec<TZ> a[kDeep];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int64_t j = base + (int64_t)u * blockDim.x + threadIdx.x;
      a[u] = j < v1 ? rz.load(j, !dz) : all_least<TZ>();
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int64_t j = base + (int64_t)u * blockDim.x + threadIdx.x;
      const uint32_t mask = j < v1 ? in_top(j) : 0;
      if (mask) strike(a[u], mask);
      top = fmaxf(top, top_of(a[u]));
    }
    if (top > m) {
      sum = mul(sum, all<2>(ex2((m - top) * p.scale)));
      m = top;
    }
    const Val<2> from = all<2>(m == -INFINITY ? 0.f : m), by = all<2>(p.scale);
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        Val<2> y = mul(sub(pair(a[u], i), from), by);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        sum = add(sum, y);
      }
  }
  cg::cluster_group cl = cg::this_cluster();
  x[0] = fmaxf(x[0], m);
  over_block<2, true>(x, red[0]);
  if (CLUSTER) {
    if (threadIdx.x == 0) share[0] = x[0];
    cl.sync();
    for (int r = 0; r < ranks; ++r) x[0] = fmaxf(x[0], *cl.map_shared_rank(share, r));
  }
  const float M = x[0] == -INFINITY ? 0.f : x[0], tmax = x[1];
  // sums: outside the top; of the top's exp(z / T), each entry once; of the teacher's weights and of their terms of the loss
  x[0] = m == -INFINITY ? 0.f : (sum.x + sum.y) * ex2((m - M) * p.scale);
  x[1] = x[2] = x[3] = 0.f;
  const float norm = tail ? p.teacher_lse[row] : tmax;
  for (int j = threadIdx.x; j < p.k; j += blockDim.x) {
    if (en.at[j] < 0) continue;
    bool first = true;
    if (twice || wraps || CLUSTER)   // (a CTA of a cluster has seen the bits of its own slots only)
      for (int e = 0; e < j; ++e) first &= en.at[e] != en.at[j];
    const float y = en.z[j] - M;
    if (first) x[1] += ex2(y * p.scale);
    const float lp = en.t[j] - norm, pj = expf(lp);
    x[2] += pj;
    if (pj > 0.f) x[3] += pj * (lp - y / p.temperature);
  }
  over_block<4, false>(x, red[1]);
  float out = x[0];
  if (CLUSTER) {
    if (threadIdx.x == 0) share[1] = out;
    cl.sync();
    out = 0.f;
    for (int r = 0; r < ranks; ++r) out += *cl.map_shared_rank(share + 1, r);
  }
  const float total = out + x[1];
  const float mass = tail ? 1.f : x[2];   // what the teacher's weights are divided by
  const float rest = tail ? fmaxf(0.f, 1.f - x[2]) : 0.f;
  if (threadIdx.x == 0 && rank == 0 && p.loss) {
    float l = tail ? x[3] + x[2] * logf(total) : x[3] / mass - logf(mass) + logf(total);
    if (rest > 0.f) l += rest * logf(rest / (out / total));
    if (total == 0.f) l = INFINITY;
    p.loss[row] = w * l;
  }
  if (dz) {
    // pass 2
    const float scale = w / p.temperature;
    const float inside = total == 0.f ? 0.f : scale / total;
    const float outside = rest > 0.f && out > 0.f ? inside - scale * (rest / out) : inside;
    const Val<2> from = all<2>(M), by = all<2>(p.scale), factor = all<2>(outside);
    for (int64_t base = v0; base < v1; base += (int64_t)kDeep * blockDim.x) {
      Vec<TZ> a[kDeep];
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const int64_t j = base + (int64_t)u * blockDim.x + threadIdx.x;
        if (j < v1) a[u] = rz.load(j, true);
      }
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const int64_t j = base + (int64_t)u * blockDim.x + threadIdx.x;
        if (j >= v1) continue;
#pragma unroll
        for (int i = 0; i < P; ++i) {
          Val<2> y = mul(sub(pair(a[u], i), from), by);
          y.x = ex2(y.x);
          y.y = ex2(y.y);
          set_pair(a[u], i, mul(y, factor));
        }
        if (together && rz.whole(j)) {
          __stcs(reinterpret_cast<uint4 *>(dz - rz.pad) + j, a[u].w);
        } else {
          const TZ *e = reinterpret_cast<const TZ *>(&a[u].w);
          for (int i = 0; i < N; ++i) {
            const int64_t s = j * N + i;
            if (s >= rz.pad && s < rz.slots) dz[s - rz.pad] = e[i];
          }
        }
      }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < p.k; j += blockDim.x) {
      const int64_t slot = (int64_t)en.at[j] + rz.pad;
      if (en.at[j] < 0 || slot < slot0 || slot >= slot1) continue;
      float pc = expf(en.t[j] - norm);
      bool first = true;
      if (twice || wraps) {   // an entry listed twice counts with both weights, in the order of the list
        pc = 0.f;
        for (int e = 0; e < p.k; ++e)
          if (en.at[e] == en.at[j]) {
            first &= e >= j;
            pc += expf(en.t[e] - norm);
          }
      }
      if (first) narrow(dz + en.at[j], ex2((en.z[j] - M) * p.scale) * inside - scale * (pc / mass));
    }
  }
  if (CLUSTER) cl.sync();   // nobody leaves while another CTA may still read its share
}

template <typename TZ, typename TT, typename TI, bool CLUSTER>
cudaError_t launch(const DistillArgs &p, int64_t r, int threads, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  auto kernel = distill_kernel<TZ, TT, TI, CLUSTER>;
  const size_t most = kMaxBits / 8 + 12 * (size_t)kMaxTop, bytes = 4 * (size_t)p.words + 12 * (size_t)p.k;
  cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), most, &done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(r * p.cluster));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim = {(unsigned)p.cluster, 1, 1};
  if (CLUSTER) { cfg.attrs = &at; cfg.numAttrs = 1; }
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename TZ, typename TT, typename TI> cudaError_t launch_rows(DistillArgs p, int64_t r, cudaStream_t s) {
  constexpr int N = Vec<TZ>::N;
  const int64_t vectors = ceil_div(p.v + N - 1, N);   // of the row on the least fortunate boundary
  // CTAs per row: one, unless the rows leave SMs empty and there are at least kDeep vectors for each thread of a CTA
  p.cluster = 1;
  while (p.cluster < kMaxCluster && r * p.cluster * 2 <= sm_count() && vectors / (p.cluster * 2) >= kDeep * kMaxThreads) p.cluster *= 2;
  const int64_t per = ceil_div(vectors, p.cluster);
  p.words = (int32_t)(std::min(kMaxBits, ceil_div(per * N, 32) * 32) / 32);
  const int threads = (int)std::min<int64_t>(kMaxThreads, std::max<int64_t>(128, ceil_div(per, 32) * 32));
  return p.cluster > 1 ? launch<TZ, TT, TI, true>(p, r, threads, s) : launch<TZ, TT, TI, false>(p, r, threads, s);
}

template <typename TZ, typename TT> cudaError_t launch_i(const DistillArgs &p, int32_t it, int64_t r, cudaStream_t s) {
  return it == DSGD_I64 ? launch_rows<TZ, TT, int64_t>(p, r, s) : launch_rows<TZ, TT, int32_t>(p, r, s);
}

ceca_status_t distill(const void *z, const void *idx, const void *t, const float *teacher_lse, const float *weight,
                      float *loss, void *dz, int64_t r, int64_t v, int64_t k, int64_t ldz, int64_t ldi, int64_t ldt,
                      int64_t lddz, int32_t logits_type, int32_t index_type, int32_t teacher_type, float temperature,
                      void *stream) {
  if (r < 0 || r >= ((int64_t)1 << 31) / kMaxCluster || v < 1 || v >= ((int64_t)1 << 31) || k < 0 || k > kMaxTop || ldz < v ||
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
  p.temperature = temperature;
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
