// Internal: rows of logits in 16-byte vectors, sums of their exponentials in frames, and a cluster's barrier.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "values.h"

namespace ceca {

constexpr int kDeep = 4;                // vectors a thread works on at a time
constexpr float kLn2 = 0.6931471805599453f;
// Exponents of this size: z c - k is exact but for its own rounding whatever k is, so a frame's k is m c rounded (kept as it is
// rounded: all that move between frames, or that use one later, go by k).  That rounding shifts a frame by up to half an ulp of k,
// 8 here and harmless; beyond, an exponential could overflow by it.  Logits below -kFar / c are masks; a row that has no others, or one
// above kFar / c, gets its own, slower sums of 2^((z - M) c).
constexpr float kFar = 0x1p27f;
// A thread looks for a larger frame as long as it has seen no exponent above this, so that additive masks (of -1e4, say) end up in
// no frame beside real logits; and the sum at which a thread that has settled starts again.  (4096 x 128000 bf16, 999 of 1000 logits
// masked: 432 us with -1e4, 431 with -infinity.)
constexpr float kLow = -3e3f, kLeave = 0x1p80f;

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
// The largest element of D vectors.
template <int D> __device__ __forceinline__ float top_of(const Vec<float> *v) {
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < D; ++u)
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[u].w.x), __uint_as_float(v[u].w.y)), fmaxf(__uint_as_float(v[u].w.z), __uint_as_float(v[u].w.w))));
  return m;
}
template <int D> __device__ __forceinline__ float top_of(const Vec<bf16> *v) {
  const auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
  __nv_bfloat162 m = h(v[0].w.x);
#pragma unroll
  for (int u = 0; u < D; ++u) m = __hmax2(m, __hmax2(__hmax2(h(v[u].w.x), h(v[u].w.y)), __hmax2(h(v[u].w.z), h(v[u].w.w))));
  return fmaxf(__low2float(m), __high2float(m));
}

// What one thread has seen: sum counts 2^(z c - k), k = m c.  m is the largest of the first vectors that are not masked, not of
// all: a frame does not have to be the maximum, only so near to it that the sum stays below kLeave.  (A sum that does not is
// taken again, in the frame of the maximum.)  Then what a factor below 2^-126 makes nothing of when frames are joined is
// below 2^-46 of the sum in the other frame, and no product with the joined sum or its reciprocal leaves the normal numbers.
__device__ __forceinline__ float frame_of(float top, float scale) { return __fmul_rn(top, scale); }   // (not part of an fma)
struct Seen {
  float k;
  Val<2> sum{0.f, 0.f};
  __device__ __forceinline__ Seen(float top, float scale) : k(fmaxf(frame_of(top, scale), -kFar)) {}
  __device__ __forceinline__ bool settled() const { return k > kLow; }
  __device__ __forceinline__ bool beyond() const { return sum.x + sum.y > kLeave; }
  template <int D, typename T> __device__ __forceinline__ void frame(const Vec<T> *a, float scale) {
    const float to = frame_of(top_of<D>(a), scale);
    if (to > k) {
      sum = mul(sum, all<2>(ex2(k - to)));   // (an edge element, or masked ones, may be in it)
      k = to;
    }
  }
  template <int D, typename T> __device__ __forceinline__ void take(const Vec<T> *a, float scale) {
    const Val<2> shift = all<2>(-k), by = all<2>(scale);
#pragma unroll
    for (int u = 0; u < D; ++u)
#pragma unroll
      for (int i = 0; i < Vec<T>::P; ++i) {
        Val<2> y = fma(pair(a[u], i), by, shift);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        sum = add(sum, y);
      }
  }
};

// The part of a row that a CTA takes, in slots: slot s is element s - pad, so that vectors of N slots lie on 16-byte
// boundaries.  Whole vectors are [w0, w1); what the row has before and after them in this part, fewer than N elements
// each, goes one to a thread (`edge`, a slot, or -1).
template <typename T> struct Part {
  static constexpr int N = Vec<T>::N;
  int pad, w0, w1;
  uint32_t slot0, slot1;
  int64_t edge;
  __device__ __forceinline__ Part(const T *row, int64_t v, int rank, int per) {
    pad = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const uint32_t slots = (uint32_t)v + pad;
    const int vectors = (int)((slots + N - 1) / N);
    const int v0 = min(vectors, rank * per), v1 = min(vectors, v0 + per);
    slot0 = (uint32_t)v0 * N;
    slot1 = (uint32_t)v1 * N;
    w0 = v0 + (v0 == 0 && pad > 0);
    w1 = max(w0, min(v1, (int)(slots / N)));
    edge = -1;
    const int i = threadIdx.x;
    if (i < N) {
      if (v0 == 0 && pad > 0 && i >= pad && i < slots) edge = i;
    } else if (i < 2 * N) {
      const uint32_t s = (uint32_t)w1 * N + i - N;
      if (v1 == vectors && v1 > v0 && s < slots && s < slot1) edge = s;
    }
  }
};

__device__ __forceinline__ float warp_max(float x) {
  asm("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(x));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive(bool published) {   // without anything published, no wait for earlier stores
  if (published) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}

}  // namespace ceca
