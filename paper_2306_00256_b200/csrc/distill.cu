// Distillation from a teacher's top logits: loss per row, and its gradient with respect to the student's logits.
//
//   q = softmax(z / T),  p_j = exp(t_j / T - N),  loss = w (sum_j p_j (log p_j - log q_j) [+ p0 log(p0 / q0)])
//   dz = (w / T) (m q - p) at the top's entries, (w / T) (m q [- p0 q / q0]) elsewhere, m = sum_j p_j [+ p0]: 1, or more where the top has more
//
// A CTA takes a row that fits in shared memory, or a cluster of up to 8 takes a part of it each, 32 KB a CTA, six CTAs an
// SM whose phases overlap; there are more to a row where there are few rows.  Every thread copies the vectors that it will
// work on, asynchronously, so a row is read once.  (Rows above 832 KB are read twice, the second time mostly from L2; for
// the loss alone nothing needs to be held.)  A first pass sums exponentials per thread, with a teacher_lse over the
// entries outside the top alone: q0 must not come from a difference of sums that may be nearly equal, so what is held of
// the top is struck out first, and the few entries are gathered and summed apart, in a frame of their own: the student's
// mass outside a top that towers over it may be too small for fp32, its logarithm and the shares of it are not.  The threads'
// sums, each in a frame of its own, meet in one exchange.  The second pass writes w / T (m / S - p0 / S0) exp((z - M) / T)
// everywhere, with S0 and M of pass 1 and S the sum of everything in that frame, and the top's entries are then written over.  Exponents are taken to
// base 2, z c - k with c = log2(e) / T and k = M c in one fma.
//
// 8192 rows of 128000 bf16 logits: 0.84 to 0.88 ms, 0.72 to 0.76 of the measured copy rate; two exponentials per logit keep the special
// function units busy for 0.48 ms of it.  2047 rows of 50001: 87 to 89 us, 0.70; 4096 rows of 32000 fp32 logits: 0.19 ms, 0.85.
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
constexpr int kMaxCluster = 8;
// Bytes that a CTA holds of a row: a whole one up to kMostHeld; of longer ones kHeld, or up to kMostHeld where kMaxCluster CTAs
// are not enough for that.  (A cluster's exchange costs some 2500 cycles, more than the second CTA on an SM that 100 KB
// leave room for saves: 2047 x 50001 bf16 88 us so, 100 us by clusters of 4.)
constexpr int64_t kHeld = 32 << 10, kMostHeld = 104 << 10;
constexpr int64_t kMaxBits = 1 << 20;   // of the bitmap; longer parts wrap around in it
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

struct DistillArgs {
  const void *z, *idx, *t;
  const float *teacher_lse, *weight;
  float *loss;
  void *dz;
  int64_t v, k, ldz, ldi, ldt, lddz;
  float scale;        // c = log2(e) / T
  float temperature;
  int32_t idx64, t16; // the types of idx and t
  int32_t cluster;    // CTAs per row
  int32_t per;        // vectors of each CTA
  int32_t words;      // of the bitmap, a multiple of 4
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

// What a warp, a CTA or a cluster knows of its part of a row: the sum of 2^(z c - k) by pass 1, and of the top, whose frame kt is
// another because either may lie beyond an exponential's reach from the other, the same sum (each entry once), the
// teacher's weights p, and p (log p - ln2 (z c - kt)).
struct alignas(16) Known {
  float k, kt, sum, top, mass, terms, pad[2];
};
// The n parts of `all` in one frame of each kind, on every lane of the warp that asks: each lane moves its own there (terms
// move by ln2 p times the distance), and the sums run over the lanes in one fixed order.
template <int MOST> __device__ __forceinline__ Known joined(const Known *all, int n) {
  const int lane = threadIdx.x & 31;
  Known q[(MOST + 31) / 32], a{-INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < (MOST + 31) / 32; ++i) {
    q[i] = lane + 32 * i < n ? all[lane + 32 * i] : Known{-INFINITY, -INFINITY};
    a.k = fmaxf(a.k, q[i].k);
    a.kt = fmaxf(a.kt, q[i].kt);
  }
  a.k = warp_max(a.k);
  a.kt = warp_max(a.kt);
#pragma unroll
  for (int i = 0; i < (MOST + 31) / 32; ++i)
    if (lane + 32 * i < n) {
      const float d = q[i].kt - a.kt;
      a.sum += q[i].sum * ex2(q[i].k - a.k);
      a.top += q[i].top * ex2(d);
      a.terms += q[i].terms - kLn2 * d * q[i].mass;
      a.mass += q[i].mass;
    }
  a.sum = warp_sum(a.sum);
  a.top = warp_sum(a.top);
  a.terms = warp_sum(a.terms);
  a.mass = warp_sum(a.mass);
  return a;
}

// Shared memory behind the bitmap: k entries of each.
struct Entries {
  int32_t *at;    // the vocabulary entry where it lies in this part, or -1
  float *t, *z;   // the teacher's logit / T, the student's logit
};

__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive(bool published) {   // without anything published, no wait for earlier stores
  if (published) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}

// HELD: the part fits in shared memory.
template <typename TZ, int THREADS, bool CLUSTER, bool HELD>
__global__ void __launch_bounds__(THREADS, 768 / THREADS) distill_kernel(const DistillArgs p) {
  constexpr int N = Vec<TZ>::N, P = Vec<TZ>::P, W = THREADS / 32, hop = kDeep * THREADS;
  extern __shared__ uint4 memory[];   // the part's whole vectors, the bitmap, the entries
  constexpr int kParts = W * (CLUSTER ? kMaxCluster : 1);
  __shared__ Known share[kParts];   // of each warp of the cluster
  __shared__ float tops[W];
  __shared__ float2 far_red[W], far_share[kMaxCluster];
  uint32_t *bitmap = reinterpret_cast<uint32_t *>(memory + (HELD ? p.per : 0));
  Entries en;
  en.at = reinterpret_cast<int32_t *>(bitmap + p.words);
  en.t = reinterpret_cast<float *>(en.at + p.k);
  en.z = en.t + p.k;
  const int tid = threadIdx.x, warp = tid >> 5, ranks = CLUSTER ? p.cluster : 1;
  const uint32_t row = CLUSTER ? blockIdx.x / ranks : blockIdx.x;
  const int rank = CLUSTER ? (int)(blockIdx.x - row * ranks) : 0;
  const TZ *z = static_cast<const TZ *>(p.z) + row * p.ldz;
  TZ *dz = p.dz ? static_cast<TZ *>(p.dz) + row * p.lddz : nullptr;
  const auto listed = [&](int j) -> int64_t {
    const int64_t i = row * p.ldi + j;
    return p.idx64 ? static_cast<const int64_t *>(p.idx)[i] : static_cast<const int32_t *>(p.idx)[i];
  };
  const auto teacher = [&](int j) -> float {
    const int64_t i = row * p.ldt + j;
    return p.t16 ? widen(static_cast<const bf16 *>(p.t)[i]) : static_cast<const float *>(p.t)[i];
  };
  const float w = p.weight ? p.weight[row] : 1.f;
  const bool tail = p.teacher_lse != nullptr;
  const float lse = tail ? p.teacher_lse[row] : 0.f;
  int64_t at = -1;   // the thread's first entry is on its way before the row is
  float tj = 0.f;
  if (tid < p.k) {
    at = listed(tid);
    tj = teacher(tid);
  }
  const Part<TZ> part(z, p.v, rank, p.per);
  const uint32_t slot0 = part.slot0, slot1 = part.slot1;
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
  const int count = part.w1 - part.w0;
  const uint4 *from = reinterpret_cast<const uint4 *>(z - part.pad) + part.w0 + tid;
  uint4 *dst = reinterpret_cast<uint4 *>(dz - part.pad) + part.w0 + tid;   // used when z and dz lie together
  const uint4 *src = HELD ? memory + tid : from;

  // every CTA of the cluster runs before anybody writes into its shared memory
  if (CLUSTER) cluster_arrive(false);
  const auto nothing = [&]() {   // no loss, a zero gradient
    if (tid == 0 && rank == 0 && p.loss) p.loss[row] = 0.f;
    if (dz) {
      if (together)
        for (int j = 0; j < count - tid; j += THREADS) __stcs(dst + j, make_uint4(0, 0, 0, 0));
      else
        for (int64_t e = (int64_t)part.w0 * N + tid; e < (int64_t)part.w1 * N; e += THREADS) narrow(dz + e - part.pad, 0.f);
      if (part.edge >= 0) narrow(dz + part.edge - part.pad, 0.f);
    }
  };
  for (int c = tid; c < p.words / 4; c += THREADS) reinterpret_cast<uint4 *>(bitmap)[c] = make_uint4(0, 0, 0, 0);
  if (w == 0.f) {
    if (CLUSTER) cluster_wait();
    nothing();
    return;
  }
  const float edge = part.edge >= 0 ? widen(z[part.edge - part.pad]) : 0.f;
  if (HELD) {
    const uint32_t to = smem_u32(memory + tid);
    for (int j = 0; j < count - tid; j += THREADS)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + j * 16), "l"(from + j) : "memory");
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  __syncthreads();
  // The top: its entries, which of them lie in this part, the bitmap.  In tail mode what is held of them becomes
  // -infinity, so that the passes need not ask.
  TZ *held = reinterpret_cast<TZ *>(memory) - (int64_t)part.w0 * N;   // slot s is held[s]
  float tmax = -INFINITY;
  bool again = false;   // whether an entry of the thread is listed twice
  for (int j = tid; j < p.k; j += THREADS) {
    if (j != tid) {
      at = listed(j);
      tj = teacher(j);
    }
    tj /= p.temperature;
    const bool there = at >= 0 && at < p.v && !(tj == -INFINITY);
    const int64_t slot = at + part.pad;
    const bool here = there && slot >= slot0 && slot < slot1;
    en.at[j] = here ? (int32_t)at : -1;
    en.t[j] = tj;
    if (there) tmax = fmaxf(tmax, tj == tj ? tj : INFINITY);   // (a NaN is there as well)
    if (here) {
      const uint32_t b = (uint32_t)((slot - slot0) & (kMaxBits - 1));
      again |= atomicOr(bitmap + (b >> 5), 1u << (b & 31)) >> (b & 31) & 1;
      const bool kept = HELD && slot >= (int64_t)part.w0 * N && slot < (int64_t)part.w1 * N;
      en.z[j] = kept && !tail ? widen(held[slot]) : widen(z[at]);   // (listed twice, it is -infinity there by now)
      if (kept && tail) narrow(held + slot, -INFINITY);
    }
  }
  tmax = warp_max(tmax);
  if ((tid & 31) == 0) tops[warp] = tmax;
  const bool twice = __syncthreads_or(again);
#pragma unroll
  for (int i = 0; i < W; ++i) tmax = fmaxf(tmax, tops[i]);
  if (CLUSTER) cluster_wait();
  if (tmax == -INFINITY) {   // no teacher entry
    nothing();
    return;
  }

  // which of the N slots from s on (a multiple of N) are in the top
  const uint8_t *bytes = reinterpret_cast<const uint8_t *>(bitmap);
  const auto in_top = [&](int64_t s) -> uint32_t {
    const uint32_t b = (uint32_t)((s - slot0) & (kMaxBits - 1));
    uint32_t m = N == 8 ? bytes[b >> 3] : bytes[b >> 3] >> (b & 4) & 15u;
    if (!HELD && m && slot1 - slot0 > kMaxBits) {   // the bitmap wraps around: the bit may be another slot's
      m = 0;
      for (int e = 0; e < p.k; ++e) {
        const int64_t d = (int64_t)en.at[e] + part.pad - s;
        if (en.at[e] >= 0 && d >= 0 && d < N) m |= 1u << d;
      }
    }
    return m;
  };
  const auto counts = [&](int64_t s) { return !tail || !(in_top(s / N * N) >> (s % N) & 1); };   // in pass 1's sum

  // pass 1: maximum and sum, in tail mode over the entries outside the top
  const bool edge_counts = part.edge >= 0 && counts(part.edge);
  Seen seen(edge_counts ? edge : -INFINITY, p.scale);
  if (edge_counts) seen.sum.x = ex2(fmaf(edge, p.scale, -seen.k));
  const int64_t s0 = (int64_t)(part.w0 + tid) * N;
  for (int base = 0; base < count; base += hop) {
    Vec<TZ> a[kDeep];
    const int left = count - base - tid;
    if (base + hop <= count) {
#pragma unroll
      for (int u = 0; u < kDeep; ++u) a[u].w = src[base + u * THREADS];
    } else {
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        a[u] = all_least<TZ>();
        if (u * THREADS < left) a[u].w = src[base + u * THREADS];
      }
    }
    if (!HELD && tail) {
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const uint32_t mask = u * THREADS < left ? in_top(s0 + (int64_t)(base + u * THREADS) * N) : 0;
        if (mask) strike(a[u], mask);
      }
    }
    if (!seen.settled()) seen.frame<kDeep>(a, p.scale);
    seen.take<kDeep>(a, p.scale);
  }
  if (seen.beyond()) {   // once more, a vector at a time
    const auto vector = [&](int j) {
      Vec<TZ> a{src[j]};
      const uint32_t mask = !HELD && tail ? in_top(s0 + (int64_t)j * N) : 0;
      if (mask) strike(a, mask);
      return a;
    };
    float top = edge_counts ? edge : -INFINITY;
    for (int j = 0; j < count - tid; j += THREADS) {
      const Vec<TZ> a = vector(j);
      top = fmaxf(top, top_of<1>(&a));
    }
    seen = Seen(top, p.scale);
    if (edge_counts) seen.sum.x = ex2(fmaf(edge, p.scale, -seen.k));
    for (int j = 0; j < count - tid; j += THREADS) {
      const Vec<TZ> a = vector(j);
      seen.take<1>(&a, p.scale);
    }
  }
  // the warp's part in frames of its own, then everybody's
  Known all_of;
  float kt = -kFar;
  for (int j = tid; j < p.k; j += THREADS)
    if (en.at[j] >= 0) kt = fmaxf(kt, frame_of(en.z[j], p.scale));
  all_of.k = warp_max(seen.k);
  all_of.kt = warp_max(kt);
  kt = all_of.kt;
  const float norm = tail ? lse : tmax;
  float sums[4] = {(seen.sum.x + seen.sum.y) * ex2(seen.k - all_of.k), 0.f, 0.f, 0.f};
  const auto entry = [&](int j, float y) {   // what entry j adds, its exponent being y
    bool first = true;
    if (twice)
      for (int e = 0; e < j; ++e) first &= en.at[e] != en.at[j];
    if (tail && first) sums[1] += ex2(y);
    const float lp = en.t[j] - norm, pj = expf(lp);
    sums[2] += pj;
    if (pj > 0.f) sums[3] += pj * (lp - kLn2 * y);
  };
  for (int j = tid; j < p.k; j += THREADS)
    if (en.at[j] >= 0) entry(j, fmaf(en.z[j], p.scale, -kt));
  const auto gather = [&]() {
    all_of.sum = warp_sum(sums[0]);
    all_of.top = warp_sum(sums[1]);
    all_of.mass = warp_sum(sums[2]);
    all_of.terms = warp_sum(sums[3]);
    const int lane = tid & 31;
    if (CLUSTER) {
      if (lane < ranks) *cg::this_cluster().map_shared_rank(share + rank * W + warp, lane) = all_of;
      cluster_arrive(true);
      cluster_wait();
    } else if (W > 1) {
      if (lane == 0) share[warp] = all_of;
      __syncthreads();
    }
    if (CLUSTER || W > 1) all_of = joined<kParts>(share, W * ranks);
  };
  gather();
  // The frames: K of pass 1's sum, Kt of the top's, Ka of everything, and how far below Ka the others lie (without a
  // teacher_lse pass 1 has seen everything, and Kt may lie above).  A far row's are 0, and its logits less these M.
  const float K = all_of.k, Kt = all_of.kt, Ka = tail ? fmaxf(K, Kt) : K;
  float M = 0.f, Mt = 0.f, Ma = 0.f, under = K - Ka, under_top = Kt - Ka;
  const bool far = !(fabsf(fmaxf(K, Kt)) < kFar && all_of.sum < INFINITY);
  if (far) {   // exponents beyond +-kFar, infinities or NaN: once more, element by element
    const int64_t s1 = min((int64_t)slot1, p.v + part.pad);
    M = Mt = -INFINITY;
    for (int64_t s = max((int64_t)slot0, (int64_t)part.pad) + tid; s < s1; s += THREADS)
      if (counts(s)) M = fmaxf(M, widen(z[s - part.pad]));
    for (int j = tid; j < p.k; j += THREADS)
      if (en.at[j] >= 0) Mt = fmaxf(Mt, en.z[j]);
    M = warp_max(M);
    Mt = warp_max(Mt);
    if ((tid & 31) == 0) far_red[warp] = make_float2(M, Mt);
    __syncthreads();
    const auto greatest = [&](const float2 *of, int n) {
      for (int i = 0; i < n; ++i) {
        M = fmaxf(M, of[i].x);
        Mt = fmaxf(Mt, of[i].y);
      }
    };
    greatest(far_red, W);
    if (CLUSTER) {
      if (tid < ranks) *cg::this_cluster().map_shared_rank(far_share + rank, tid) = make_float2(M, Mt);
      cluster_arrive(tid < 32);
      cluster_wait();
      greatest(far_share, ranks);
    }
    Ma = tail ? fmaxf(M, Mt) : M;   // where there is nothing, there are no distances either
    under = M == -INFINITY ? 0.f : (M - Ma) * p.scale;
    under_top = Mt == -INFINITY || Ma == -INFINITY ? 0.f : (Mt - Ma) * p.scale;
    if (M == -INFINITY) M = 0.f;
    if (Mt == -INFINITY) Mt = 0.f;
    if (Ma == -INFINITY) Ma = 0.f;
    sums[0] = sums[1] = sums[2] = sums[3] = 0.f;
    for (int64_t s = max((int64_t)slot0, (int64_t)part.pad) + tid; s < s1; s += THREADS)
      if (counts(s)) sums[0] += ex2((widen(z[s - part.pad]) - M) * p.scale);
    for (int j = tid; j < p.k; j += THREADS)
      if (en.at[j] >= 0) entry(j, (en.z[j] - Mt) * p.scale);
    all_of.k = all_of.kt = 0.f;   // the same frames for all
    if (CLUSTER) {    // everybody has read the first parts
      cluster_arrive(false);
      cluster_wait();
    } else {
      __syncthreads();
    }
    gather();
  }
  const float out = all_of.sum, total = out * ex2(under) + (tail ? all_of.top * ex2(under_top) : 0.f);
  const float mass = tail ? 1.f : all_of.mass;   // what the teacher's weights are divided by
  // (a NaN of the teacher goes on from here: fmaxf would end it)
  const float rest = tail && !(all_of.mass >= 1.f) ? 1.f - all_of.mass : 0.f;
  const float compared = tail && !(all_of.mass <= 1.f) ? all_of.mass : 1.f;   // with log q, the top's mass and the rest
  if (tid == 0 && rank == 0 && p.loss) {
    const float log_total = logf(total) - kLn2 * under_top;   // in the top's frame
    float l = tail ? all_of.terms + all_of.mass * log_total : all_of.terms / mass - logf(mass) + log_total;
    if (rest > 0.f) l += rest * (logf(rest * (total / out)) - kLn2 * under);
    if (total == 0.f && all_of.mass == all_of.mass) l = INFINITY;
    p.loss[row] = w * l;
  }
  if (!dz) return;
  // pass 2
  const float scale = w / p.temperature;
  // The frames of the second pass, and what their exponentials are multiplied by besides: q is a share of everything at the top's
  // entries, of pass 1's sum elsewhere.  Over a low temperature a q below 2^-126 is a gradient that is not, so frames are lowered by
  // the binades of w / T; and where a sum shows a frame far below its maximum, they are raised by the sum's, so that the factor
  // stays a normal number.  Not otherwise: an exponent's rounding grows with it, and is least for the largest q in a frame that is the maximum.
  float low = K, low_all = Ka, drop = 1.f, drop_all = 1.f, lift = 0.f;
  if (fabsf(scale) >= 2.f || fmaxf(out, total) >= 0x1p32f) {
    const auto binade = [](float x) { return (float)((__float_as_int(fabsf(x)) >> 23) - 127); };
    lift = fminf(fmaxf(binade(scale), 0.f), 32.f);
    low = K + ((out >= 0x1p32f ? binade(out) : 0.f) - lift);
    low_all = Ka + ((total >= 0x1p32f ? binade(total) : 0.f) - lift);
    drop = ex2(far ? -lift : low - K);
    drop_all = ex2(far ? -lift : low_all - Ka);
  }
  const auto raised = [&](float v, float m, float low) { return ex2(far ? fmaf(v - m, p.scale, lift) : fmaf(v, p.scale, -low)); };
  const float part_of_all = (total == 0.f ? 0.f : scale / total) * compared, inside = part_of_all * drop_all;
  const float outside = (part_of_all * ex2(under) - (rest > 0.f && out > 0.f ? scale * (rest / out) : 0.f)) * drop;
  if (together && !far) {
    const Val<2> shift = all<2>(-low), by = all<2>(p.scale), factor = all<2>(outside);
    const auto turn = [&](Vec<TZ> v) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        Val<2> y = fma(pair(v, i), by, shift);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        set_pair(v, i, mul(y, factor));
      }
      return v.w;
    };
    for (int base = 0; base < count; base += hop) {
      Vec<TZ> a[kDeep];
      if (base + hop <= count) {
#pragma unroll
        for (int u = 0; u < kDeep; ++u) a[u].w = src[base + u * THREADS];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) __stcs(dst + base + u * THREADS, turn(a[u]));
      } else {
        const int left = count - base - tid;
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
          if (u * THREADS < left) a[u].w = src[base + u * THREADS];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
          if (u * THREADS < left) __stcs(dst + base + u * THREADS, turn(a[u]));
      }
    }
    if (part.edge >= 0) narrow(dz + part.edge - part.pad, raised(edge, M, low) * outside);
  } else {   // element by element, from memory (where dz is z, each thread reads what it writes over)
    const int64_t s1 = min((int64_t)slot1, p.v + part.pad);
    for (int64_t s = max((int64_t)slot0, (int64_t)part.pad) + tid; s < s1; s += THREADS)
      narrow(dz + s - part.pad, raised(widen(z[s - part.pad]), M, low) * outside);
  }
  __syncthreads();
  for (int j = tid; j < p.k; j += THREADS) {
    if (en.at[j] < 0) continue;
    float pc = expf(en.t[j] - norm);
    bool first = true;
    if (twice) {   // an entry listed twice counts with both weights, in the order of the list
      pc = 0.f;
      for (int e = 0; e < p.k; ++e)
        if (en.at[e] == en.at[j]) {
          first &= e >= j;
          pc += expf(en.t[e] - norm);
        }
    }
    if (first) narrow(dz + en.at[j], raised(en.z[j], Ma, low_all) * inside - scale * (pc / mass));
  }
}

template <typename TZ, int THREADS, bool CLUSTER, bool HELD> cudaError_t launch(const DistillArgs &p, int64_t r, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  auto kernel = distill_kernel<TZ, THREADS, CLUSTER, HELD>;
  const size_t fixed = 12 * (size_t)kMaxTop, most = fixed + (HELD ? kMostHeld + kMostHeld / sizeof(TZ) / 8 + 16 : kMaxBits / 8);
  const size_t bytes = (HELD ? 16 * (size_t)p.per : 0) + 4 * (size_t)p.words + 12 * (size_t)p.k;
  cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), most, &done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(r * p.cluster));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim = {(unsigned)p.cluster, 1, 1};
  if (CLUSTER) { cfg.attrs = &at; cfg.numAttrs = 1; }
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename TZ> cudaError_t launch_rows(DistillArgs p, int64_t r, cudaStream_t s) {
  constexpr int N = Vec<TZ>::N;
  const int64_t vectors = ceil_div(p.v + N - 1, N);   // of the row on the least fortunate boundary
  // The loss alone needs no second pass, and nothing held: a CTA streams a row, as long as there are rows for all SMs.
  if (!p.dz && r >= 4 * sm_count() && 16 * vectors > kHeld / 2) {
    p.cluster = 1;
    p.per = (int32_t)vectors;
    p.words = (int32_t)(std::min(kMaxBits, ceil_div(vectors * N, 128) * 128) / 32);
    return launch<TZ, 128, false, false>(p, r, s);
  }
  // CTAs per row: what holds the row, and more where the rows leave SMs empty and a part is still 16 vectors a thread
  const auto part = [&](int64_t ctas) { return 16 * ceil_div(vectors, ctas); };
  p.cluster = 1;
  if (part(1) > kMostHeld)
    while (p.cluster < kMaxCluster && part(p.cluster) > kHeld) p.cluster *= 2;
  while (p.cluster < kMaxCluster && r * p.cluster * 2 <= 4 * sm_count() && vectors >= 2 * 16 * 128 * p.cluster) p.cluster *= 2;
  const int64_t per = ceil_div(vectors, p.cluster);
  p.per = (int32_t)per;
  p.words = (int32_t)(std::min(kMaxBits, ceil_div(per * N, 128) * 128) / 32);
  if (16 * per > kMostHeld) return launch<TZ, 256, true, false>(p, r, s);
  if (16 * per > kHeld) return p.cluster > 1 ? launch<TZ, 256, true, true>(p, r, s) : launch<TZ, 256, false, true>(p, r, s);
  if (p.cluster > 1) return launch<TZ, 128, true, true>(p, r, s);
  // few vectors a thread for short rows, so that many of them are at work on an SM
  if (per <= 8 * 32) return launch<TZ, 32, false, true>(p, r, s);
  return per <= 16 * 64 ? launch<TZ, 64, false, true>(p, r, s) : launch<TZ, 128, false, true>(p, r, s);
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
  p.idx64 = index_type == DSGD_I64;
  p.t16 = teacher_type == DSGD_BF16;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = logits_type == DSGD_F32 ? launch_rows<float>(p, r, s) : launch_rows<bf16>(p, r, s);
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
