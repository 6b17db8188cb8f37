// Log-probabilities of tokens, and the policy and preference losses that are made of them, with their gradients.
//
//   l = log softmax(z / T)[token],  dz = (c / T) (one-hot - q),  c the derivative of the loss by l
//
// A row is summed without its token: with R = sum of 2^(z c - k) over the others and y the token's exponent in that frame, 1 - q = R / (R + 2^y)
// and l = -log(1 + R / 2^y) keep their digits where the model is sure, and the others' share of the gradient is (c / T) (1 - q) / R each.
//
// Memory bounds it, and how often a row is read.  Where the derivative follows from the row's own sum (the policy's) it is read once, and stays in registers
// between the sum and the gradient: several short rows a warp, 16 or 32 KB a CTA, up to 256 KB (512 KB with larger CTAs) a cluster of eight.  The preference's
// derivative waits for the rows of two whole sequences: rows are summed in a stream of 8 KB parts, a warp each, joined, the pairs' losses taken, and
// all are read again (from L2 no faster: the writes are what takes the time there).  The four launches begin early, each waiting for the one before.
//
// 2047 rows of 50001 fp32 logits: log-probabilities 64 us (0.98 of the measured copy rate), policy gradient 163 (0.76).  8192 x 128000 bf16: 299 us (all of it),
// 819 (0.78: no one unit is full, special functions 51 %, issue slots 47 %; load, sum, exchange between eight CTAs and write of a row follow one another).
// 16384 x 32000 bf16: policy gradient 388 us (0.82), preference gradient 492 (0.97 for the three passes that it takes, 0.65 for two); 8192 x 8192 bf16 54 us
// (0.76; by CTAs of 128 threads a fifth more).
// Tried for the policy's rows and slower: clusters that stay and fetch their next row to shared memory meanwhile (907 us), 256 threads of 8 vectors each
// (915), 6 or 4 CTAs an SM instead of 5 (889, 884), and loops without a question for each vector (886).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

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
  int32_t parts, per;   // of a row, and vectors of each
  int32_t ranks;        // CTAs that hold a row
  RowOut *rows;         // workspace, r of each; NULL without a gradient
  float2 *sums;         // r x parts
  float *row_logp, *row_slopes;   // of the preference loss, the second with a gradient
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
  const float adv = p.advantage[i], past = l - p.old_logp[i], ratio = expf(past);
  const float plain = adv == 0.f && past < INFINITY ? 0.f : ratio * adv;   // (0 too where a finite ratio is beyond fp32)
  const float clipped = fminf(fmaxf(ratio, p.low), p.high) * adv;
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
  return {s.k, s.rest == 0.f ? (own == own ? 0.f : own) : own / s.rest, own, s.far ? 1 : 0};   // (a NaN is one for the whole row)
}

// Over a low temperature, or a large weight, a share below 2^-126 is a gradient that is not: where the factor is above 1 the frame is lowered by
// its binades, and the factor by what that is.  A far row's exponents get them added, `lift`.
__device__ __forceinline__ float lifted(RowOut &o) {
  if (!(fabsf(o.factor) >= 2.f)) return 0.f;
  const float lift = fminf((float)((int)(__float_as_uint(o.factor) >> 23 & 255u) - 127), 64.f);
  const float low = o.far ? -lift : o.k - lift, by = o.far ? -lift : low - o.k;   // (as it is rounded)
  if (!o.far) o.k = low;
  o.factor *= exp2f(by);
  return o.far ? lift : 0.f;
}

constexpr int kWarps = 4, kThreads = 32 * kWarps;
// Warps work on their own: on a part of a row of up to 16 vectors a lane, whose loads are all under way at a time.
constexpr int kVectors = 16, kPart = 32 * kVectors;
constexpr int kMostRanks = 8;   // CTAs of a cluster

// The part of a row that a warp takes, in slots: slot s is element s - pad, so that vectors of N slots lie on 16-byte boundaries.  Whole vectors are
// [w0, w1); what the row has before and after them in this part goes one to a lane (`edge`, a slot, or -1).
template <typename T> struct WarpPart {
  static constexpr int N = Vec<T>::N;
  int pad, w0, w1, edge;
  __device__ __forceinline__ WarpPart(const T *row, int64_t v, int part, int per) {
    pad = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const uint32_t slots = (uint32_t)v + pad;
    const int vectors = (int)((slots + N - 1) / N), v0 = min(vectors, part * per), v1 = min(vectors, v0 + per), lane = threadIdx.x & 31;
    w0 = v0 + (v0 == 0 && pad > 0);
    w1 = max(w0, min(v1, (int)(slots / N)));
    edge = -1;
    if (lane < N) {
      if (v0 == 0 && v1 > 0 && pad > 0 && lane >= pad && lane < slots) edge = lane;
    } else if (lane < 2 * N) {
      const uint32_t s = (uint32_t)w1 * N + lane - N;
      if (v1 == vectors && v1 > v0 && s < slots && s < (uint32_t)v1 * N) edge = (int)s;
    }
  }
};

// Whether a row is looked at: it has a token, and a weight.
__device__ __forceinline__ bool is_live(const TokenArgs &p, int64_t i, int64_t tok, float &w) {
  w = p.what == kPolicy && p.weight ? p.weight[i] : 1.f;
  return tok >= 0 && tok < p.v && w != 0.f;
}

// Sums of 2^(z c - k) over the parts of rows without their tokens, each in the frame of its own maximum.
template <typename TZ> __global__ void __launch_bounds__(kThreads) sum_kernel(const TokenArgs p) {
  constexpr int N = Vec<TZ>::N;
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5), i = task / p.parts;
  if (i < p.r) {
    const int64_t tok = index_of(p.tokens, p.idx64, i);
    float w;
    if (is_live(p, i, tok, w)) {
      const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
      const WarpPart<TZ> part(z, p.v, (int)(task - i * p.parts), p.per);
      const uint4 *from = reinterpret_cast<const uint4 *>(z - part.pad) + part.w0 + lane;
      const int count = part.w1 - part.w0 - lane;   // of this lane's vectors, every 32nd
      Vec<TZ> a[kVectors];
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        a[u] = all_least<TZ>();
        if (32 * u < count) a[u].w = __ldcs(from + 32 * u);
      }
      const int64_t slot = tok + part.pad;
      float edge = part.edge >= 0 && part.edge != slot ? widen(z[part.edge - part.pad]) : -INFINITY;
      const int64_t at = slot / N - part.w0 - lane;   // the token's vector, as this lane counts
      if (at >= 0 && at < count && at % 32 == 0) {
#pragma unroll
        for (int u = 0; u < kVectors; ++u)
          if (at == 32 * u) strike(a[u], 1u << (slot % N));
      }
      // the frame of the warp: masked ones alone have a low one
      const float k = warp_max(fmaxf(frame_of(fmaxf(edge, top_of<kVectors>(a)), p.scale), -kFar));
      const Val<2> shift = all<2>(-k), by = all<2>(p.scale);
      Val<2> sum{ex2(fmaf(edge, p.scale, -k)), 0.f};
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        if (32 * u >= count) break;
#pragma unroll
        for (int e = 0; e < Vec<TZ>::P; ++e) {
          Val<2> y = fma(pair(a[u], e), by, shift);
          y.x = ex2(y.x);
          y.y = ex2(y.y);
          sum = add(sum, y);
        }
      }
      const float total = warp_sum(sum.x + sum.y);
      if (lane == 0) p.sums[task] = make_float2(k, total);
    }
  }
  follow_early();
}

// The sums of a far row, by a warp, element by element.
template <typename TZ> __device__ __noinline__ void far_sums(const TokenArgs &p, const TZ *z, int64_t tok, float own, RowSum &s) {
  const int lane = threadIdx.x & 31;
  float m = -INFINITY, sum = 0.f;
  for (int64_t c = lane; c < p.v; c += 32)
    if (c != tok) m = fmaxf(m, widen(z[c]));
  m = warp_max(m);
  s.k = m == -INFINITY ? own : m;
  for (int64_t c = lane; c < p.v; c += 32) {
    const float x = widen(z[c]);
    if (c != tok) sum += m == -INFINITY ? (x == -INFINITY ? 0.f : NAN) : ex2((x - s.k) * p.scale);
  }
  s.rest = warp_sum(sum);
}
// The token's exponent in the frame of the others.
__device__ __forceinline__ float own_exponent(const TokenArgs &p, const RowSum &s, float own) {
  return own == -INFINITY ? own : own == INFINITY ? NAN : s.far ? (own - s.k) * p.scale : fmaf(own, p.scale, -s.k);
}
// What is written of a row besides its gradient, by one thread; and what the gradient needs.
__device__ __forceinline__ RowOut finish_row(const TokenArgs &p, int64_t i, const RowSum &s, float w, bool writes) {
  const Odds o = odds_of(s);
  RowOut out = row_out(p, s, o, 1.f);   // of the preference loss: the sequence's slope comes later
  if (p.what == kLogprob && writes) p.logp[i] = o.logp;
  if (p.what == kPolicy) {
    const float2 l = policy(p, i, w, o.logp);
    out = row_out(p, s, o, l.y);
    if (writes) p.loss[i] = l.x;
    if (writes && p.logp) p.logp[i] = o.logp;
  }
  if (p.what == kPreference && writes) p.row_logp[i] = o.logp;
  if (p.rows && writes) p.rows[i] = out;
  if (p.row_slopes && writes) p.row_slopes[i] = 0.f;   // of rows outside all sequences
  return out;
}
__device__ __forceinline__ void finish_dead_row(const TokenArgs &p, int64_t i) {
  if (p.what == kLogprob || (p.what == kPolicy && p.logp)) p.logp[i] = 0.f;
  if (p.what == kPolicy) p.loss[i] = 0.f;
  if (p.what == kPreference) p.row_logp[i] = 0.f;
  if (p.rows) p.rows[i] = {0.f, 0.f, 0.f, 0};
  if (p.row_slopes) p.row_slopes[i] = 0.f;
}

// A warp joins a row's parts: its token's log-probability, the loss, and what the gradient needs.
template <typename TZ> __global__ void __launch_bounds__(kThreads) join_kernel(const TokenArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const bool in = i < p.r;
  const int64_t tok = in ? index_of(p.tokens, p.idx64, i) : -1;
  float w = 0.f;
  const bool live = in && is_live(p, i, tok, w);
  const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
  const float own = live ? widen(z[tok]) : 0.f;
  after_first();
  if (live) {
    RowSum s;
    s.k = -INFINITY;
    for (int q = lane; q < p.parts; q += 32) s.k = fmaxf(s.k, p.sums[i * p.parts + q].x);
    s.k = warp_max(s.k);
    float sum = 0.f;
    for (int q = lane; q < p.parts; q += 32) {
      const float2 a = p.sums[i * p.parts + q];
      sum += a.y * ex2(a.x - s.k);
    }
    s.rest = warp_sum(sum);
    s.far = !(fabsf(s.k) < kFar && s.rest < INFINITY);
    if (s.far) far_sums(p, z, tok, own, s);   // exponents beyond +-kFar, infinities or NaN
    s.y = own_exponent(p, s, own);
    finish_row(p, i, s, w, lane == 0);
  } else if (in && lane == 0) {
    finish_dead_row(p, i);
  }
  follow_early();
}

// ---------------------------------------------------------------------------------------------- rows held in registers
// Rows are read once: their vectors stay in the threads' registers, 16 each, from the sum to the gradient.

// Of short rows a warp holds ROWS, 16 / ROWS vectors of each a lane.  What is computed of a row but once, lane j does for row j (modulo ROWS): that
// costs as much as all the exponentials of 500 logits.
template <typename TZ, int ROWS> __global__ void __launch_bounds__(kThreads, 5) short_kernel(const __grid_constant__ TokenArgs p) {
  constexpr int N = Vec<TZ>::N, V = kVectors / ROWS;
  const int lane = threadIdx.x & 31, j0 = lane % ROWS;
  const int64_t first = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * ROWS, i = first + j0;   // this lane's row
  if (first >= p.r) return;
  const bool in = i < p.r;
  const int64_t tok = in ? index_of(p.tokens, p.idx64, i) : -1;
  float w = 0.f;
  const bool live = in && is_live(p, i, tok, w);
  const TZ *z = static_cast<const TZ *>(p.z) + first * p.ldz;
  TZ *dz = p.dz && p.what == kPolicy ? static_cast<TZ *>(p.dz) + first * p.lddz : nullptr;
  const float own = live ? widen(z[j0 * p.ldz + tok]) : 0.f;
  const uint32_t lives = __ballot_sync(0xffffffffu, live);
  // of row j: whole vectors [begin, end), the element before or behind them that is this lane's, or -1
  const auto pad_of = [&](int j) { return (int)(((uint32_t)reinterpret_cast<uintptr_t>(z) + (uint32_t)j * (uint32_t)p.ldz * (uint32_t)sizeof(TZ) & 15) / sizeof(TZ)); };
  const auto end_of = [&](int pad) { return (int)(((uint32_t)p.v + pad) / N); };
  const auto edge_of = [&](int pad) {
    const int end = end_of(pad);
    if (lane < N) return pad > 0 && lane >= pad && lane < p.v + pad ? lane - pad : -1;
    const int c = end * N + lane - N - pad;
    return lane < 2 * N && end >= (pad > 0) && c < p.v ? c : -1;
  };
  Vec<TZ> a[ROWS][V];
  float edges[ROWS];
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const int pad = pad_of(j), begin = pad > 0, count = end_of(pad) - begin - lane;
    const uint4 *from = reinterpret_cast<const uint4 *>(z + j * p.ldz - pad) + begin + lane;
    const bool there = lives >> j & 1;
#pragma unroll
    for (int u = 0; u < V; ++u) {
      a[j][u] = all_least<TZ>();
      if (there && 32 * u < count) a[j][u].w = __ldcs(from + 32 * u);
    }
    const int edge = edge_of(pad);
    edges[j] = there && edge >= 0 ? widen(z[j * p.ldz + edge]) : -INFINITY;
  }
  RowSum s;
  s.k = s.rest = 0.f;
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const int pad = pad_of(j), begin = pad > 0, count = end_of(pad) - begin - lane;
    const int t = __shfl_sync(0xffffffffu, (int)tok, j);   // (of a live row it is below 2^31)
    if (!(lives >> j & 1)) continue;
    const int slot = t + pad, at = slot / N - begin - lane;   // the token's vector, as this lane counts
    if (at >= 0 && at < count && at % 32 == 0) {
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (at == 32 * u) strike(a[j][u], 1u << (slot % N));
    }
    if (edge_of(pad) == t) edges[j] = -INFINITY;
    const float k = warp_max(fmaxf(frame_of(fmaxf(edges[j], top_of<V>(a[j])), p.scale), -kFar));
    const Val<2> shift = all<2>(-k), by = all<2>(p.scale);
    Val<2> sum{ex2(fmaf(edges[j], p.scale, -k)), 0.f};
#pragma unroll
    for (int u = 0; u < V; ++u) {
      if (32 * u >= count) break;
#pragma unroll
      for (int q = 0; q < Vec<TZ>::P; ++q) {
        Val<2> y = fma(pair(a[j][u], q), by, shift);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        sum = add(sum, y);
      }
    }
    const float rest = warp_sum(sum.x + sum.y);
    if (j0 == j) {
      s.k = k;
      s.rest = rest;
    }
  }
  s.far = live && !(fabsf(s.k) < kFar && s.rest < INFINITY);
  const uint32_t fars = __ballot_sync(0xffffffffu, s.far);
#pragma unroll 1
  for (int j = 0; j < ROWS; ++j)
    if (fars >> j & 1) {
      RowSum f{};
      far_sums(p, z + j * p.ldz, __shfl_sync(0xffffffffu, tok, j), __shfl_sync(0xffffffffu, own, j), f);
      if (j0 == j) {
        s.k = f.k;
        s.rest = f.rest;
      }
    }
  RowOut o{0.f, 0.f, 0.f, 0};
  if (live) {
    s.y = own_exponent(p, s, own);
    o = finish_row(p, i, s, w, lane < ROWS);
  } else if (in && lane < ROWS) {
    finish_dead_row(p, i);
  }
  if (!dz) return;
  const float my_lift = lifted(o);
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    if (first + j >= p.r) break;
    const float lift = __shfl_sync(0xffffffffu, my_lift, j), k = __shfl_sync(0xffffffffu, o.k, j), by_all = __shfl_sync(0xffffffffu, o.factor, j), at_token = __shfl_sync(0xffffffffu, o.own, j);
    const int t = (lives >> j & 1) ? __shfl_sync(0xffffffffu, (int)tok, j) : -1;
    const bool far = fars >> j & 1, still = by_all == 0.f;   // (not for a NaN)
    const TZ *row = z + j * p.ldz;
    TZ *drow = dz + j * p.lddz;
    const int pad = pad_of(j), begin = pad > 0, end = end_of(pad), count = end - begin - lane, edge = edge_of(pad);
    const auto turned = [&](float x) { return still ? 0.f : -by_all * ex2(far ? fmaf(x - k, p.scale, lift) : fmaf(x, p.scale, -k)); };
    if (((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(drow)) & 15) == 0 && !far) {
      uint4 *to = reinterpret_cast<uint4 *>(drow - pad) + begin + lane;
      const Val<2> shift = all<2>(-k), by = all<2>(p.scale), factor = all<2>(-by_all);
#pragma unroll
      for (int u = 0; u < V; ++u) {
        if (32 * u >= count) break;
        if (still) {
          a[j][u].w = make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
          for (int q = 0; q < Vec<TZ>::P; ++q) {
            Val<2> y = fma(pair(a[j][u], q), by, shift);
            y.x = ex2(y.x);
            y.y = ex2(y.y);
            set_pair(a[j][u], q, mul(y, factor));
          }
        }
        __stcs(to + 32 * u, a[j][u].w);
      }
      if (t >= 0) {   // by the lane that wrote over it
        const int at = (t + pad) / N - begin - lane;
        if (at >= 0 && at < count && at % 32 == 0) narrow(drow + t, at_token);
      }
    } else {
      for (int c = begin * N - pad + lane; c < end * N - pad; c += 32) narrow(drow + c, c == t ? at_token : turned(still ? 0.f : widen(row[c])));
    }
    if (edge >= 0) narrow(drow + edge, edge == t ? at_token : turned(edges[j]));
  }
}

// A CTA or a cluster of CTAs holds a longer row.  The warps' sums meet in one exchange.

template <typename TZ, int THREADS, bool CLUSTER> __global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 640 / THREADS) hold_kernel(const __grid_constant__ TokenArgs p) {
  constexpr int N = Vec<TZ>::N, W = THREADS / 32, kShares = W * (CLUSTER ? kMostRanks : 1);
  __shared__ float2 share[kShares];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ranks = CLUSTER ? p.ranks : 1;
  const int64_t i = CLUSTER ? blockIdx.x / ranks : blockIdx.x;
  const int rank = CLUSTER ? (int)(blockIdx.x - i * ranks) : 0;
  if (CLUSTER) cluster_arrive(false);   // every CTA of the cluster runs before anybody writes into its shared memory
  const int64_t tok = index_of(p.tokens, p.idx64, i);
  const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
  TZ *dz = p.dz && p.what == kPolicy ? static_cast<TZ *>(p.dz) + i * p.lddz : nullptr;
  // whole vectors of the row, [v0, v0 + count) this CTA's; what lies before and behind them goes to the first and last CTA, an element a thread
  const int pad = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(TZ)), begin = pad > 0, end = (int)(((uint32_t)p.v + pad) / N), per = (max(end - begin, 0) + ranks - 1) / ranks;
  const int v0 = begin + min(rank * per, max(end - begin, 0)), left = max(0, min(per, end - v0)), count = left - tid;
  int64_t edge = -1;
  if (rank == 0 && pad > 0 && tid < N && tid >= pad && tid < p.v + pad) edge = tid - pad;
  if (rank == ranks - 1 && tid >= N && tid < 2 * N && end >= begin) {
    const int64_t c = (int64_t)end * N + tid - N - pad;
    if (c < p.v) edge = c;
  }
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
  const uint4 *from = reinterpret_cast<const uint4 *>(z - pad) + v0 + tid;
  uint4 *to = reinterpret_cast<uint4 *>(dz - pad) + v0 + tid;   // used where z and dz lie together
  const int64_t c0 = (int64_t)v0 * N - pad, c1 = c0 + (int64_t)left * N;   // the elements of the CTA's whole vectors
  float w;
  if (!is_live(p, i, tok, w)) {
    if (CLUSTER) cluster_wait();
    if (tid == 0 && rank == 0) finish_dead_row(p, i);
    if (!dz) return;
    if (together)
      for (int j = 0; j < count; j += THREADS) __stcs(to + j, make_uint4(0, 0, 0, 0));
    else
      for (int64_t c = c0 + tid; c < c1; c += THREADS) narrow(dz + c, 0.f);
    if (edge >= 0) narrow(dz + edge, 0.f);
    return;
  }
  Vec<TZ> a[kVectors];
#pragma unroll
  for (int u = 0; u < kVectors; ++u) {
    a[u] = all_least<TZ>();
    if (THREADS * u < count) a[u].w = __ldcs(from + THREADS * u);
  }
  const float own = widen(z[tok]), e = edge >= 0 && edge != tok ? widen(z[edge]) : -INFINITY;
  const int64_t slot = tok + pad, at = slot / N - v0 - tid;   // the token's vector, as this thread counts
  const bool mine = at >= 0 && at < count && at % THREADS == 0;
  if (mine) {
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
      if (at == THREADS * u) strike(a[u], 1u << (slot % N));
  }
  RowSum s;
  const float k = warp_max(fmaxf(frame_of(fmaxf(e, top_of<kVectors>(a)), p.scale), -kFar));
  {
    const Val<2> shift = all<2>(-k), by = all<2>(p.scale);
    Val<2> sum{ex2(fmaf(e, p.scale, -k)), 0.f};
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
      if (THREADS * u >= count) break;
#pragma unroll
      for (int q = 0; q < Vec<TZ>::P; ++q) {
        Val<2> y = fma(pair(a[u], q), by, shift);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        sum = add(sum, y);
      }
    }
    s.k = k;
    s.rest = warp_sum(sum.x + sum.y);
  }
  if (CLUSTER) {
    cluster_wait();
    if (lane < ranks) *cooperative_groups::this_cluster().map_shared_rank(share + rank * W + warp, lane) = make_float2(s.k, s.rest);
    cluster_arrive(true);
    cluster_wait();
  } else {
    if (lane == 0) share[warp] = make_float2(s.k, s.rest);
    __syncthreads();
  }
  {   // a share a lane (of 64 two), in one order for all
    float2 q[(kShares + 31) / 32];
#pragma unroll
    for (int j = 0; j < (kShares + 31) / 32; ++j) {
      q[j] = lane + 32 * j < W * ranks ? share[lane + 32 * j] : make_float2(-INFINITY, 0.f);
      s.k = j == 0 ? q[j].x : fmaxf(s.k, q[j].x);
    }
    s.k = warp_max(s.k);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < (kShares + 31) / 32; ++j)
      if (lane + 32 * j < W * ranks) sum += q[j].y * ex2(q[j].x - s.k);
    s.rest = warp_sum(sum);
  }
  s.far = !(fabsf(s.k) < kFar && s.rest < INFINITY);   // the same for all
  if (s.far) {
    far_sums(p, z, tok, own, s);
    if (CLUSTER) {   // (dz may be z)
      cluster_arrive(false);
      cluster_wait();
    } else {
      __syncthreads();
    }
  }
  s.y = own_exponent(p, s, own);
  RowOut o = finish_row(p, i, s, w, tid == 0 && rank == 0);
  if (!dz) return;
  const bool still = o.factor == 0.f;   // (not for a NaN)
  const float lift = lifted(o);
  const auto turned = [&](float x) { return still ? 0.f : -o.factor * ex2(s.far ? fmaf(x - o.k, p.scale, lift) : fmaf(x, p.scale, -o.k)); };
  if (together && !s.far) {
    const Val<2> shift = all<2>(-o.k), by = all<2>(p.scale), factor = all<2>(-o.factor);
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
      if (THREADS * u >= count) break;
      if (still) {
        a[u].w = make_uint4(0, 0, 0, 0);
      } else {
#pragma unroll
        for (int q = 0; q < Vec<TZ>::P; ++q) {
          Val<2> y = fma(pair(a[u], q), by, shift);
          y.x = ex2(y.x);
          y.y = ex2(y.y);
          set_pair(a[u], q, mul(y, factor));
        }
      }
      __stcs(to + THREADS * u, a[u].w);
    }
    if (mine) narrow(dz + tok, o.own);   // by the thread that wrote over it
  } else {
    for (int64_t c = c0 + tid; c < c1; c += THREADS) narrow(dz + c, c == tok ? o.own : turned(still ? 0.f : widen(z[c])));
  }
  if (edge >= 0) narrow(dz + edge, edge == tok ? o.own : turned(e));
}

template <typename TZ, int THREADS, bool CLUSTER> cudaError_t launch_hold(const TokenArgs &p, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.r * p.ranks));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim = {(unsigned)p.ranks, 1, 1};
  if (CLUSTER) { cfg.attrs = &at; cfg.numAttrs = 1; }
  return cudaLaunchKernelEx(&cfg, hold_kernel<TZ, THREADS, CLUSTER>, p);
}
template <typename TZ, int ROWS> cudaError_t launch_short(const TokenArgs &p, cudaStream_t s) {
  short_kernel<TZ, ROWS><<<(unsigned)ceil_div(p.r, kWarps * ROWS), kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

__device__ __forceinline__ int64_t bound(const TokenArgs &p, int64_t j) { return min(max(index_of(p.bounds, p.bounds64, j), (int64_t)0), p.r); }

constexpr int kPairThreads = 512, kPairWarps = kPairThreads / 32;

// A CTA takes a pair: its sequences' sums in 64 bits, the loss, and the slope of each of its rows.
__global__ void __launch_bounds__(kPairThreads) pair_kernel(const TokenArgs p) {
  __shared__ double sums[2][kPairWarps];
  __shared__ int64_t counts[2][kPairWarps];
  __shared__ float slopes[2];
  const int warp = threadIdx.x >> 5;
  after_first();
  for (int64_t q = blockIdx.x; q < p.pairs; q += gridDim.x) {
    const float w = p.weight ? p.weight[q] : 1.f;
    const int64_t cut[3] = {bound(p, 2 * q), bound(p, 2 * q + 1), bound(p, 2 * q + 2)};
    __syncthreads();
    for (int k = 0; k < 2; ++k) {
      double s = 0.;
      int64_t n = 0;
      for (int64_t i = cut[k] + threadIdx.x; i < cut[k + 1]; i += kPairThreads) {
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
    if (threadIdx.x == 0) {
      double l[2], by[2];
      for (int k = 0; k < 2; ++k) {
        int64_t n = 0;
        l[k] = 0.;
        for (int i = 0; i < kPairWarps; ++i) {
          l[k] += sums[k][i];
          n += counts[k][i];
        }
        by[k] = p.average ? 1. / (double)max(n, (int64_t)1) : 1.;
        l[k] *= by[k];
        if (p.logp) p.logp[2 * q + k] = (float)l[k];
        if (p.ref_logp) l[k] -= (double)p.ref_logp[2 * q + k];
      }
      const double m = (double)p.beta * (l[0] - l[1]), e = exp(-fabs(m)), small = e / (1. + e);
      const double up = log1p(e) + fmax(-m, 0.), down = log1p(e) + fmax(m, 0.);                          // -log sigmoid(m), -log sigmoid(-m)
      const double at_minus = m >= 0. ? small : 1. / (1. + e), at = m >= 0. ? 1. / (1. + e) : small;     // sigmoid(-m), sigmoid(m)
      const double eps = (double)p.smoothing;
      if (p.loss) p.loss[q] = w == 0.f ? 0.f : (float)((double)w * ((eps < 1. ? (1. - eps) * up : 0.) + (eps > 0. ? eps * down : 0.)));   // (either may be infinite)
      const double slope = w == 0.f ? 0. : (double)w * (double)p.beta * (eps * at - (1. - eps) * at_minus);
      slopes[0] = (float)(slope * by[0]);
      slopes[1] = (float)(-slope * by[1]);
    }
    if (!p.row_slopes) continue;
    __syncthreads();
    for (int k = 0; k < 2; ++k)
      for (int64_t i = cut[k] + threadIdx.x; i < cut[k + 1]; i += kPairThreads) p.row_slopes[i] = slopes[k];
  }
  follow_early();
}

// A warp writes a part of a row's gradient.
template <typename TZ> __global__ void __launch_bounds__(kThreads) turn_kernel(const TokenArgs p) {
  constexpr int N = Vec<TZ>::N;
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5), i = task / p.parts;
  if (i >= p.r) return;
  const int64_t tok = index_of(p.tokens, p.idx64, i);
  const TZ *z = static_cast<const TZ *>(p.z) + i * p.ldz;
  TZ *dz = static_cast<TZ *>(p.dz) + i * p.lddz;
  const WarpPart<TZ> part(z, p.v, (int)(task - i * p.parts), p.per);
  const int64_t slot = tok >= 0 && tok < p.v ? tok + part.pad : -1;
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
  after_first();
  RowOut o = p.rows ? p.rows[i] : RowOut{};
  if (p.row_slopes) {
    const float slope = p.row_slopes[i];
    const bool stays = slope == 0.f || slot < 0;   // without a token whatever the sequence's slope is, a NaN too
    o.factor = stays ? 0.f : o.factor * slope;
    o.own = stays ? 0.f : o.own * slope;
  }
  const bool still = o.factor == 0.f;   // (not for a NaN)
  const float lift = lifted(o);
  const auto turned = [&](float x) { return still ? 0.f : -o.factor * ex2(o.far ? fmaf(x - o.k, p.scale, lift) : fmaf(x, p.scale, -o.k)); };
  const auto element = [&](int64_t s) { narrow(dz + s - part.pad, s == slot ? o.own : turned(still ? 0.f : widen(z[s - part.pad]))); };
  if (together && !o.far) {
    const uint4 *from = reinterpret_cast<const uint4 *>(z - part.pad) + part.w0 + lane;
    uint4 *to = reinterpret_cast<uint4 *>(dz - part.pad) + part.w0 + lane;
    const int count = part.w1 - part.w0 - lane;
    const Val<2> shift = all<2>(-o.k), by = all<2>(p.scale), factor = all<2>(-o.factor);
    const int64_t at = slot / N - part.w0 - lane;
    constexpr int kBatch = 8;
#pragma unroll
    for (int h = 0; h < kVectors; h += kBatch) {
      Vec<TZ> a[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (!still && 32 * (h + u) < count) a[u].w = __ldcs(from + 32 * (h + u));
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (32 * (h + u) >= count) break;
        if (still) {
          a[u].w = make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < Vec<TZ>::P; ++e) {
            Val<2> y = fma(pair(a[u], e), by, shift);
            y.x = ex2(y.x);
            y.y = ex2(y.y);
            set_pair(a[u], e, mul(y, factor));
          }
        }
        __stcs(to + 32 * (h + u), a[u].w);
      }
    }
    if (part.edge >= 0) element(part.edge);
    __syncwarp();
    if (slot >= 0 && at >= 0 && at < count && at % 32 == 0) narrow(dz + tok, o.own);   // by the lane that wrote over it
  } else {
    for (int64_t s = (int64_t)part.w0 * N + lane; s < (int64_t)part.w1 * N; s += 32) element(s);
    if (part.edge >= 0) element(part.edge);
  }
}

constexpr int64_t kMost = ((int64_t)1 << 31) - 1024;
bool sizes_ok(int64_t r, int64_t v) { return r >= 0 && r < ((int64_t)1 << 28) && v >= 1 && v < kMost && r * ceil_div(v, 4 * kPart) < kMost; }

float scale_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }
bool common_ok(int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t logits_type, int32_t index_type, float temperature) {
  return sizes_ok(r, v) && ldz >= v && lddz >= v && is_type(logits_type) && is_index(index_type) && temperature > 0.f && std::isfinite(temperature) &&
         std::isfinite(scale_of(temperature));
}

int64_t parts_of(int64_t v, int32_t logits_type) {
  const int64_t n = 16 / type_bytes(logits_type);
  return ceil_div(ceil_div(v + n - 1, n), kPart);
}

TokenArgs common(int32_t what, const void *z, const void *tokens, void *dz, int64_t r, int64_t v, int64_t ldz, int64_t lddz, int32_t logits_type,
                 int32_t index_type, float temperature, void *workspace) {
  TokenArgs p{};
  p.what = what;
  p.z = z; p.tokens = tokens; p.dz = dz;
  p.r = r; p.v = v; p.ldz = ldz; p.lddz = lddz;
  p.scale = scale_of(temperature);
  p.temperature = temperature;
  p.idx64 = index_type == DSGD_I64;
  const int64_t n = 16 / type_bytes(logits_type), vectors = ceil_div(v + n - 1, n);   // of the row on the least fortunate boundary
  p.parts = (int32_t)parts_of(v, logits_type);
  p.per = (int32_t)ceil_div(vectors, p.parts);
  RowOut *rows = static_cast<RowOut *>(workspace);
  p.rows = dz ? rows : nullptr;
  p.sums = reinterpret_cast<float2 *>(rows + r);
  p.row_logp = reinterpret_cast<float *>(p.sums + r * p.parts);
  p.row_slopes = what == kPreference && dz ? p.row_logp + r : nullptr;
  return p;
}

bool workspace_ok(const void *workspace, size_t bytes, int64_t r, int64_t v, int64_t pairs) {
  const size_t need = dsgd_token_workspace_bytes(r, v, pairs);
  return need == 0 || (workspace && bytes >= need && !(reinterpret_cast<uintptr_t>(workspace) & 15));
}

// Whether what is written lies apart from what other threads may still read.
bool apart(const float *loss, const float *logp, std::initializer_list<const float *> inputs) {
  for (const float *x : inputs)
    if (x && (x == loss || x == logp)) return false;
  return !loss || loss != logp;
}

// Which form a call takes: a row that 128 threads hold is read once whatever is wanted of it, a longer one where its gradient follows from
// its own sum, as long as a cluster holds it, or where there are so few that one launch instead of two is what counts (256 rows of 32000
// bf16: 7.6 us in two, 6.1 in one).  Other rows are streamed.
template <typename TZ> cudaError_t run(TokenArgs p, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  const unsigned parts = (unsigned)ceil_div(p.r * p.parts, kWarps);
  const int64_t whole = p.v / Vec<TZ>::N;
  p.ranks = 1;
  while (p.ranks < kMostRanks && whole > (int64_t)kThreads * kVectors * p.ranks) p.ranks *= 2;
  const bool turns = p.dz && p.what == kPolicy && whole <= (int64_t)256 * kVectors * kMostRanks;
  if (turns) p.rows = nullptr;
  if (p.r == 0 || (p.what == kPreference && p.pairs == 0)) {
  } else if (whole <= kPart) {   // several rows a warp where there are enough of them to keep all SMs at work
    const bool many = p.r >= 32 * (int64_t)sm_count();
    e = many && whole <= kPart / 4 ? launch_short<TZ, 4>(p, s) : many && whole <= kPart / 2 ? launch_short<TZ, 2>(p, s) : launch_short<TZ, 1>(p, s);
  } else if (whole <= 64 * kVectors) {
    e = launch_hold<TZ, 64, false>(p, s);
  } else if (whole <= kThreads * kVectors) {
    e = launch_hold<TZ, kThreads, false>(p, s);
  } else if ((turns || p.r * p.ranks <= 5 * (int64_t)sm_count()) && whole <= (int64_t)kThreads * kVectors * kMostRanks) {
    e = launch_hold<TZ, kThreads, true>(p, s);
  } else if (turns) {
    e = launch_hold<TZ, 256, true>(p, s);
  } else {
    sum_kernel<TZ><<<parts, kThreads, 0, s>>>(p);
    e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_after(join_kernel<TZ>, p, dim3((unsigned)ceil_div(p.r, kWarps)), kThreads, 0, s);
  }
  if (e == cudaSuccess && p.what == kPreference && p.pairs > 0) e = launch_after(pair_kernel, p, dim3((unsigned)std::min<int64_t>(p.pairs, 1 << 20)), kPairThreads, 0, s);
  if (e == cudaSuccess && p.dz && p.r > 0 && !turns) e = launch_after(turn_kernel<TZ>, p, dim3(parts), kThreads, 0, s);
  return e;
}

ceca_status_t run(const TokenArgs &p, int32_t logits_type, void *stream) {
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return (logits_type == DSGD_F32 ? run<float>(p, s) : run<bf16>(p, s)) == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
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
  if (!apart(loss, logp, {old_logp, advantage, ref_logp})) return CECA_ERR_UNSUPPORTED;
  TokenArgs p = common(kPolicy, z, tokens, dz, r, v, ldz, lddz, logits_type, index_type, temperature, workspace);
  p.old_logp = old_logp; p.advantage = advantage; p.ref_logp = ref_logp; p.weight = weight; p.loss = loss; p.logp = logp;
  p.low = 1.f - clip_low; p.high = 1.f + clip_high; p.kl = kl;
  return run(p, logits_type, stream);
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
  if (pairs > 0 && !apart(loss, logp, {ref_logp})) return CECA_ERR_UNSUPPORTED;
  TokenArgs p = common(kPreference, z, tokens, dz, r, v, ldz, lddz, logits_type, index_type, temperature, workspace);
  p.bounds = bounds; p.bounds64 = bounds_type == DSGD_I64;
  p.ref_logp = ref_logp; p.weight = weight; p.loss = loss; p.logp = logp; p.pairs = pairs;
  p.beta = beta; p.smoothing = smoothing; p.average = average != 0;
  if (pairs == 0) {   // a gradient of 0, for which nothing is summed
    p.rows = nullptr;
    p.row_slopes = nullptr;
  }
  return run(p, logits_type, stream);
}

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" size_t dsgd_token_workspace_bytes(int64_t r, int64_t v, int64_t pairs) {
  if (!sizes_ok(r, v) || pairs < 0 || pairs >= ((int64_t)1 << 27) || (pairs == 0 && v <= 4 * kThreads * kVectors)) return 0;   // (rows of so many are held)
  return (size_t)r * (sizeof(RowOut) + sizeof(float2) * (size_t)parts_of(v, DSGD_F32) + 2 * sizeof(float)) + 16;
}

extern "C" ceca_status_t dsgd_token_logprob(const void *z, const void *tokens, float *logp, int64_t r, int64_t v, int64_t ldz, int32_t logits_type,
                                            int32_t index_type, float temperature, void *workspace, size_t workspace_bytes, void *stream) {
  if (!common_ok(r, v, ldz, v, logits_type, index_type, temperature)) return CECA_ERR_INVALID_ARG;
  if (r == 0) return CECA_OK;
  if (!z || !tokens || !logp) return CECA_ERR_INVALID_ARG;
  if (!workspace_ok(workspace, workspace_bytes, r, v, 0)) return CECA_ERR_WORKSPACE;
  TokenArgs p = common(kLogprob, z, tokens, nullptr, r, v, ldz, v, logits_type, index_type, temperature, workspace);
  p.logp = logp;
  return run(p, logits_type, stream);
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
