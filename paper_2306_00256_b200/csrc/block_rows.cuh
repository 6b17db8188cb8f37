// Internal: the end of a block and the start of the next, and its gradient, for rows that a group of threads holds in registers.
//
// A group takes every so-many-th row of an agent.  The next rows are copied to a ring in shared memory while one is computed on, so that loads are always
// under way; the weights (of the gradient in shared memory), and the sums of their gradients, stay in registers.
//
// Forward: two sums over the group a row, y^2 and h_out^2.  Gradient, with q = s g w_post yn (what the block added), f = w_pre du and t = dh_out + r f:
// the three sums A = hn f, B = q t, C = q hn at once, then m = A / d, dh = t - r m hn and mean(yn e) = (B - r m C) / d.
//
// Bytes and instructions bound these kernels together: some 30 instructions a channel forward, 50 in the gradient.  Of the measured copy rate they reach
// (8 x 4096 x 2048, silu gates) 0.82 forward and 0.90 in the gradient in bf16, 0.85 and 0.86 with an fp32 stream, 0.85 and 0.69 where 8 bits are written
// and read; rows of 771 fp32 channels 0.78 and 0.82, of 2047 bf16 channels, read and written one by one, 0.56 and 0.58, of 64 bf16 channels, four rows a
// warp, 0.79 and 0.77 (0.22 and 0.26 with a warp for each).
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "block_norm.cuh"
#include "tma.h"

namespace ceca {

constexpr int kKept = 2;      // besides DSGD_F32 and DSGD_BF16
constexpr int kAnyType = -1;  // of a template: the call says which
// What a kernel is compiled for: the whole of the formulas without a gate or with one of the two, or any part of them, as the call says.  (Branches
// between the parts keep loads and products apart that could overlap: the gradient of 8 x 4096 x 2048 bf16 takes 183 us whole, and 206 without dh_out, a fifth
// less to read and write.  A model has few blocks of that kind.)
enum Parts : int { kPlain, kSigmoid, kSilu, kAnyParts };

__device__ __forceinline__ void copy_16(uint32_t to, const void *from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_16(uint32_t to, const void *from, int bytes) {   // zeros behind the first `bytes`
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_8(uint32_t to, const void *from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy_4(uint32_t to, const void *from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_but(int behind) {   // waits for all groups but the last `behind`
  switch (behind) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
  }
}

// The channels of a thread of a group of G, eight in each of its passes: V = 8: eight neighbours, a 16-byte word of bf16; V = 4: twice four, words of fp32;
// V = 1: every G-th one, for rows on any boundary.  They are computed on in pairs.
template <int G, int V> __device__ __forceinline__ int channel(int rank, int j, int e) {
  return V == 8 ? 8 * (rank + G * j) + e : V == 4 ? 4 * (rank + G * (2 * j + e / 4)) + e % 4 : rank + G * (8 * j + e);
}
struct Pairs8 {
  Val<2> v[4];
};

// A place in shared memory for a row of a tensor, or for a kept row, and its copy and reading.  V = 8 and 4: each warp copies what it will read, in
// whole sectors.  V = 1: the group copies the 16-byte words that the row touches (of the first and last one the bytes inside the row
// count), and must meet between copying and reading.
template <int G, int PASSES, int V> struct Place {
  static constexpr int kEights = G * PASSES;
  // types: DSGD_F32, DSGD_BF16, kKept
  __host__ __device__ static constexpr int room(int64_t d, int32_t type) {
    if (V == 1) return type == kKept ? (int)kept_row_bytes(d) : (int)((d * (type == DSGD_BF16 ? 2 : 4) + 47) / 16 * 16);
    return type == kKept ? (9 * kEights + 15) / 16 * 16 : (type == DSGD_BF16 ? 16 : 32) * kEights;
  }
  __device__ static void copy(uint32_t to, const uint8_t *from, int32_t type, int d, int rank) {
    constexpr int kLanes = G < 32 ? G : 32;   // that copy together
    const int lane = rank % kLanes;
    if (V == 8) {   // bf16, or kept: its exponents behind the whole numbers
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        const int at = rank + G * j;
        if (8 * at >= d) continue;
        if (type == kKept) {
          copy_8(to + 8 * at, from + 8 * at);
          if (at % 16 == 0) copy_4(to + 8 * kEights + at / 4, from + d + at / 4);   // (a word of exponents: d is a multiple of 8)
        } else {
          copy_16(to + 16 * at, from + 16 * at);
        }
      }
    } else if (V == 4) {   // as it lies in memory; a warp's channels of a half pass are 128 neighbours
      const int c0 = 4 * (rank - lane);
      if (type == DSGD_F32) {
#pragma unroll
        for (int k = 0; k < 2 * PASSES; ++k) {
          const int c = c0 + 4 * (G * k + lane);
          if (c < d) copy_16(to + 4 * c, from + 4 * c);
        }
      } else if (type == DSGD_BF16) {
#pragma unroll
        for (int j = 0; j < PASSES; ++j) {
          const int c = c0 + 4 * G * (2 * j + lane / (kLanes / 2)) + 8 * (lane % (kLanes / 2));
          if (c < d) copy_16(to + 2 * c, from + 2 * c);
        }
      } else {
        const int c = c0 + 4 * G * (lane / (kLanes / 4)) + 16 * (lane % (kLanes / 4)), e = c0 / kBlock8 + G / 8 * lane;   // (the last copy may take exponents with it)
        if (lane < kLanes / 2 * PASSES && c < d) copy_16(to + c, from + c);
        if (lane < (G < 32 ? 1 : 2 * PASSES) && e * kBlock8 < d) copy_4(to + d + e, from + d + e);
      }
    } else {
      const int pad = (int)(reinterpret_cast<uintptr_t>(from) & 15), end = pad + (type == kKept ? (int)kept_row_bytes(d) : d * (type == DSGD_BF16 ? 2 : 4));
      from -= pad;
      for (int at = 16 * rank; at < end; at += 16 * G) copy_16(to + at, from + at, min(16, end - at));
    }
  }
  // the eight channels of pass j; zeros outside the row
  __device__ static Pairs8 read(const uint8_t *place, int pad, int32_t type, int d, int rank, int j) {
    Pairs8 r{};
    if (V == 8) {
      const int at = rank + G * j;
      if (8 * at >= d) return r;
      if (type == kKept) {
        const uint2 q = reinterpret_cast<const uint2 *>(place)[at];
        const Val<2> step = all<2>(step8(place[8 * kEights + at / 4]));
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = mul(whole_numbers(i < 2 ? q.x : q.y, 2 * (i & 1)), step);
      } else {
        const uint4 w = reinterpret_cast<const uint4 *>(place)[at];
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = unpack_bf16((&w.x)[i]);
      }
    } else if (V == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int at = rank + G * (2 * j + k);
        if (4 * at >= d) continue;
        if (type == kKept) {
          const uint32_t q = reinterpret_cast<const uint32_t *>(place)[at];
          const Val<2> step = all<2>(step8(place[d + at / 8]));
          r.v[2 * k] = mul(whole_numbers(q, 0), step);
          r.v[2 * k + 1] = mul(whole_numbers(q, 2), step);
        } else if (type == DSGD_BF16) {
          const uint2 w = reinterpret_cast<const uint2 *>(place)[at];
          r.v[2 * k] = unpack_bf16(w.x);
          r.v[2 * k + 1] = unpack_bf16(w.y);
        } else {
          const float4 a = reinterpret_cast<const float4 *>(place)[at];
          r.v[2 * k] = {a.x, a.y};
          r.v[2 * k + 1] = {a.z, a.w};
        }
      }
    } else {
      place += pad;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = channel<G, V>(rank, j, e);
        float x = 0.f;
        if (c < d) {
          if (type == kKept) x = (float)(int8_t)place[c] * step8(place[d + c / kBlock8]);
          else x = type == DSGD_BF16 ? widen(reinterpret_cast<const bf16 *>(place)[c]) : reinterpret_cast<const float *>(place)[c];
        }
        (e & 1 ? r.v[e / 2].y : r.v[e / 2].x) = x;
      }
    }
    return r;
  }
  // writes eight channels of a row
  __device__ static void write(void *row, int32_t type, const Pairs8 &x, int d, int rank, int j) {
    if (V == 8) {
      const int at = rank + G * j;
      if (8 * at < d) static_cast<uint4 *>(row)[at] = make_uint4(pack_bf16(x.v[0]), pack_bf16(x.v[1]), pack_bf16(x.v[2]), pack_bf16(x.v[3]));
    } else if (V == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int at = rank + G * (2 * j + k);
        if (4 * at >= d) continue;
        const Val<2> a = x.v[2 * k], b = x.v[2 * k + 1];
        if (type == DSGD_BF16) static_cast<uint2 *>(row)[at] = make_uint2(pack_bf16(a), pack_bf16(b));
        else static_cast<float4 *>(row)[at] = make_float4(a.x, a.y, b.x, b.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = channel<G, V>(rank, j, e);
        if (c < d) store(row, type, c, e & 1 ? x.v[e / 2].y : x.v[e / 2].x);
      }
    }
  }
  // Keeps a row in 8 bits; whole warps call it.  x: the thread's channels; with V = 1 it takes eight neighbours from the row's place instead, so that it
  // writes them together and asks three lanes, not all, for their largest.
  __device__ static void keep(uint8_t *row, const Pairs8 *x, const uint8_t *place, int pad, int32_t type, int d, int rank) {
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      if (V == 4) {
        keep_fours(row, x[j], d, rank, j);
      } else if (V == 8) {
        keep_eight(row, x[j], d, rank + G * j);
      } else {
        const int c = 8 * (rank + G * j);
        Pairs8 r{};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (c + e >= d) continue;
          const float v = type == DSGD_BF16 ? widen(reinterpret_cast<const bf16 *>(place + pad)[c + e]) : reinterpret_cast<const float *>(place + pad)[c + e];
          (e & 1 ? r.v[e / 2].y : r.v[e / 2].x) = v;
        }
        keep_eight(row, r, d, rank + G * j);
      }
    }
    const int from = d + (int)blocks8(d), to = (int)kept_row_bytes(d);   // the bytes behind the exponents, fewer than 16
    if (rank < to - from) row[from + rank] = 0;
    if (G < 16 && rank + G < to - from) row[from + rank + G] = 0;
  }
  __device__ static void keep_eight(uint8_t *row, const Pairs8 &x, int d, int at) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = greatest(most, x.v[i]);
    uint32_t top = __float_as_uint(most);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const bool cut = __any_sync(0xffffffffu, cut8(top));   // of one warp in thirty: a branch, not a choice for each
    if (8 * at >= d) return;
    const uint32_t e = exponent8(top);
    const Val<2> by = all<2>(scale8(e));
    uint2 q = make_uint2(hold_four(x.v[0], x.v[1], by, cut), hold_four(x.v[2], x.v[3], by, cut));
    if (e == 255u) q = make_uint2(0, 0);
    if (V == 8 || 8 * at + 8 <= d) reinterpret_cast<uint2 *>(row)[at] = q;
    else
      for (int c = 8 * at; c < d; ++c) row[c] = (uint8_t)((c & 4 ? q.y : q.x) >> 8 * (c & 3));
    if (at % 4 == 0) row[d + at / 4] = (uint8_t)e;
  }
  __device__ static void keep_fours(uint8_t *row, const Pairs8 &x, int d, int rank, int j) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int at = rank + G * (2 * j + k);
      uint32_t top = __float_as_uint(greatest(greatest(0.f, x.v[2 * k]), x.v[2 * k + 1]));
#pragma unroll
      for (int o = 1; o < 8; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const bool cut = __any_sync(0xffffffffu, cut8(top));
      if (4 * at >= d) continue;
      const uint32_t e = exponent8(top);
      reinterpret_cast<uint32_t *>(row)[at] = e == 255u ? 0 : hold_four(x.v[2 * k], x.v[2 * k + 1], all<2>(scale8(e)), cut);
      if (at % 8 == 0) row[d + at / 8] = (uint8_t)e;
    }
  }
};

// The sum over a group, in one order, the same on all its threads.  `turn` says which of two places is used: consecutive
// sums take the other one, so that one barrier is enough.
__host__ __device__ constexpr int warps_of(int group) { return group <= 32 ? 1 : group / 32; }
template <int G> __device__ __forceinline__ float group_sum(float x, float (*place)[4 * warps_of(G)], int turn) {
  constexpr int W = warps_of(G);
#pragma unroll
  for (int o = (G < 32 ? G : 32) / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (G <= 32) return x;
  const int lane = threadIdx.x & 31;
  if (lane == 0) place[turn][threadIdx.x >> 5] = x;
  __syncthreads();
  x = place[turn][lane % W];   // each lane reads one warp's, and the warps' are summed as the lanes' were
#pragma unroll
  for (int o = W / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// Three sums at once: lanes first share out the numbers (x to lanes 0 to 7, y to 8 to 15, z to 16 to 23; 24 to 31 have a zero), so that most steps move one.
template <int G> __device__ __forceinline__ float3 group_sums(float3 v, float (*place)[4 * warps_of(G)], int turn) {
  if (G < 32) return make_float3(group_sum<G>(v.x, place, turn), group_sum<G>(v.y, place, turn), group_sum<G>(v.z, place, turn));
  const int lane = threadIdx.x & 31;
  const bool upper = lane & 16, odd = lane & 8;
  const float a = __shfl_xor_sync(0xffffffffu, upper ? v.x : v.z, 16), b = __shfl_xor_sync(0xffffffffu, upper ? v.y : 0.f, 16);
  const float p = (upper ? v.z : v.x) + a, q = upper ? 0.f : v.y + b;
  float x = (odd ? q : p) + __shfl_xor_sync(0xffffffffu, odd ? p : q, 8);
#pragma unroll
  for (int o = 4; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (G > 32) {
    constexpr int W = warps_of(G);
    if ((lane & 7) == 0) place[turn][4 * (threadIdx.x >> 5) + lane / 8] = x;
    __syncthreads();
    // lane 8 n + w reads number n of warp w (of 16 warps two), and the warps' are summed as the lanes' were
    const int w = lane & 7;
    x = place[turn][4 * (w % W) + lane / 8];
    if (W > 8) x += place[turn][4 * (8 + w) + lane / 8];
#pragma unroll
    for (int o = (W < 8 ? W : 8) / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  }
  return make_float3(__shfl_sync(0xffffffffu, x, 0), __shfl_sync(0xffffffffu, x, 8), __shfl_sync(0xffffffffu, x, 16));
}

__device__ __forceinline__ float total(const Pairs8 &a) {
  const Val<2> s = add(add(a.v[0], a.v[1]), add(a.v[2], a.v[3]));
  return s.x + s.y;
}

// A tensor's rows that a group takes: the next one to copy, and where one lies.
struct Walk {
  const uint8_t *at;
  int64_t hop;
  uint32_t low, low_hop;   // of the row that is computed on
  __device__ Walk(const dsgd_rows_t &x, int64_t agent, int64_t first, int64_t rows, int bytes)
      : at(static_cast<const uint8_t *>(x.at) + place(x, agent, first) * bytes), hop(rows * x.row_stride * bytes), low((uint32_t)reinterpret_cast<uintptr_t>(at)), low_hop((uint32_t)hop) {}
  __device__ Walk(const dsgd_rows_t &x, int64_t row, int64_t rows, int64_t row_bytes)   // a kept tensor's
      : at(static_cast<const uint8_t *>(x.at) + row * row_bytes), hop(rows * row_bytes), low(0), low_hop(0) {}
  __device__ int pad() const { return low & 15; }
  __device__ void next() { low += low_hop; }
};

// A thread's weights, times a number; zeros outside the row and where there are none.
template <int G, int PASSES, int V>
__device__ __forceinline__ void weights(Pairs8 *w, const void *from, int32_t type, int64_t at, float by, int d, int rank) {
  const auto fill = [&](auto *values) {
#pragma unroll
    for (int j = 0; j < PASSES; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = channel<G, V>(rank, j, e);
        (e & 1 ? w[j].v[e / 2].y : w[j].v[e / 2].x) = values && c < d ? by * widen(values[c]) : 0.f;
      }
  };
  if (type == DSGD_BF16) fill(from ? static_cast<const bf16 *>(from) + at : nullptr);
  else fill(from ? static_cast<const float *>(from) + at : nullptr);
}

// Each warp's copy of a row's two statistics, in words of 16 bytes.
__host__ __device__ constexpr int stats_room(int group) { return group <= 32 ? 16 : group / 4; }

#define CECA_TYPES                                                           \
  const int32_t ts = TS == kAnyType ? p.stream_type : TS;                    \
  const int32_t ta = TA == kAnyType ? p.act_type : TA;                       \
  const int sb = ts == DSGD_BF16 ? 2 : 4, ab = ta == DSGD_BF16 ? 2 : 4

template <int G, int PASSES, int V, int TS, int TA, int PARTS>
__global__ void __launch_bounds__(G * groups_of(G), resident_block(G, PASSES)) block_kernel(const __grid_constant__ BlockArgs p) {
  using X = Place<G, PASSES, V>;
  extern __shared__ uint4 ring[];
  __shared__ alignas(16) float sums[2][4 * warps_of(G)];
  constexpr int kGroups = groups_of(G);
  CECA_TYPES;
  const int rank = threadIdx.x % G, group = threadIdx.x / G, width = (int)p.d, d = width;
  const int64_t agent = blockIdx.x / p.part_count, first = (blockIdx.x - agent * p.part_count) * kGroups + group, hop = (int64_t)p.part_count * kGroups;
  constexpr bool kAny = PARTS == kAnyParts;
  const bool y = !kAny || p.y.at != nullptr, gated = kAny ? p.gate.at != nullptr : PARTS != kPlain, u = !kAny || p.w_pre != nullptr, silu = kAny ? p.silu : PARTS == kSilu;
  // a row's places in a stage of the ring, where they can be known by now
  const auto room = [&](int i, int32_t type, bool there) { return V > 1 && !kAny ? there ? X::room(0, type) : 0 : p.room[i]; };
  const int off_y = room(0, ts, true), off_g = off_y + room(1, ta, y), stage_bytes = off_g + room(2, ta, gated);
  uint8_t *mine = reinterpret_cast<uint8_t *>(ring) + (size_t)group * p.stages * stage_bytes;
  const uint32_t mine32 = smem_u32(mine);
  Walk wh(p.h, agent, first, hop, sb), wy(p.y, agent, first, hop, ab), wg(p.gate, agent, first, hop, ab);
  const auto count = [&](int64_t from) { return from < p.t ? (int)((p.t - 1 - from) / hop) + 1 : 0; };
  // groups that share a warp stay together: for as many rows as the first of them has
  const int rows = count(first), rounds = G < 32 ? count(first - group % (32 / (G < 32 ? G : 32))) : rows, ring_bytes = p.stages * stage_bytes;
  int fill = 0, left = rows;   // the place that is filled next, the rows that are not on their way
  const auto bring = [&]() {
    if (--left >= 0) {
      const uint32_t to = mine32 + fill;
      X::copy(to, wh.at, ts, d, rank);
      if (y) X::copy(to + off_y, wy.at, ta, d, rank);
      if (gated) X::copy(to + off_g, wg.at, ta, d, rank);
    }
    wh.at += wh.hop;
    wy.at += wy.hop;
    wg.at += wg.hop;
    fill += stage_bytes;
    if (fill == ring_bytes) fill = 0;
    copies_end();
  };
  for (int i = 0; i + 1 < p.stages; ++i) bring();
  const float scale = p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f, over_d = 1.f / (float)p.d;
  Pairs8 wq[PASSES], wp[PASSES];   // scale w_post, w_pre
  weights<G, PASSES, V>(wq, y ? p.w_post : nullptr, p.weights_type, agent * p.w_post_stride, scale, d, rank);
  weights<G, PASSES, V>(wp, u ? p.w_pre : nullptr, p.weights_type, agent * p.w_pre_stride, 1.f, d, rank);
  const auto norm = [&](const Pairs8 *a, int turn) {
    const auto squares = [&](float unit) {
      Pairs8 s{};
#pragma unroll
      for (int j = 0; j < PASSES; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const Val<2> v = unit == 1.f ? a[j].v[k] : mul(a[j].v[k], all<2>(unit));
          s.v[k] = fma(v, v, s.v[k]);
        }
      return total(s);
    };
    const float sum = group_sum<G>(squares(1.f), sums, turn);
    const bool beyond = sum == INFINITY;   // the same for a group, and, where a warp has several, asked for all of them
    if (G < 32 ? __any_sync(0xffffffffu, beyond) : beyond) {
      if (G > 32) __syncthreads();
      const float less = group_sum<G>(squares(kLess), sums, turn);
      if (beyond) return inverse_rms_beyond(less, over_d);
    }
    return inverse_rms(sum, over_d, p.eps);
  };
  uint8_t *to_h = static_cast<uint8_t *>(p.h_out.at) + place(p.h_out, agent, first) * sb, *to_u = static_cast<uint8_t *>(p.u.at) + place(p.u, agent, first) * ab;
  const int64_t hop_h = hop * p.h_out.row_stride * sb, hop_u = hop * p.u.row_stride * ab;
  int64_t kept_at = (agent * p.t + first) * p.row_bytes;
  float *stats = p.stats ? p.stats + 2 * (agent * p.t + first) : nullptr;
  int from = 0;
  for (int i = 0; i < rounds; ++i) {
    bring();
    const int d = G < 32 && i >= rows ? 0 : width;   // (a row of nothing)
    copies_but(p.stages - 1);
    if (V > 1 || G <= 32) __syncwarp();   // (lanes copy for one another)
    else __syncthreads();
    const uint8_t *at = mine + from;
    from += stage_bytes;
    if (from == ring_bytes) from = 0;
    Pairs8 h[PASSES];
    float rho = 0.f;
#pragma unroll
    for (int j = 0; j < PASSES; ++j) h[j] = X::read(at, wh.pad(), ts, d, rank, j);
    if (p.h8) X::keep(p.h8 + kept_at, h, at, wh.pad(), ts, d, rank);
    if (y) {
      Pairs8 a[PASSES];
#pragma unroll
      for (int j = 0; j < PASSES; ++j) a[j] = X::read(at + off_y, wy.pad(), ta, d, rank, j);
      rho = norm(a, 0);
      if (p.y8) X::keep(p.y8 + kept_at, a, at + off_y, wy.pad(), ta, d, rank);
      if (gated) {
        Pairs8 g[PASSES];
#pragma unroll
        for (int j = 0; j < PASSES; ++j) g[j] = X::read(at + off_g, wg.pad(), ta, d, rank, j);
        if (p.gate8) X::keep(p.gate8 + kept_at, g, at + off_g, wg.pad(), ta, d, rank);
#pragma unroll
        for (int j = 0; j < PASSES; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) h[j].v[k] = fma(mul(wq[j].v[k], gates_of(g[j].v[k], silu).g), mul(a[j].v[k], all<2>(rho)), h[j].v[k]);
      } else {
#pragma unroll
        for (int j = 0; j < PASSES; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) h[j].v[k] = fma(wq[j].v[k], mul(a[j].v[k], all<2>(rho)), h[j].v[k]);
      }
#pragma unroll
      for (int j = 0; j < PASSES; ++j) X::write(to_h, ts, h[j], d, rank, j);
    }
    float r = 0.f;
    if (u) {
      r = norm(h, 1);
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
#pragma unroll
        for (int k = 0; k < 4; ++k) h[j].v[k] = mul(mul(h[j].v[k], all<2>(r)), wp[j].v[k]);
        X::write(to_u, ta, h[j], d, rank, j);
      }
    }
    if (stats) {
      if (rank == 0 && (G >= 32 || d)) *reinterpret_cast<float2 *>(stats) = make_float2(rho, r);
      stats += 2 * hop;
    }
    to_h += hop_h;
    to_u += hop_u;
    kept_at += hop * p.row_bytes;
    wh.next();
    wy.next();
    wg.next();
    if (G > 32 && (V == 1 || !y || !u)) __syncthreads();   // the place is written again only when everybody has read it, and a sum's when everybody has it
    else __syncwarp();
  }
  copies_but(0);
}

template <int G, int PASSES, int V, int TS, int TA, bool KEPT, int PARTS>
__global__ void __launch_bounds__(G * groups_of(G), resident_grad(G)) block_grad_kernel(const __grid_constant__ BlockArgs p) {
  using X = Place<G, PASSES, V>;
  extern __shared__ uint4 ring[];
  __shared__ alignas(16) float sums[2][4 * warps_of(G)];
  constexpr int kGroups = groups_of(G);
  CECA_TYPES;
  const int32_t held_s = KEPT ? kKept : ts, held_a = KEPT ? kKept : ta;
  const int rank = threadIdx.x % G, group = threadIdx.x / G, width = (int)p.d, d = width;
  const int64_t agent = blockIdx.x / p.part_count, cta = blockIdx.x - agent * p.part_count;
  const int64_t first = cta * kGroups + group, hop = (int64_t)p.part_count * kGroups;
  constexpr bool kAny = PARTS == kAnyParts;
  const bool y = !kAny || p.y.at != nullptr, gated = kAny ? p.gate.at != nullptr : PARTS != kPlain, u = !kAny || p.w_pre != nullptr, silu = kAny ? p.silu : PARTS == kSilu;
  const bool past = !kAny || p.dh_out.at != nullptr;
  const auto room = [&](int i, int32_t type, bool there) { return V > 1 && !kAny ? there ? X::room(0, type) : 0 : p.room[i]; };
  const int off_y = room(0, held_s, true), off_g = off_y + room(1, held_a, y), off_u = off_g + room(2, held_a, gated), off_p = off_u + room(3, ta, u),
            off_s = off_p + room(4, ts, past), stage_bytes = off_s + stats_room(G);
  uint8_t *mine = reinterpret_cast<uint8_t *>(ring) + (size_t)group * (p.stages * stage_bytes + aside_grad(G, PASSES));
  const uint32_t mine32 = smem_u32(mine);
  const auto held = [&](const dsgd_rows_t &x, int bytes) {
    return KEPT ? Walk(x, agent * p.t + first, hop, p.row_bytes) : Walk(x, agent, first, hop, bytes);
  };
  Walk wh = held(p.h, sb), wy = held(p.y, ab), wg = held(p.gate, ab), wu(p.du, agent, first, hop, ab), wo(p.dh_out, agent, first, hop, sb);
  const auto count = [&](int64_t from) { return from < p.t ? (int)((p.t - 1 - from) / hop) + 1 : 0; };
  // groups that share a warp stay together: for as many rows as the first of them has
  const int rows = count(first), rounds = G < 32 ? count(first - group % (32 / (G < 32 ? G : 32))) : rows, ring_bytes = p.stages * stage_bytes;
  int fill = 0, left = rows;   // the place that is filled next, the rows that are not on their way
  const float *stats = p.stats + 2 * (agent * p.t + first);
  const auto bring = [&]() {
    if (--left >= 0) {
      const uint32_t to = mine32 + fill;
      if (rank % 32 == 0) copy_8(to + off_s + rank / 32 * 8, stats);   // each warp its own
      X::copy(to, wh.at, held_s, d, rank);
      if (y) X::copy(to + off_y, wy.at, held_a, d, rank);
      if (gated) X::copy(to + off_g, wg.at, held_a, d, rank);
      if (u) X::copy(to + off_u, wu.at, ta, d, rank);
      if (past) X::copy(to + off_p, wo.at, ts, d, rank);
    }
    wh.at += wh.hop;
    wy.at += wy.hop;
    wg.at += wg.hop;
    wu.at += wu.hop;
    wo.at += wo.hop;
    stats += 2 * hop;
    fill += stage_bytes;
    if (fill == ring_bytes) fill = 0;
    copies_end();
  };
  for (int i = 0; i + 1 < p.stages; ++i) bring();
  const float scale = p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f, over_d = 1.f / (float)p.d;
  // scale w_post and w_pre, in registers or aside
  Pairs8 wq[PASSES], wp[PASSES];
  float4 *aside = reinterpret_cast<float4 *>(mine + ring_bytes) + rank;
  weights<G, PASSES, V>(wq, y ? p.w_post : nullptr, p.weights_type, agent * p.w_post_stride, scale, d, rank);
  weights<G, PASSES, V>(wp, u ? p.w_pre : nullptr, p.weights_type, agent * p.w_pre_stride, 1.f, d, rank);
  const auto put_aside = [&](const Pairs8 &w, int at) {
    aside[2 * at * G] = make_float4(w.v[0].x, w.v[0].y, w.v[1].x, w.v[1].y);
    aside[(2 * at + 1) * G] = make_float4(w.v[2].x, w.v[2].y, w.v[3].x, w.v[3].y);
  };
  const auto from_aside = [&](Pairs8 &w, int at) {
    if (!aside_grad(G, PASSES)) return;
    const float4 a = aside[2 * at * G], b = aside[(2 * at + 1) * G];
    w = {{{a.x, a.y}, {a.z, a.w}, {b.x, b.y}, {b.z, b.w}}};
  };
  if (aside_grad(G, PASSES)) {
    put_aside(wq[0], 0);
    put_aside(wp[0], 1);
  }
  Pairs8 sum_pre[PASSES], sum_post[PASSES];
#pragma unroll
  for (int j = 0; j < PASSES; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) sum_pre[j].v[k] = sum_post[j].v[k] = {0.f, 0.f};
  uint8_t *dh = static_cast<uint8_t *>(p.dh.at) + place(p.dh, agent, first) * sb, *dy = static_cast<uint8_t *>(p.dy.at) + place(p.dy, agent, first) * ab;
  uint8_t *da = static_cast<uint8_t *>(p.dgate.at) + place(p.dgate, agent, first) * ab;
  const int64_t hop_h = hop * p.dh.row_stride * sb, hop_y = hop * p.dy.row_stride * ab, hop_a = hop * p.dgate.row_stride * ab;
  int from = 0, turn = 0;
  for (int i = 0; i < rounds; ++i) {
    bring();
    const int d = G < 32 && i >= rows ? 0 : width;   // (a row of nothing)
    copies_but(p.stages - 1);
    if (V > 1 || G <= 32) __syncwarp();   // (lanes copy for one another)
    else __syncthreads();
    const uint8_t *at = mine + from;
    from += stage_bytes;
    if (from == ring_bytes) from = 0;
    const float2 now = G >= 32 || d ? *reinterpret_cast<const float2 *>(at + off_s + rank / 32 * 8) : make_float2(0.f, 0.f);
    const Val<2> rho = all<2>(now.x), r = all<2>(now.y);
    Pairs8 hn[PASSES], t[PASSES], yn[PASSES], g[PASSES], slope[PASSES];
    Val<2> a{0.f, 0.f}, b{0.f, 0.f}, c{0.f, 0.f};
    from_aside(wq[0], 0);
    from_aside(wp[0], 1);
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      Pairs8 q{};
      if (y) {
        yn[j] = X::read(at + off_y, wy.pad(), held_a, d, rank, j);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          yn[j].v[k] = mul(yn[j].v[k], rho);
          q.v[k] = mul(wq[j].v[k], yn[j].v[k]);
        }
        if (gated) {
          g[j] = X::read(at + off_g, wg.pad(), held_a, d, rank, j);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const Gates x = gates_of(g[j].v[k], silu);
            g[j].v[k] = x.g;
            slope[j].v[k] = x.slope;
            q.v[k] = mul(q.v[k], x.g);
          }
        }
      }
      if (past) {
        t[j] = X::read(at + off_p, wo.pad(), ts, d, rank, j);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) t[j].v[k] = {0.f, 0.f};
      }
      if (u) {
        hn[j] = X::read(at, wh.pad(), held_s, d, rank, j);
        const Pairs8 du = X::read(at + off_u, wu.pad(), ta, d, rank, j);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          hn[j].v[k] = mul(add(hn[j].v[k], q.v[k]), r);
          const Val<2> f = mul(wp[j].v[k], du.v[k]);
          a = fma(hn[j].v[k], f, a);
          t[j].v[k] = fma(r, f, t[j].v[k]);
          c = fma(q.v[k], hn[j].v[k], c);
          sum_pre[j].v[k] = fma(hn[j].v[k], du.v[k], sum_pre[j].v[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) b = fma(q.v[k], t[j].v[k], b);
    }
    const float3 s = group_sums<G>(make_float3(a.x + a.y, b.x + b.y, c.x + c.y), sums, turn);
    turn ^= 1;
    from_aside(wq[0], 0);
    const float rm = u ? now.y * s.x * over_d : 0.f, my = (s.y - rm * s.z) * over_d;
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      if (u) {
#pragma unroll
        for (int k = 0; k < 4; ++k) t[j].v[k] = fma(all<2>(-rm), hn[j].v[k], t[j].v[k]);
      }
      X::write(dh, ts, t[j], d, rank, j);
      if (y) {
        Pairs8 oy, oa;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          Val<2> e = mul(wq[j].v[k], t[j].v[k]), by = t[j].v[k];
          if (gated) {
            oa.v[k] = mul(mul(slope[j].v[k], yn[j].v[k]), e);
            e = mul(g[j].v[k], e);
            by = mul(g[j].v[k], by);
          }
          oy.v[k] = mul(rho, fma(all<2>(-my), yn[j].v[k], e));
          sum_post[j].v[k] = fma(yn[j].v[k], by, sum_post[j].v[k]);
        }
        X::write(dy, ta, oy, d, rank, j);
        if (gated) X::write(da, ta, oa, d, rank, j);
      }
    }
    dh += hop_h;
    dy += hop_y;
    da += hop_a;
    wh.next();
    wy.next();
    wg.next();
    wu.next();
    wo.next();
    __syncwarp();   // (of larger groups all have met since they read the place)
  }
  copies_but(0);
  follow_early();
  // the group's sums; those of a CTA's groups are joined in their order
  const int64_t q = agent * p.part_count + cta;
  float *to = p.parts + 2 * q * p.d, dot = 0.f;
#pragma unroll
  for (int j = 0; j < PASSES; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = channel<G, V>(rank, j, e);
      const float x = e & 1 ? sum_pre[j].v[e / 2].y : sum_pre[j].v[e / 2].x, z = e & 1 ? sum_post[j].v[e / 2].y : sum_post[j].v[e / 2].x;
      if (c >= d) continue;
      if (y) dot = fmaf(load(p.w_post, p.weights_type, agent * p.w_post_stride + c), z, dot);
      if (kGroups == 1) {
        to[c] = x;
        to[p.d + c] = z;
      }
    }
  if (kGroups > 1) {
    __syncthreads();
    float *all_of = reinterpret_cast<float *>(ring);   // kGroups x 2 x d
#pragma unroll
    for (int j = 0; j < PASSES; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = channel<G, V>(rank, j, e);
        if (c >= d) continue;
        all_of[(2 * group) * d + c] = e & 1 ? sum_pre[j].v[e / 2].y : sum_pre[j].v[e / 2].x;
        all_of[(2 * group + 1) * d + c] = e & 1 ? sum_post[j].v[e / 2].y : sum_post[j].v[e / 2].x;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * d; c += G * kGroups) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) x += all_of[2 * i * d + c];
      to[c] = x;
    }
  }
  if (p.dscale) {
    const float s = group_sum<G>(dot, sums, turn);   // (the other place than the last row's)
    if (rank == 0) p.scale_parts[q * kGroups + group] = s;
  }
}

// ---------------------------------------------------------------------------------------------- launches

constexpr int kMostShared = 220 << 10;

template <int G, int PASSES, int V, int TS, int TA, int PARTS> cudaError_t launch_block(BlockArgs p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  using X = Place<G, PASSES, V>;
  auto kernel = block_kernel<G, PASSES, V, TS, TA, PARTS>;
  constexpr int kGroups = groups_of(G), kThreads = G * kGroups;
  const cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), kMostShared, &done);
  if (e != cudaSuccess) return e;
  p.room[0] = X::room(p.d, p.stream_type);
  p.room[1] = p.y.at ? X::room(p.d, p.act_type) : 0;
  p.room[2] = p.gate.at ? X::room(p.d, p.act_type) : 0;
  p.stage_bytes = p.room[0] + p.room[1] + p.room[2];
  const int64_t resident = resident_block(G, PASSES);
  p.stages = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, (int64_t)(200 << 10) / (resident * kGroups * p.stage_bytes)));
  const int64_t bytes = (int64_t)p.stages * p.stage_bytes * kGroups;
  if (bytes > kMostShared) return cudaErrorInvalidConfiguration;
  p.part_count = (int32_t)std::max<int64_t>(1, std::min((int64_t)sm_count() * resident / p.n, ceil_div(p.t, kGroups)));
  kernel<<<(unsigned)(p.n * p.part_count), kThreads, (size_t)bytes, s>>>(p);
  return cudaGetLastError();
}

template <int G, int PASSES, int V, int TS, int TA, bool KEPT, int PARTS> cudaError_t launch_block_grad(BlockArgs p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  using X = Place<G, PASSES, V>;
  auto kernel = block_grad_kernel<G, PASSES, V, TS, TA, KEPT, PARTS>;
  constexpr int kGroups = groups_of(G), kThreads = G * kGroups;
  cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), kMostShared, &done);
  if (e != cudaSuccess) return e;
  constexpr int64_t aside = kGroups * aside_grad(G, PASSES);
  p.room[0] = X::room(p.d, KEPT ? kKept : p.stream_type);
  p.room[1] = p.y.at ? X::room(p.d, KEPT ? kKept : p.act_type) : 0;
  p.room[2] = p.gate.at ? X::room(p.d, KEPT ? kKept : p.act_type) : 0;
  p.room[3] = p.w_pre ? X::room(p.d, p.act_type) : 0;
  p.room[4] = p.dh_out.at ? X::room(p.d, p.stream_type) : 0;
  p.stage_bytes = p.room[0] + p.room[1] + p.room[2] + p.room[3] + p.room[4] + stats_room(G);
  p.stages = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, ((int64_t)(200 << 10) / resident_grad(G) - aside) / (kGroups * p.stage_bytes)));
  const int64_t bytes = std::max((int64_t)p.stages * p.stage_bytes * kGroups + aside, kGroups > 1 ? kGroups * 8 * p.d : 0);
  if (bytes > kMostShared) return cudaErrorInvalidConfiguration;
  p.part_count = (int32_t)block_grad_parts(p.n, p.t, p.d);
  p.scale_count = p.part_count * kGroups;
  p.parts = reinterpret_cast<float *>(p.means);   // the workspace
  p.scale_parts = p.parts + (size_t)p.n * p.part_count * 2 * p.d;   // the rest of part_floats
  kernel<<<(unsigned)(p.n * p.part_count), kThreads, (size_t)bytes, s>>>(p);
  e = cudaGetLastError();
  return e == cudaSuccess ? finish_block_grad(p, s) : e;
}

template <int V, int TS, int TA> cudaError_t launch_rows(const BlockArgs &p, bool grad, cudaStream_t s) {
  const auto with = [&](auto widest, auto parts) {
    constexpr Shape f = shape_of(decltype(widest)::value), g = grad_shape_of(decltype(widest)::value);
    constexpr int PARTS = decltype(parts)::value;
    if (!grad) return launch_block<f.group, f.passes, V, TS, TA, PARTS>(p, s);
    return p.kept ? launch_block_grad<g.group, g.passes, V, TS, TA, true, PARTS>(p, s) : launch_block_grad<g.group, g.passes, V, TS, TA, false, PARTS>(p, s);
  };
  const auto by = [&](auto widest) {
    if constexpr (TS != kAnyType) {
      if (p.y.at && p.w_pre && (!grad || p.dh_out.at)) {
        if (!p.gate.at) return with(widest, std::integral_constant<int, kPlain>());
        return p.silu ? with(widest, std::integral_constant<int, kSilu>()) : with(widest, std::integral_constant<int, kSigmoid>());
      }
    }
    return with(widest, std::integral_constant<int, kAnyParts>());
  };
  if (p.d <= 64) return by(std::integral_constant<int, 64>());
  if (p.d <= 128) return by(std::integral_constant<int, 128>());
  if (p.d <= 256) return by(std::integral_constant<int, 256>());
  if (p.d <= 512) return by(std::integral_constant<int, 512>());
  if (p.d <= 1024) return by(std::integral_constant<int, 1024>());
  if (p.d <= 2048) return by(std::integral_constant<int, 2048>());
  if (p.d <= 4096) return by(std::integral_constant<int, 4096>());
  return by(std::integral_constant<int, 8192>());
}

}  // namespace ceca
