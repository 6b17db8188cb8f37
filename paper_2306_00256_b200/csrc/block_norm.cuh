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

// Rows of up to kWidest channels: a group of threads holds a row in registers, 8 channels each (kWidest: 16).  kWidest is what 512 threads
// can hold with the weights and their gradients' sums.
constexpr int64_t kWidest = 8192;
// The threads of a group, and of a CTA, for rows of d channels.
inline int group_of(int64_t d) { return d <= 256 ? 32 : d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : 512; }
inline int cta_of(int64_t d) { return group_of(d) == 32 ? 128 : group_of(d); }
// Whether a tensor's rows all start on 16-byte boundaries.
inline bool on_words(const dsgd_rows_t &x, int32_t type) {
  const int64_t n = 16 / type_bytes(type);
  return !x.at || ((reinterpret_cast<uintptr_t>(x.at) & 15) == 0 && x.agent_stride % n == 0 && x.row_stride % n == 0);
}
cudaError_t launch_block_rows(BlockArgs p, bool words, cudaStream_t s);        // block_rows.cu
cudaError_t launch_block_grad_rows(BlockArgs p, bool words, cudaStream_t s);   // block_grad_rows.cu
cudaError_t finish_block_grad(const BlockArgs &p, cudaStream_t s);             // block_norm.cu: joins the parts
// CTAs an SM (at least one) that run the gradient's kernel at a time: what its parts are counted by.
int64_t block_grad_parts(int64_t n, int64_t t, int64_t d);

#ifdef __CUDACC__
__device__ __forceinline__ float load(const void *p, int32_t type, int64_t i) {
  return type == DSGD_BF16 ? widen(static_cast<const bf16 *>(p)[i]) : static_cast<const float *>(p)[i];
}
__device__ __forceinline__ void store(void *p, int32_t type, int64_t i, float v) {
  if (type == DSGD_BF16) narrow(static_cast<bf16 *>(p) + i, v);
  else narrow(static_cast<float *>(p) + i, v);
}
__device__ __forceinline__ int64_t place(const dsgd_rows_t &x, int64_t agent, int64_t row) { return agent * x.agent_stride + row * x.row_stride; }

// A gate's factor and its derivative.  The smaller of sigmoid and 1 - sigmoid comes from the exponential itself, so neither loses digits.
struct Gate {
  float g, slope;
};
__device__ __forceinline__ Gate gate_of(float a, bool silu) {
  const float e = ex2(-1.4426950408889634f * fabsf(a)), r = rcp(1.f + e), s = e * r;   // (fabsf keeps a NaN)
  const float sig = a < 0.f ? s : r, slope = s * r;
  return silu ? Gate{a * sig, fmaf(a, slope, sig)} : Gate{sig, slope};
}

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

// The channels of a thread of a group of G: with WORDS 8 neighbours (channel 8 (rank + G j) on, in 16-byte words), else every G-th one.
// They are computed on in pairs.  PASSES: eights a thread.
template <int G, int PASSES, bool WORDS> struct Lay {
  static constexpr int kPairs = 4 * PASSES;
  __device__ static int channel(int rank, int j, int e) { return WORDS ? 8 * (rank + G * j) + e : rank + G * (8 * j + e); }
};
struct Pairs8 {
  Val<2> v[4];
};

// A place in shared memory for a row of a tensor, or for a kept row, and its copy and reading.  With WORDS each thread copies what it will
// read; else the group copies the 16-byte words that the row touches (of the first and last one the bytes inside the row count), and
// must meet between copying and reading.
template <int G, int PASSES, bool WORDS> struct Place {
  using L = Lay<G, PASSES, WORDS>;
  __device__ static int room(int64_t d, int32_t type) { return type == 2 ? (int)(WORDS ? 12 * G * PASSES : kept_row_bytes(d)) : (int)(WORDS ? (16 * G * PASSES) * (type == DSGD_BF16 ? 1 : 2) : d * (type == DSGD_BF16 ? 2 : 4) + 32); }
  // type 2: kept
  __device__ static void copy(uint32_t to, const uint8_t *from, int32_t type, int d, int rank) {
    if (WORDS) {
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        const int at = rank + G * j;
        if (8 * at >= d) continue;
        if (type == 2) {
          copy_8(to + 8 * at, from + 8 * at);
          copy_4(to + 8 * G * PASSES + 4 * at, from + ((d + at / 4) & ~3));
        } else if (type == DSGD_BF16) {
          copy_16(to + 16 * at, from + 16 * at);
        } else {
          copy_16(to + 16 * at, from + 32 * at);
          copy_16(to + 16 * (G * PASSES + at), from + 32 * at + 16);
        }
      }
    } else {
      const int pad = (int)(reinterpret_cast<uintptr_t>(from) & 15), end = pad + (type == 2 ? (int)kept_row_bytes(d) : d * (type == DSGD_BF16 ? 2 : 4));
      from -= pad;
      for (int at = 16 * rank; at < end; at += 16 * G) copy_16(to + at, from + at, min(16, end - at));
    }
  }
  // the eight channels of pass j; zeros outside the row
  __device__ static Pairs8 read(const uint8_t *place, int pad, int32_t type, int d, int rank, int j) {
    Pairs8 r;
    if (WORDS) {
      const int at = rank + G * j;
      if (8 * at >= d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = {0.f, 0.f};
      } else if (type == 2) {
        const uint2 q = reinterpret_cast<const uint2 *>(place)[at];
        const uint32_t e = reinterpret_cast<const uint32_t *>(place + 8 * G * PASSES)[at] >> 8 * ((d + at / 4) & 3) & 255u;
        const Val<2> step = all<2>(step8(e));
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = mul(bytes8(i < 2 ? q.x : q.y, 2 * (i & 1)), step);
      } else if (type == DSGD_BF16) {
        const uint4 w = reinterpret_cast<const uint4 *>(place)[at];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = (&w.x)[i];
          r.v[i] = {__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)};
        }
      } else {
        const float4 a = reinterpret_cast<const float4 *>(place)[at], b = reinterpret_cast<const float4 *>(place)[G * PASSES + at];
        r.v[0] = {a.x, a.y};
        r.v[1] = {a.z, a.w};
        r.v[2] = {b.x, b.y};
        r.v[3] = {b.z, b.w};
      }
    } else {
      place += pad;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::channel(rank, j, e);
        float x = 0.f;
        if (c < d) {
          if (type == 2) x = (float)(int8_t)place[c] * step8(place[d + c / kBlock8]);
          else x = type == DSGD_BF16 ? widen(reinterpret_cast<const bf16 *>(place)[c]) : reinterpret_cast<const float *>(place)[c];
        }
        (e & 1 ? r.v[e / 2].y : r.v[e / 2].x) = x;
      }
    }
    return r;
  }
  // bytes `from` and from + 1 of w, two whole numbers
  __device__ static Val<2> bytes8(uint32_t w, int from) {
    w ^= 0x80808080u;   // (x + 128) + 2^23, less 2^23 + 128
    const Val<2> v = {__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | from)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650u | (from + 1)))};
    return add(v, all<2>(-8388736.f));
  }
  // writes eight channels of a row
  __device__ static void write(void *row, int32_t type, const Pairs8 &x, int d, int rank, int j) {
    if (WORDS) {
      const int at = rank + G * j;
      if (8 * at >= d) return;
      if (type == DSGD_BF16) {
        uint4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(x.v[i].x, x.v[i].y);
          (&w.x)[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        static_cast<uint4 *>(row)[at] = w;
      } else {
        static_cast<float4 *>(row)[2 * at] = make_float4(x.v[0].x, x.v[0].y, x.v[1].x, x.v[1].y);
        static_cast<float4 *>(row)[2 * at + 1] = make_float4(x.v[2].x, x.v[2].y, x.v[3].x, x.v[3].y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::channel(rank, j, e);
        if (c < d) store(row, type, c, e & 1 ? x.v[e / 2].y : x.v[e / 2].x);
      }
    }
  }
  // keeps eight channels of a row in 8 bits; whole warps call it
  __device__ static void keep(uint8_t *row, const Pairs8 &x, int d, int rank, int j) {
    if (WORDS) {
      const int at = rank + G * j;
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(magnitude(x.v[i].x), magnitude(x.v[i].y)));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      if (8 * at >= d) return;
      const uint32_t e = exponent8(top);
      const Val<2> by = all<2>(scale8(e));
      uint32_t b[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Val<2> v = mul(x.v[i], by);
        // rounded to the nearest whole number in the low bits of a sum with 1.5 2^23 (a NaN times 0 becomes 0 first: fmaxf drops it, to -127, so it is asked for)
        b[2 * i] = __float_as_uint(fminf(fmaxf(v.x, -127.f), 127.f) + 12582912.f);
        b[2 * i + 1] = __float_as_uint(fminf(fmaxf(v.y, -127.f), 127.f) + 12582912.f);
      }
      uint2 q;
      q.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
      q.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
      if (e == 255u) q = make_uint2(0, 0);
      reinterpret_cast<uint2 *>(row)[at] = q;
      if (at % 4 == 0) row[d + at / 4] = (uint8_t)e;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = L::channel(rank, j, e);
        const float v = e & 1 ? x.v[e / 2].y : x.v[e / 2].x;
        const uint32_t b = exponent8(__reduce_max_sync(0xffffffffu, magnitude(v)));
        if (c < d) {
          row[c] = (uint8_t)(int8_t)hold8(v, scale8(b));
          if (c % kBlock8 == 0) row[d + c / kBlock8] = (uint8_t)b;
        }
      }
    }
  }
  // the bytes behind a kept row's exponents
  __device__ static void keep_end(uint8_t *row, int d, int rank) {
    const int from = d + (int)blocks8(d), to = (int)kept_row_bytes(d);
    if (rank < to - from) row[from + rank] = 0;
  }
};

// The sum over a group, in one order, the same on all its threads.  `turn` says which of two places is used: consecutive sums take
// the other one, so that one barrier a sum is enough.
template <int G> __device__ __forceinline__ float group_sum(float x, float (*part)[G / 32], int turn) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (G == 32) return x;
  if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int i = 0; i < G / 32; ++i) x += part[turn][i];
  return x;
}

__device__ __forceinline__ float total(const Pairs8 &a) {
  const Val<2> s = add(add(a.v[0], a.v[1]), add(a.v[2], a.v[3]));
  return s.x + s.y;
}

// 1 / sqrt(sum / d + eps) of a sum of squares; one that overflowed is taken again by `again`, of the values times 2^-100.
template <typename Again> __device__ __forceinline__ float inverse_rms(float sum, int64_t d, float eps, Again again) {
  float unit = 1.f;
  if (sum == INFINITY) {
    unit = 0x1p-100f;
    sum = again(unit);
  }
  return unit / sqrtf(fmaf(eps * unit, unit, sum / (float)d));
}
#endif

}  // namespace ceca
