// Activations kept in 8 bits, and brought back.
//
// Both directions stream: what bounds them is memory, and how much of it is under way (kDeep vectors of 16 bytes of x a thread).  A thread stays at its place
// in a row and goes from row to row, so that nothing is divided on the way.  Keeping, the lanes that share a block of 32 channels find its largest
// magnitude by exchange; where x does not start on a 16-byte boundary a lane shifts its channels out of two words.  Bringing back, a lane takes the
// 16-byte words of x, and shifts the whole numbers.
// 8 x 8192 x 2048 bf16: kept in 80 us, brought back in 71 (0.77 and 0.88 of the measured copy rate); 2047
// channels, shifted: 133 and 101.
#include <cuda_runtime.h>

#include <algorithm>

#include "ceca.h"
#include "keep8.cuh"
#include "tma.h"

namespace ceca {
namespace {

// Few rows at a time and many more CTAs than run at once: that way some read while others write, and the last ones end together.  (8 x 8192 x 2048 bf16: 80 us
// kept, 71 brought back; with 4 rows at a time, or one CTA for each place on an SM, 10 to 30 us more.)
constexpr int kThreads = 256, kDeep = 2, kWaves = 48;

struct KeepArgs {
  dsgd_rows_t x;
  uint8_t *kept;
  int64_t t, rows, row_bytes, hop, step_x, step_kept;   // a thread takes kDeep neighbouring rows of every kDeep hop, so many times
  int32_t rounds, d, blocks, per_row, flat;          // vectors of a row; flat: the rows lie at equal distances throughout
};

// The rows that a thread takes: row 0 to kDeep - 1 from `row` on, then kDeep hop further.
template <typename T> struct Rows {
  int64_t row;
  T *x;            // of rows at equal distances
  uint8_t *kept;
  __device__ __forceinline__ Rows(const KeepArgs &p, uint32_t first) : row((int64_t)first * kDeep), x(static_cast<T *>(p.x.at) + row * p.x.row_stride), kept(p.kept + row * p.row_bytes) {}
  __device__ __forceinline__ T *at(const KeepArgs &p, int u) const {
    if (p.flat) return x + u * p.x.row_stride;
    const int64_t agent = (row + u) / p.t;
    return static_cast<T *>(p.x.at) + agent * p.x.agent_stride + (row + u - agent * p.t) * p.x.row_stride;
  }
  __device__ __forceinline__ void next(const KeepArgs &p) {
    row += p.hop * kDeep;
    x += p.step_x;
    kept += p.step_kept;
  }
};

// N values of 16 bytes, in pairs.
template <int N> struct Values {
  Val<2> v[N / 2];
};
__device__ __forceinline__ Values<4> widened(uint4 a, const float *) { return {{{__uint_as_float(a.x), __uint_as_float(a.y)}, {__uint_as_float(a.z), __uint_as_float(a.w)}}}; }
__device__ __forceinline__ Values<8> widened(uint4 a, const bf16 *) { return {{unpack_bf16(a.x), unpack_bf16(a.y), unpack_bf16(a.z), unpack_bf16(a.w)}}; }
__device__ __forceinline__ uint4 narrowed(const Values<4> &a) { return make_uint4(__float_as_uint(a.v[0].x), __float_as_uint(a.v[0].y), __float_as_uint(a.v[1].x), __float_as_uint(a.v[1].y)); }
__device__ __forceinline__ uint4 narrowed(const Values<8> &a) { return make_uint4(pack_bf16(a.v[0]), pack_bf16(a.v[1]), pack_bf16(a.v[2]), pack_bf16(a.v[3])); }

// The bits of the largest magnitude of 16 bytes of values (two bf16 at a time).
__device__ __forceinline__ uint32_t top_of(uint4 a, const float *) {
  const uint32_t m = 0x7fffffffu;
  return max(max(a.x & m, a.y & m), max(a.z & m, a.w & m));
}
__device__ __forceinline__ uint32_t top_of(uint4 a, const bf16 *) {
  const uint32_t m = 0x7fff7fffu, t = __vmaxu2(__vmaxu2(a.x & m, a.y & m), __vmaxu2(a.z & m, a.w & m));
  return max(t << 16, t & 0xffff0000u);
}

// 16 bytes from any boundary on, of a row that ends at `end` (what lies behind is anything).
template <bool WORDS> __device__ __forceinline__ uint4 take(const void *at, const void *end) {
  if (WORDS) return __ldg(static_cast<const uint4 *>(at));
  const uint32_t pad = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15);
  const uint4 *word = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(at) - pad);
  const uint4 a = __ldg(word), b = pad && static_cast<const void *>(word + 1) < end ? __ldg(word + 1) : make_uint4(0, 0, 0, 0);
  uint32_t w[7] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z}, last = b.w;
  if (pad & 8) {
    w[0] = w[2], w[1] = w[3], w[2] = w[4], w[3] = w[5], w[4] = w[6], w[5] = last;
  }
  if (pad & 4) {
    w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = w[4], w[4] = w[5];
  }
  const uint32_t by = 8 * (pad & 3);
  return make_uint4(__funnelshift_r(w[0], w[1], by), __funnelshift_r(w[1], w[2], by), __funnelshift_r(w[2], w[3], by), __funnelshift_r(w[3], w[4], by));
}

template <typename T, bool WORDS> __global__ void __launch_bounds__(kThreads, 6) keep_kernel(const __grid_constant__ KeepArgs p) {
  constexpr int N = 16 / sizeof(T);
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x, first = id / (uint32_t)p.per_row;
  const int c = N * (int)(id - first * p.per_row);
  const bool taken = first < p.hop, here = taken && c < p.d;
  Rows<const T> at(p, first);
  for (int i = 0; i < p.rounds; ++i, at.next(p)) {   // the same for all, who exchange
    uint4 a[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      a[u] = make_uint4(0, 0, 0, 0);
      if (!here || at.row + u >= p.rows) continue;
      const T *x = at.at(p, u);
      a[u] = take<WORDS>(x + c, x + p.d);
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      if (!WORDS && c + N > p.d) {   // what lies behind the row's last ones
        uint8_t *bytes = reinterpret_cast<uint8_t *>(&a[u]);
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (c + k / (int)sizeof(T) >= p.d) bytes[k] = 0;
      }
      const Values<N> v = widened(a[u], static_cast<const T *>(nullptr));
      uint32_t top = top_of(a[u], static_cast<const T *>(nullptr));
#pragma unroll
      for (int o = 1; o < kBlock8 / N; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const bool cut = __any_sync(0xffffffffu, cut8(top));   // of one warp in thirty: a branch, not a choice for each
      if (!taken || at.row + u >= p.rows) continue;
      uint8_t *to = at.kept + u * p.row_bytes;
      const uint32_t e = exponent8(top);
      if (c < p.d) {
        const Val<2> by = all<2>(scale8(e));
        uint32_t q[2];
#pragma unroll
        for (int k = 0; k < N / 4; ++k) q[k] = e == 255u ? 0 : hold_four(v.v[2 * k], v.v[2 * k + 1], by, cut);
        if (!WORDS && c + N > p.d) {
          for (int k = 0; c + k < p.d; ++k) to[c + k] = (uint8_t)(q[k / 4] >> 8 * (k & 3));
        } else if (N == 8) {
          *reinterpret_cast<uint2 *>(to + c) = make_uint2(q[0], q[1]);
        } else {
          *reinterpret_cast<uint32_t *>(to + c) = q[0];
        }
      }
      if (c % kBlock8 == 0) {
        to[p.d + c / kBlock8] = (uint8_t)e;
        if (c / kBlock8 == p.blocks - 1)
          for (int64_t k = p.d + p.blocks; k < p.row_bytes; ++k) to[k] = 0;
      }
    }
  }
}

template <typename T, bool WORDS> __global__ void __launch_bounds__(kThreads, 6) bring_kernel(const __grid_constant__ KeepArgs p) {
  constexpr int N = 16 / sizeof(T);
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x, first = id / (uint32_t)p.per_row;
  if (first >= p.hop) return;
  const int slot = N * (int)(id - first * p.per_row);
  Rows<T> rows(p, first);
  for (int i = 0; i < p.rounds; ++i, rows.next(p)) {
    T *x[kDeep];
    int c[kDeep];
    uint32_t w[kDeep][3], e[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      c[u] = p.d;
      if (rows.row + u >= p.rows) continue;
      const uint8_t *from = rows.kept + u * p.row_bytes;
      x[u] = rows.at(p, u);
      c[u] = WORDS ? slot : slot - (int)((reinterpret_cast<uintptr_t>(x[u]) & 15) / sizeof(T));
      if (c[u] >= p.d) continue;
      if (WORDS) {
        if (N == 8) {
          const uint2 q = __ldg(reinterpret_cast<const uint2 *>(from + c[u]));
          w[u][0] = q.x;
          w[u][1] = q.y;
        } else {
          w[u][0] = __ldg(reinterpret_cast<const uint32_t *>(from + c[u]));
        }
        e[u] = __ldg(from + p.d + c[u] / kBlock8);
      } else {
        const int at = c[u] & ~3;   // whole words of the kept row, which begins and ends on one
#pragma unroll
        for (int k = 0; k <= N / 4; ++k) w[u][k] = at + 4 * k >= 0 && at + 4 * k < p.row_bytes ? __ldg(reinterpret_cast<const uint32_t *>(from + at + 4 * k)) : 0;
        const int b = max(c[u], 0) / kBlock8;
        e[u] = __ldg(from + p.d + b) | (uint32_t)__ldg(from + p.d + min(b + 1, p.blocks - 1)) << 8;
      }
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      if (c[u] >= p.d) continue;
      Values<N> v;
      if (WORDS) {
        const Val<2> step = all<2>(step8(e[u]));
#pragma unroll
        for (int k = 0; k < N / 2; ++k) v.v[k] = mul(whole_numbers(w[u][k / 2], 2 * (k & 1)), step);
        *reinterpret_cast<uint4 *>(x[u] + c[u]) = narrowed(v);
      } else {
        const uint32_t by = 8 * (c[u] & 3);
        const float step = step8(e[u] & 255u), next = step8(e[u] >> 8);
        const int turn = (max(c[u], 0) / kBlock8 + 1) * kBlock8 - c[u];   // where the next block begins
#pragma unroll
        for (int k = 0; k < N / 2; ++k)
          v.v[k] = mul(whole_numbers(__funnelshift_r(w[u][k / 2], w[u][k / 2 + 1], by), 2 * (k & 1)), Val<2>{2 * k < turn ? step : next, 2 * k + 1 < turn ? step : next});
        if (c[u] >= 0 && c[u] + N <= p.d) {
          *reinterpret_cast<uint4 *>(x[u] + c[u]) = narrowed(v);
        } else {
#pragma unroll
          for (int k = 0; k < N; ++k)
            if (c[u] + k >= 0 && c[u] + k < p.d) narrow(x[u] + c[u] + k, k & 1 ? v.v[k / 2].y : v.v[k / 2].x);
        }
      }
    }
  }
}

template <typename T, bool WORDS> cudaError_t launch(const dsgd_rows_t &x, void *kept, int32_t n, int64_t t, int64_t d, bool back, cudaStream_t s) {
  constexpr int N = 16 / sizeof(T);
  KeepArgs p{};
  p.x = x;
  p.kept = static_cast<uint8_t *>(kept);
  p.t = t; p.rows = n * t; p.row_bytes = kept_row_bytes(d); p.d = (int32_t)d; p.blocks = (int32_t)blocks8(d);
  p.flat = n == 1 || x.agent_stride == t * x.row_stride;
  // keeping: whole blocks, so that a block's lanes lie in one warp; bringing back: the words that a row on the least fortunate boundary touches
  const int64_t per_row = !back ? p.blocks * (kBlock8 / N) : WORDS ? d / N : ceil_div(d + N - 1, N);
  p.per_row = (int32_t)per_row;
  p.hop = std::max<int64_t>(1, std::min(ceil_div(p.rows, kDeep), (int64_t)sm_count() * kWaves * kThreads / per_row));
  p.step_x = p.hop * kDeep * x.row_stride;
  p.step_kept = p.hop * kDeep * p.row_bytes;
  p.rounds = (int32_t)ceil_div(p.rows, p.hop * kDeep);
  const int64_t grid = ceil_div(p.hop * per_row, kThreads);
  if (back) bring_kernel<T, WORDS><<<(unsigned)grid, kThreads, 0, s>>>(p);
  else keep_kernel<T, WORDS><<<(unsigned)grid, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

ceca_status_t keep8(const dsgd_rows_t &x, void *kept, int32_t n, int64_t t, int64_t d, int32_t type, bool back, void *stream) {
  const int64_t most = ((int64_t)1 << 31) - 1024;
  if (n < 1 || n > 65535 || t < 0 || t >= most || d < 1 || d >= most || x.row_stride < d || x.agent_stride < 0 || (back && n > 1 && x.agent_stride < d) || !is_type(type))
    return CECA_ERR_INVALID_ARG;
  if (t == 0) return CECA_OK;
  if (!x.at || !kept) return CECA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(kept) & 15) return CECA_ERR_ALIGNMENT;
  const int64_t word = 16 / type_bytes(type);
  const bool words = (reinterpret_cast<uintptr_t>(x.at) & 15) == 0 && d % word == 0 && (t == 1 || x.row_stride % word == 0) && (n == 1 || x.agent_stride % word == 0);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (type == DSGD_F32) e = words ? launch<float, true>(x, kept, n, t, d, back, s) : launch<float, false>(x, kept, n, t, d, back, s);
  else e = words ? launch<bf16, true>(x, kept, n, t, d, back, s) : launch<bf16, false>(x, kept, n, t, d, back, s);
  return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

}  // namespace
}  // namespace ceca

extern "C" int64_t dsgd_kept_row_bytes(int64_t d) { return d < 1 ? 0 : ceca::kept_row_bytes(d); }

extern "C" ceca_status_t dsgd_keep8(dsgd_rows_t x, void *kept, int32_t n, int64_t t, int64_t d, int32_t type, void *stream) {
  return ceca::keep8(x, kept, n, t, d, type, false, stream);
}

extern "C" ceca_status_t dsgd_bring8(const void *kept, dsgd_rows_t x, int32_t n, int64_t t, int64_t d, int32_t type, void *stream) {
  return ceca::keep8(x, const_cast<void *>(kept), n, t, d, type, true, stream);
}
