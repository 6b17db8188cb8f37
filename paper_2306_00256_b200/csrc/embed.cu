// Token embedding of n agents and its gradient.
//
//   out[i, s, :] = scale E_i[tok[i, s], :]          dE_i[w, :] = scale sum_{s : tok[i, s] = w} dout[i, s, :]
//
// Both directions move rows and do one multiplication or addition per element, so bytes bound them.  The
// gradient runs in three launches without atomics on values, in one order of additions:
//   token_list_kernel   lists every table row's positions in ascending order, by token;
//   embed_grad_kernel   cuts the list into chunks of up to 32 places.  A warp takes the rows that begin in its chunk, or,
//                       of a row with more positions than a chunk has places, the piece
//                       that lies in it: however the tokens are distributed, its work is the same.  Other CTAs fill the rows that no position holds;
//   embed_join_kernel   adds up the pieces of the rows that have several.
// 8 x 8192 positions in bf16 of 32000 x 1024 fp32 tables: 0.23 ms, 0.79 of the measured copy rate, of which the list takes
// 22 to 24 us (the block with the most frequent tokens, whose shared-memory counters every token passes) and the join 10.
// Lookup of 8 x 8192 rows of 2048 bf16: 68 us, 0.84.  bf16 rows on 8-byte boundaries move four elements a lane (1044 columns,
// lookup and gradient: 67 and 192 us, 107 and 299 with one), rows on other boundaries one (1031 columns: lookup 0.27 in bf16, 0.53 in
// fp32, gradient 0.35 and 0.57).  Accumulating, the 8 x 8192 positions take 0.16 ms, 0.33: list, pieces and join, few rows to write.
// For up to kFew positions these three launches would take longer than their work: embed_few_kernel looks the positions of
// every row up as it goes (4 x 129 positions, 4097 x 256 fp32: 18 us by three launches, 9 to 10 us so).
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "ceca.h"
#include "tma.h"
#include "values.h"

namespace ceca {
namespace {

struct EmbedArgs {
  const void *src;     // the tables (lookup) or dout (gradient)
  void *dst;           // out (lookup) or the gradient's tables
  const void *tokens;
  int64_t t, v, d;
  int64_t table_agent, table_row, tokens_agent, out_agent, out_row;
  int32_t n;
  float scale;
  int32_t accumulate;
  int32_t *row_start;  // n x (v + 1): where each table row's positions begin in `list`
  int2 *list;          // n x t: positions, by token and then ascending, each with its token
  float *pieces;       // n x chunks x 2 x d: sums of the pieces of long lists
  int32_t bins;        // table rows per block of token_list_kernel
  int64_t part;        // tokens that it places, a multiple of 32 for each warp
  int32_t chunk;       // places of the list for a warp, at most 32
  int32_t chunks;      // of an agent's list
  int32_t slices;      // of a row
  int32_t fills;       // CTAs that fill kFill rows each with zeros
};

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kFill = 64;      // table rows
constexpr int kJoin = 2;       // chunks
constexpr int kFew = 256;      // positions
constexpr int64_t kMaxWidth = 65535 * 256;   // columns of a gradient: its slices are a dimension of the grid
constexpr int kFewRows = 16;   // table rows of a CTA
constexpr int kDeep = 4;       // rows of dout that a warp has on their way at a time
constexpr int kListThreads = 1024;
constexpr int kListWarps = kListThreads / 32;
constexpr int kMaxBins = kListThreads;   // a row for each thread

// V adjacent elements, moved at once: 8 where both of a call's types are bf16, otherwise 4; where rows lie on 8-byte
// boundaries only, 4 in bf16; 1 for rows on any boundary.
template <typename T, int V> struct Pack;
template <int V> struct alignas(V * 4) Pack<float, V> {
  float e[V];
  __device__ __forceinline__ void get(float *x) const {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = e[i];
  }
  __device__ __forceinline__ void set(const float *x) {
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = x[i];
  }
};
template <> struct Pack<bf16, 1> {
  bf16 e;
  __device__ __forceinline__ void get(float *x) const { *x = __bfloat162float(e); }
  __device__ __forceinline__ void set(const float *x) { e = __float2bfloat16_rn(*x); }
};
template <int V> struct alignas(V * 2) Pack<bf16, V> {
  uint32_t w[V / 2];
  __device__ __forceinline__ void get(float *x) const {   // a bf16 is the upper half of the fp32 of the same value
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float *x) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
  }
};
template <typename T, int V> __device__ __forceinline__ void add_to(float *acc, const Pack<T, V> &v) {
  float x[V];
  v.get(x);
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] += x[i];
}
template <typename T, int V> __device__ __forceinline__ void put(T *p, const float *x) {
  Pack<T, V> v;
  v.set(x);
  *reinterpret_cast<Pack<T, V> *>(p) = v;
}
template <typename T, int V> __device__ __forceinline__ Pack<T, V> get(const T *p) { return *reinterpret_cast<const Pack<T, V> *>(p); }
// A warp works on a slice of a row at a time: U packs of a lane, 32 V elements apart.
template <int V> struct Slice {
  static constexpr int U = V == 8 ? 2 : V == 4 ? 4 : 8, kElements = 32 * U * V;
};

template <int V> constexpr int kLookupPacks = V == 1 ? 16 : 4;   // that a lane has on their way at a time

template <typename TE, typename TO, typename TI, int V>
__global__ void __launch_bounds__(kThreads) embed_lookup_kernel(const EmbedArgs p) {
  constexpr int U = kLookupPacks<V>;
  const int lane = threadIdx.x & 31;
  const int64_t units = (int64_t)p.n * p.t * p.slices, step = (int64_t)gridDim.x * kWarps;
  const auto token = [&](int64_t unit) -> int64_t {   // of the unit's position
    const int64_t row = p.slices == 1 ? unit : unit / p.slices, i = row / p.t;
    return static_cast<const TI *>(p.tokens)[i * p.tokens_agent + (row - i * p.t)];
  };
  int64_t unit = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  int64_t tok = unit < units ? token(unit) : 0;
  for (; unit < units; unit += step) {
    const int64_t coming = unit + step < units ? token(unit + step) : 0;   // on its way before the rows are
    const int64_t row = p.slices == 1 ? unit : unit / p.slices, i = row / p.t;
    const int64_t c0 = (unit - row * p.slices) * (32 * U * V) + lane * V;
    const bool some = tok >= 0 && tok < p.v;
    const TE *e = static_cast<const TE *>(p.src) + i * p.table_agent + (some ? tok : 0) * p.table_row + c0;
    TO *o = static_cast<TO *>(p.dst) + i * p.out_agent + (row - i * p.t) * p.out_row + c0;
    Pack<TE, V> v[U];
    if (some) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 32 * V < p.d) v[u] = get<TE, V>(e + u * 32 * V);
    } else {
      const float zero[V] = {};
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 32 * V < p.d) put<TO, V>(o + u * 32 * V, zero);
      tok = coming;
      continue;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * 32 * V < p.d) {
        float x[V];
        v[u].get(x);
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] *= p.scale;
        put<TO, V>(o + u * 32 * V, x);
      }
    tok = coming;
  }
}

// Block (x, i, part) lists those positions of the table rows [lo, hi) of agent i that lie in a part of the agent's tokens.
// It counts the row's tokens before, in and after the part, and those below lo, which is where its rows' lists
// begin; then it places its part's.  A warp owns a contiguous segment of the part and takes it in order, so a list is
// ascending; nothing is exchanged between blocks.  Counting all tokens in every block is cheap; placing them is not (ranks
// among the lanes of a warp, stores anywhere), and frequent tokens lie together in one block: parts divide that.
template <typename TI>
__global__ void __launch_bounds__(kListThreads) token_list_kernel(const EmbedArgs p) {
  extern __shared__ __align__(16) int32_t count[];   // [kListWarps + 2][pitch]: of each warp, before and after the part
  __shared__ int32_t sums[kListWarps], below_all;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = blockIdx.y;
  const int64_t lo = (int64_t)blockIdx.x * p.bins;
  const int32_t bins = (int32_t)min((int64_t)p.bins, p.v - lo), pitch = (p.bins + 3) & ~3;
  const TI *tok = static_cast<const TI *>(p.tokens) + i * p.tokens_agent;
  const int64_t p0 = min(p.t, blockIdx.z * p.part), p1 = min(p.t, p0 + p.part);
  const int64_t seg = p.part / kListWarps, s0 = min(p1, p0 + warp * seg), s1 = min(p1, s0 + seg);
  int32_t *mine = count + warp * pitch, *before = count + kListWarps * pitch, *after = before + pitch;

  for (int k = threadIdx.x; k < (kListWarps + 2) * pitch / 4; k += kListThreads) reinterpret_cast<int4 *>(count)[k] = make_int4(0, 0, 0, 0);
  if (threadIdx.x == 0) below_all = 0;
  __syncthreads();
  // (compared as unsigned numbers: negative tokens lie above every row)
  using U = typename std::make_unsigned<TI>::type;
  const U ulo = (U)lo, ubins = (U)bins;
  int32_t below = 0;
  const auto tally = [&](int64_t s, int32_t *counts) {
    const U w = (U)tok[s], r = w - ulo;
    below += w < ulo;
    if (r < ubins) atomicAdd(counts + r, 1);
  };
#pragma unroll 8
  for (int64_t s = s0 + lane; s < s1; s += 32) tally(s, mine);
#pragma unroll 4
  for (int64_t s = threadIdx.x; s < p0; s += kListThreads) tally(s, before);
#pragma unroll 4
  for (int64_t s = p1 + threadIdx.x; s < p.t; s += kListThreads) tally(s, after);
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) atomicAdd(&below_all, below);
  __syncthreads();

  // counts become the places where each (row, warp) begins: exclusive sums over the rows, warps within
  const int r = threadIdx.x;
  int32_t sum = 0;
  if (r < bins)
#pragma unroll 8
    for (int w = 0; w < kListWarps + 2; ++w) sum += count[w * pitch + r];
  int32_t upto = sum;
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  int32_t lower = lane < warp ? sums[lane] : 0;
  lower = __reduce_add_sync(0xffffffffu, lower);
  int32_t at = below_all + lower + upto - sum;
  if (r < bins) {
    if (blockIdx.z == 0) {
      int32_t *start = p.row_start + i * (p.v + 1) + lo;
      start[r] = at;
      if (r == bins - 1 && lo + bins == p.v) start[bins] = at + sum;
    }
    at += before[r];
#pragma unroll 8
    for (int w = 0; w < kListWarps; ++w) {
      const int32_t c = count[w * pitch + r];
      count[w * pitch + r] = at;
      at += c;
    }
  }
  __syncthreads();

  int2 *list = p.list + i * p.t;
  constexpr int kAhead = 8;   // groups of 32 tokens on their way at a time
  for (int64_t s = s0; s < s1; s += 32 * kAhead) {
    U w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) w[k] = s + 32 * k + lane < s1 ? (U)tok[s + 32 * k + lane] - ulo : ubins;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool in = w[k] < ubins;
      const uint32_t some = __ballot_sync(0xffffffffu, in);
      if (some == 0) continue;
      if (in) {
        const int32_t row = (int32_t)w[k];
        const uint32_t same = __match_any_sync(some, row);
        const int32_t rank = __popc(same & ((1u << lane) - 1)), place = mine[row] + rank;
        list[place] = make_int2((int32_t)(s + 32 * k + lane), (int32_t)lo + row);
        __syncwarp(some);
        if (rank == 0) mine[row] += __popc(same);
      }
      __syncwarp();
    }
  }
}

// The slice's packs of a finished row.
template <typename TE, int V> __device__ __forceinline__ void finish_row(const EmbedArgs &p, TE *g, int64_t c0, float (*acc)[V]) {
#pragma unroll
  for (int u = 0; u < Slice<V>::U; ++u)
    if (c0 + u * 32 * V < p.d) {
      float x[V];
#pragma unroll
      for (int k = 0; k < V; ++k) x[k] = acc[u][k] * p.scale;
      if (p.accumulate) add_to(x, get<TE, V>(g + u * 32 * V));
      put<TE, V>(g + u * 32 * V, x);
    }
}

// Zeros for the columns [c, c + count) of a row, by a warp: rows on any boundary get 16 bytes at a time too.
template <typename TE, int V> __device__ __forceinline__ void zero_row(TE *g, int64_t count) {
  const int lane = threadIdx.x & 31;
  if (V > 1) {
    const float zero[V] = {};
    for (int64_t c = lane * V; c < count; c += 32 * V) put<TE, V>(g + c, zero);
    return;
  }
  const int64_t head = min(count, (int64_t)((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / (int64_t)sizeof(TE));
  constexpr int N = 16 / sizeof(TE);
  const int64_t whole = (count - head) / N, tail = head + whole * N;
  if (lane < head) narrow(g + lane, 0.f);
  for (int64_t k = lane; k < whole; k += 32) reinterpret_cast<uint4 *>(g + head)[k] = make_uint4(0, 0, 0, 0);
  if (tail + lane < count) narrow(g + tail + lane, 0.f);
}

// Block (x, slice, agent): kFewRows rows, a warp each in turn, for agents with at most kFew positions.
template <typename TE, typename TO, typename TI, int V> __global__ void __launch_bounds__(kThreads) embed_few_kernel(const EmbedArgs p) {
  constexpr int U = Slice<V>::U;
  __shared__ int32_t tok[kFew];
  __shared__ uint8_t places[kWarps][kFew];   // a row's positions
  __shared__ uint32_t present;   // which of the rows have positions
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = blockIdx.z, r0 = (int64_t)blockIdx.x * kFewRows;
  const int64_t c0 = (int64_t)blockIdx.y * Slice<V>::kElements + lane * V;
  if (threadIdx.x == 0) present = 0;
  __syncthreads();
  const int64_t w = threadIdx.x < p.t ? (int64_t) static_cast<const TI *>(p.tokens)[i * p.tokens_agent + threadIdx.x] : -1;
  const bool here = w >= r0 && w < min(p.v, r0 + kFewRows);
  tok[threadIdx.x] = here ? (int32_t)(w - r0) : -1;
  if (here) atomicOr(&present, 1u << (w - r0));
  __syncthreads();
  const uint32_t some = present;
  const TO *o = static_cast<const TO *>(p.src) + i * p.out_agent + c0;
  for (int r = warp; r < kFewRows && r0 + r < p.v; r += kWarps) {
    TE *g = static_cast<TE *>(p.dst) + i * p.table_agent + (r0 + r) * p.table_row;
    if (!(some >> r & 1)) {
      const int64_t first = (int64_t)blockIdx.y * Slice<V>::kElements;
      if (!p.accumulate) zero_row<TE, V>(g + first, min((int64_t)Slice<V>::kElements, p.d - first));
      continue;
    }
    float acc[U][V] = {};
    int count = 0;
    for (int k = 0; k < p.t; k += 32) {
      const bool mine = tok[k + lane] == r;
      const uint32_t them = __ballot_sync(0xffffffffu, mine);
      if (mine) places[warp][count + __popc(them & ((1u << lane) - 1))] = (uint8_t)(k + lane);
      count += __popc(them);
    }
    __syncwarp();
    for (int s = 0; s < count; s += kDeep) {
      Pack<TO, V> v[kDeep][U];
#pragma unroll
      for (int q = 0; q < kDeep; ++q)
        if (s + q < count)
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (c0 + u * 32 * V < p.d) v[q][u] = get<TO, V>(o + places[warp][s + q] * p.out_row + u * 32 * V);
#pragma unroll
      for (int q = 0; q < kDeep; ++q)
        if (s + q < count)
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (c0 + u * 32 * V < p.d) add_to(acc[u], v[q][u]);
    }
    __syncwarp();
    finish_row<TE, V>(p, g + c0, c0, acc);
  }
}

// The sum of `count` entries, a contiguous share of them by each warp of a CTA; warp 0 ends up with it in `acc`.  `add(j)` adds
// entry j's packs to acc.
template <int V, typename Add> __device__ __forceinline__ void sum_by_warps(float (*acc)[V], int count, float (*shared)[Slice<V>::kElements], Add add) {
  constexpr int U = Slice<V>::U;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (count + kWarps - 1) / kWarps, from = min(count, warp * per), to = min(count, from + per);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < V; ++k) acc[u][k] = 0.f;
#pragma unroll 4
  for (int j = from; j < to; ++j) add(j);
  __syncthreads();   // the last sum has been read
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < V; ++k) shared[warp][(u * V + k) * 32 + lane] = acc[u][k];
  __syncthreads();
  if (warp == 0)
    for (int w = 1; w < kWarps; ++w)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < V; ++k) acc[u][k] += shared[w][(u * V + k) * 32 + lane];
}

// Blocks (x, slice, agent): first a chunk for each warp, then kFill rows for each CTA.
template <typename TE, typename TO, int V> __global__ void __launch_bounds__(kThreads, 2) embed_grad_kernel(const EmbedArgs p) {
  constexpr int U = Slice<V>::U;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = blockIdx.z;
  const int64_t c0 = (int64_t)blockIdx.y * Slice<V>::kElements + lane * V;
  const int32_t *start = p.row_start + i * (p.v + 1);
  const int2 *list = p.list + i * p.t;
  TE *table = static_cast<TE *>(p.dst) + i * p.table_agent + c0;
  const int work = gridDim.x - p.fills;
  if ((int)blockIdx.x >= work) {
    const int64_t r0 = (int64_t)(blockIdx.x - work) * kFill;
    constexpr int kRows = kFill / kWarps;   // of each warp: warp, warp + kWarps, ...
    const int64_t row = r0 + warp + lane * kWarps;
    const bool empty = lane < kRows && row < p.v && start[row] == start[row + 1];
    uint32_t todo = __ballot_sync(0xffffffffu, empty);
    const int64_t width = min((int64_t)Slice<V>::kElements, p.d - (int64_t)blockIdx.y * Slice<V>::kElements);
    for (; todo; todo &= todo - 1)
      zero_row<TE, V>(table - lane * V + (r0 + warp + (__ffs(todo) - 1) * kWarps) * p.table_row, width);
    return;
  }
  const int j = blockIdx.x * kWarps + warp, chunk = p.chunk;
  const int32_t total = start[p.v], from = j * chunk, to = min(from + chunk, total);
  if (from >= total) return;
  // the chunk's places and the next ones, for a row that goes on there; each lane knows where its place's row begins and ends
  const int32_t place0 = from + lane < total ? list[from + lane].x : 0, place1 = from + 32 + lane < total ? list[from + 32 + lane].x : 0;
  const int32_t w = list[min(from + lane, to - 1)].y;
  const int32_t begin = start[w], end = start[w + 1];
  const TO *o = static_cast<const TO *>(p.src) + i * p.out_agent + c0;
  // the places [s0, s1) are this warp's: not those of a whole row that the warp of the chunk before has, but all of a whole
  // row that goes on after the chunk
  const int32_t b0 = __shfl_sync(0xffffffffu, begin, 0), e0 = __shfl_sync(0xffffffffu, end, 0);
  const int32_t bl = __shfl_sync(0xffffffffu, begin, 31), el = __shfl_sync(0xffffffffu, end, 31);
  const int32_t s0 = b0 < from && e0 - b0 <= chunk ? min(e0, to) : from;
  const int32_t s1 = el - bl > chunk || bl < from ? to : el;
  float acc[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < V; ++k) acc[u][k] = 0.f;
  for (int32_t s = s0; s < s1; s += kDeep) {
    Pack<TO, V> v[kDeep][U];
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
      const int32_t k = s + q - from, p0 = __shfl_sync(0xffffffffu, place0, k & 31), p1 = __shfl_sync(0xffffffffu, place1, k & 31);
      const TO *r = o + (k < 32 ? p0 : p1) * p.out_row;
      if (s + q < s1)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * 32 * V < p.d) v[q][u] = get<TO, V>(r + u * 32 * V);
    }
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
      if (s + q >= s1) break;
      const int k = min(s + q, to - 1) - from;   // a place after the chunk is of the chunk's last row
      const int32_t b = __shfl_sync(0xffffffffu, begin, k), e = __shfl_sync(0xffffffffu, end, k), row = __shfl_sync(0xffffffffu, w, k);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 32 * V < p.d) add_to(acc[u], v[q][u]);
      if (s + q + 1 < e && s + q + 1 < s1) continue;   // the row, or its piece, goes on
      if (e - b > chunk) {   // a piece: [0] where it begins the chunk, [1] where it only ends it
        float *out = p.pieces + ((i * p.chunks + j) * 2 + (b > from)) * p.d + c0;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int x = 0; x < V; ++x)
            if (c0 + u * 32 * V < p.d) out[u * 32 * V + x] = acc[u][x];
      } else {
        finish_row<TE, V>(p, table + row * p.table_row, c0, acc);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int x = 0; x < V; ++x) acc[u][x] = 0.f;
    }
  }
}

// Block (x, slice, agent): the rows with several pieces whose lists begin in the chunks [x kJoin, (x + 1) kJoin).  Such a row
// ends its chunk.
template <typename TE, int V> __global__ void __launch_bounds__(kThreads) embed_join_kernel(const EmbedArgs p) {
  constexpr int U = Slice<V>::U;
  __shared__ float shared[kWarps][Slice<V>::kElements];
  const int64_t i = blockIdx.z;
  const int lane = threadIdx.x & 31;
  const int32_t *start = p.row_start + i * (p.v + 1);
  const int32_t total = start[p.v], mine = ((int)blockIdx.x * kJoin + lane) * p.chunk;
  int32_t w = 0, b = 0, e = 0;
  if (lane < kJoin && mine < total) {
    w = p.list[i * p.t + min(mine + p.chunk, total) - 1].y;
    b = start[w];
    e = start[w + 1];
  }
  uint32_t todo = __ballot_sync(0xffffffffu, e - b > p.chunk && b >= mine);   // the same in every warp
  const int64_t c0 = (int64_t)blockIdx.y * Slice<V>::kElements + lane * V;
  for (; todo; todo &= todo - 1) {
    const int k0 = __ffs(todo) - 1, j = blockIdx.x * kJoin + k0;
    const int32_t row = __shfl_sync(0xffffffffu, w, k0), from = __shfl_sync(0xffffffffu, b, k0), to = __shfl_sync(0xffffffffu, e, k0);
    const float *pieces = p.pieces + (i * p.chunks + j) * 2 * p.d + c0;
    float acc[U][V];
    sum_by_warps<V>(acc, (to - 1) / p.chunk - j + 1, shared, [&](int k) {
      const float *r = pieces + (2 * (int64_t)k + (k == 0 && from > j * p.chunk)) * p.d;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q)
          if (c0 + u * 32 * V < p.d) acc[u][q] += r[u * 32 * V + q];
    });
    if (threadIdx.x < 32) finish_row<TE, V>(p, static_cast<TE *>(p.dst) + i * p.table_agent + row * p.table_row + c0, c0, acc);
  }
}

// How the list kernel is split: into parts of the tokens (of 4096 at least: each counts all of them) as far as two blocks an
// SM allow, then into ranges of table rows, which are at most kMaxBins.
struct ListSplit { int32_t bins, parts; };
ListSplit list_split(int32_t n, int64_t t, int64_t v) {
  const int64_t room = 2 * 148 / n, least = ceil_div(v, kMaxBins);
  const int64_t parts = std::max<int64_t>(1, std::min({room / least, ceil_div(t, 4096), (int64_t)8}));
  const int64_t blocks = std::max<int64_t>({least, room / parts, 1});
  return {(int32_t)ceil_div(v, blocks), (int32_t)parts};
}

// Places of a chunk: 32, or fewer where that would leave the SMs without work.
int32_t chunk_of(int32_t n, int64_t t, int64_t d) {
  int32_t c = 32;
  while (c > 8 && n * ceil_div(t, c) * ceil_div(d, 512) < 16 * 148) c /= 2;
  return c;
}

size_t round16(size_t bytes) { return (bytes + 15) / 16 * 16; }

bool embed_args_ok(int32_t n, int64_t t, int64_t v, int64_t d, int64_t table_agent, int64_t table_row,
                   int64_t tokens_agent, int64_t out_agent, int64_t out_row, int32_t table_type,
                   int32_t tokens_type, int32_t out_type) {
  // (places and positions are 32-bit numbers, up to a few chunks beyond t)
  return n >= 1 && n <= 65535 && t >= 0 && t < ((int64_t)1 << 31) - 1024 && v >= 1 && v < ((int64_t)1 << 31) && d >= 1 && d < ((int64_t)1 << 31) &&
         table_agent >= 0 && table_row >= d && tokens_agent >= 0 && out_agent >= 0 && out_row >= 0 &&
         is_type(table_type) && is_index(tokens_type) && is_type(out_type);
}

// Elements of a pack: both tensors' packs must lie on a boundary of their own size.
int pack_of(const EmbedArgs &p, const void *table, int64_t te, const void *out, int64_t to) {
  const auto fits = [&](int v, const void *base, int64_t agent, int64_t row, int64_t size) {
    return (uintptr_t)base % (v * size) == 0 && (p.n == 1 || agent % v == 0) && row % v == 0;
  };
  for (int v = te == 2 && to == 2 ? 8 : 4; v >= 4; v /= 2)
    if (p.d % v == 0 && fits(v, table, p.table_agent, p.table_row, te) && fits(v, out, p.out_agent, p.out_row, to)) return v;
  return 1;
}

template <typename TE, typename TO, typename TI, int V> cudaError_t launch_lookup(EmbedArgs p, cudaStream_t s) {
  p.slices = (int32_t)ceil_div(p.d, 32 * kLookupPacks<V> * V);
  const int64_t units = (int64_t)p.n * p.t * p.slices;
  const int grid = (int)std::min<int64_t>(ceil_div(units, kWarps), (int64_t)sm_count() * 8);
  embed_lookup_kernel<TE, TO, TI, V><<<grid, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

template <typename TI> cudaError_t launch_list(const EmbedArgs &p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto bytes = [](int bins) { return (int)sizeof(int32_t) * (kListWarps + 2) * ((bins + 3) / 4 * 4); };
  const cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(token_list_kernel<TI>), bytes(kMaxBins), &done);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)ceil_div(p.v, p.bins), (unsigned)p.n, (unsigned)ceil_div(p.t, p.part));
  token_list_kernel<TI><<<grid, kListThreads, bytes(p.bins), s>>>(p);
  return cudaGetLastError();
}

template <typename TE, typename TO, typename TI, int V> cudaError_t launch_grad(EmbedArgs p, cudaStream_t s) {
  p.slices = (int32_t)ceil_div(p.d, Slice<V>::kElements);
  if (p.t <= kFew) {
    embed_few_kernel<TE, TO, TI, V><<<dim3((unsigned)ceil_div(p.v, kFewRows), p.slices, p.n), kThreads, 0, s>>>(p);
    return cudaGetLastError();
  }
  const cudaError_t listed = launch_list<TI>(p, s);
  if (listed != cudaSuccess) return listed;
  p.fills = p.accumulate ? 0 : (int32_t)ceil_div(p.v, kFill);
  const unsigned blocks = (unsigned)(ceil_div(p.chunks, kWarps) + p.fills);
  if (blocks > 0) embed_grad_kernel<TE, TO, V><<<dim3(blocks, p.slices, p.n), kThreads, 0, s>>>(p);
  if (p.chunks > 1) embed_join_kernel<TE, V><<<dim3((unsigned)ceil_div(p.chunks, kJoin), p.slices, p.n), kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

// Calls go(TE, TO, TI, V) for the types of a call.
template <typename TE, typename TO, typename Go> cudaError_t with_index(bool i64, int pack, Go go) {
  const auto with_pack = [&](auto ti) {
    if (pack == 1) return go(TE(), TO(), ti, std::integral_constant<int, 1>());
    if constexpr (sizeof(TE) == 2 && sizeof(TO) == 2)
      if (pack == 8) return go(TE(), TO(), ti, std::integral_constant<int, 8>());
    return go(TE(), TO(), ti, std::integral_constant<int, 4>());
  };
  return i64 ? with_pack(int64_t()) : with_pack(int32_t());
}
template <typename Go> ceca_status_t with_types(int32_t te, int32_t to, int32_t ti, int pack, Go go) {
  const bool i64 = ti == DSGD_I64;
  cudaError_t e;
  if (te == DSGD_F32) e = to == DSGD_F32 ? with_index<float, float>(i64, pack, go) : with_index<float, bf16>(i64, pack, go);
  else e = to == DSGD_F32 ? with_index<bf16, float>(i64, pack, go) : with_index<bf16, bf16>(i64, pack, go);
  return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" ceca_status_t dsgd_embed_lookup(const void *E, const void *tokens, void *out, int32_t n, int64_t t,
                                           int64_t v, int64_t d, int64_t agent_stride, int64_t row_stride,
                                           int64_t tokens_stride, int64_t out_agent_stride, int64_t out_row_stride,
                                           int32_t table_type, int32_t tokens_type, int32_t out_type, float scale,
                                           void *stream) {
  if (!embed_args_ok(n, t, v, d, agent_stride, row_stride, tokens_stride, out_agent_stride, out_row_stride,
                     table_type, tokens_type, out_type) ||
      out_row_stride < d || (n > 1 && t > 0 && out_agent_stride == 0))
    return CECA_ERR_INVALID_ARG;
  if (t == 0) return CECA_OK;
  if (!E || !tokens || !out) return CECA_ERR_INVALID_ARG;
  EmbedArgs p{};
  p.src = E; p.dst = out; p.tokens = tokens;
  p.t = t; p.v = v; p.d = d; p.n = n;
  p.table_agent = agent_stride; p.table_row = row_stride; p.tokens_agent = tokens_stride;
  p.out_agent = out_agent_stride; p.out_row = out_row_stride; p.scale = scale;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int pack = pack_of(p, E, type_bytes(table_type), out, type_bytes(out_type));
  return with_types(table_type, out_type, tokens_type, pack, [&](auto te, auto to, auto ti, auto v) {
    return launch_lookup<decltype(te), decltype(to), decltype(ti), v.value>(p, s);
  });
}

extern "C" size_t dsgd_embed_workspace_bytes(int32_t n, int64_t t, int64_t v, int64_t d) {
  if (!embed_args_ok(n, t, v, d, 0, d, 0, 0, d, DSGD_F32, DSGD_I32, DSGD_F32) || t <= kFew || d > kMaxWidth) return 0;
  return round16(sizeof(int32_t) * (size_t)n * (size_t)(v + 1)) + round16(sizeof(int2) * (size_t)n * (size_t)t) +
         sizeof(float) * 2 * (size_t)n * (size_t)ceil_div(t, chunk_of(n, t, d)) * (size_t)d;
}

extern "C" ceca_status_t dsgd_embed_grad(const void *dout, const void *tokens, void *dE, int32_t n, int64_t t,
                                         int64_t v, int64_t d, int64_t agent_stride, int64_t row_stride,
                                         int64_t tokens_stride, int64_t out_agent_stride, int64_t out_row_stride,
                                         int32_t table_type, int32_t tokens_type, int32_t out_type, float scale,
                                         int32_t accumulate, void *workspace, size_t workspace_bytes, void *stream) {
  if (!embed_args_ok(n, t, v, d, agent_stride, row_stride, tokens_stride, out_agent_stride, out_row_stride,
                     table_type, tokens_type, out_type) ||
      !dE || (t > 0 && (!dout || !tokens)) || (n > 1 && agent_stride < (v - 1) * row_stride + d))
    return CECA_ERR_INVALID_ARG;
  if (d > kMaxWidth) return CECA_ERR_UNSUPPORTED;
  const size_t need = dsgd_embed_workspace_bytes(n, t, v, d);
  if (need > 0 && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16)) return CECA_ERR_WORKSPACE;
  EmbedArgs p{};
  p.src = dout; p.dst = dE; p.tokens = tokens;
  p.t = t; p.v = v; p.d = d; p.n = n;
  p.table_agent = agent_stride; p.table_row = row_stride; p.tokens_agent = tokens_stride;
  p.out_agent = out_agent_stride; p.out_row = out_row_stride; p.scale = scale; p.accumulate = accumulate != 0;
  p.row_start = static_cast<int32_t *>(workspace);
  p.list = reinterpret_cast<int2 *>(static_cast<char *>(workspace) + round16(sizeof(int32_t) * (size_t)n * (size_t)(v + 1)));
  p.pieces = reinterpret_cast<float *>(reinterpret_cast<char *>(p.list) + round16(sizeof(int2) * (size_t)n * (size_t)t));
  const ListSplit split = list_split(n, t, v);
  p.bins = split.bins;
  p.part = std::max<int64_t>(1, ceil_div(t, (int64_t)split.parts * kListThreads)) * kListThreads;
  p.chunk = chunk_of(n, t, d);
  p.chunks = (int32_t)ceil_div(t, p.chunk);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int pack = pack_of(p, dE, type_bytes(table_type), dout, type_bytes(out_type));
  return with_types(table_type, out_type, tokens_type, pack, [&](auto te, auto to, auto ti, auto v) {
    return launch_grad<decltype(te), decltype(to), decltype(ti), v.value>(p, s);
  });
}
