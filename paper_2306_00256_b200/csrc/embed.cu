// Token embedding of n agents and its gradient.
//
//   out[i, s, :] = scale E_i[tok[i, s], :]          dE_i[w, :] = scale sum_{s : tok[i, s] = w} dout[i, s, :]
//
// Both directions move rows and do one multiplication or addition per element, so bytes bound them.  The
// gradient lists every table row's positions in ascending order (token_list_kernel), then each row of dE is
// summed over its list and written once (embed_grad_kernel): no atomics on values, one order of additions.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

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
  int32_t *list;       // n x t: positions, by token and then ascending
  int32_t bins;        // table rows per block of token_list_kernel
};

constexpr int kLookupThreads = 256;
constexpr int kListThreads = 512;
constexpr int kListWarps = kListThreads / 32;
constexpr int kMaxBins = 2048;

template <typename TE, typename TO, typename TI>
__global__ void __launch_bounds__(kLookupThreads) embed_lookup_kernel(const EmbedArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)p.n * p.t;
  const int64_t step = (int64_t)gridDim.x * (kLookupThreads / 32);
  for (int64_t row = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); row < rows; row += step) {
    const int64_t i = row / p.t, s = row - i * p.t;
    const int64_t tok = static_cast<const TI *>(p.tokens)[i * p.tokens_agent + s];
    TO *o = static_cast<TO *>(p.dst) + i * p.out_agent + s * p.out_row;
    const bool some = tok >= 0 && tok < p.v;
    const TE *e = static_cast<const TE *>(p.src) + i * p.table_agent + (some ? tok : 0) * p.table_row;
    for (int64_t c = lane; c < p.d; c += 32) narrow(o + c, some ? p.scale * widen(e[c]) : 0.f);
  }
}

// Block (x, i) lists the positions of the table rows [lo, hi) of agent i.  It scans all of the agent's tokens
// twice: once to count them per (warp, row) and to count those below lo, which is where its part of the list
// begins, and once to place them.  A warp owns a contiguous segment of the positions and takes it in order, so
// the list is ascending within a row; nothing is exchanged between blocks.
template <typename TI>
__global__ void __launch_bounds__(kListThreads) token_list_kernel(const EmbedArgs p) {
  extern __shared__ int32_t count[];   // [kListWarps][bins]
  __shared__ int32_t part[kListWarps], below_all;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = blockIdx.y;
  const int64_t lo = (int64_t)blockIdx.x * p.bins;
  const int32_t bins = (int32_t)min((int64_t)p.bins, p.v - lo);
  const TI *tok = static_cast<const TI *>(p.tokens) + i * p.tokens_agent;
  const int64_t seg = (p.t + kListThreads - 1) / kListThreads * 32;
  const int64_t s0 = warp * seg, s1 = min(p.t, s0 + seg);
  int32_t *mine = count + warp * p.bins;

  for (int k = threadIdx.x; k < kListWarps * p.bins; k += kListThreads) count[k] = 0;
  if (threadIdx.x == 0) below_all = 0;
  __syncthreads();
  int32_t below = 0;
  for (int64_t s = s0 + lane; s < s1; s += 32) {
    const int64_t w = tok[s];
    below += w >= 0 && w < lo;
    if (w >= lo && w < lo + bins) atomicAdd(mine + (w - lo), 1);
  }
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) atomicAdd(&below_all, below);
  __syncthreads();

  // counts become the places where each (row, warp) begins: exclusive sums over the rows, warps within
  constexpr int kPer = kMaxBins / kListThreads;
  int32_t sum = 0;
  for (int j = 0; j < kPer; ++j) {
    const int r = threadIdx.x * kPer + j;
    if (r < bins)
      for (int w = 0; w < kListWarps; ++w) sum += count[w * p.bins + r];
  }
  int32_t upto = sum;
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) part[warp] = upto;
  __syncthreads();
  int32_t at = below_all + upto - sum;
  for (int w = 0; w < warp; ++w) at += part[w];
  int32_t *start = p.row_start + i * (p.v + 1) + lo;
  for (int j = 0; j < kPer; ++j) {
    const int r = threadIdx.x * kPer + j;
    if (r < bins) {
      start[r] = at;
      for (int w = 0; w < kListWarps; ++w) {
        const int32_t c = count[w * p.bins + r];
        count[w * p.bins + r] = at;
        at += c;
      }
      if (r == bins - 1 && lo + bins == p.v) start[bins] = at;
    }
  }
  __syncthreads();

  int32_t *list = p.list + i * p.t;
  for (int64_t s = s0; s < s1; s += 32) {
    const int64_t w = s + lane < s1 ? (int64_t)tok[s + lane] : -1;
    const bool in = w >= lo && w < lo + bins;
    const uint32_t some = __ballot_sync(0xffffffffu, in);
    if (in) {
      const int32_t r = (int32_t)(w - lo);
      const uint32_t same = __match_any_sync(some, r);
      const int32_t rank = __popc(same & ((1u << lane) - 1));
      list[mine[r] + rank] = (int32_t)(s + lane);
      __syncwarp(some);
      if (rank == 0) mine[r] += __popc(same);
    }
    __syncwarp();
  }
}

template <typename TE, typename TO>
__global__ void __launch_bounds__(kLookupThreads) embed_grad_kernel(const EmbedArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)p.n * p.v;
  const int64_t step = (int64_t)gridDim.x * (kLookupThreads / 32);
  for (int64_t row = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); row < rows; row += step) {
    const int64_t i = row / p.v, w = row - i * p.v;
    const int32_t *start = p.row_start + i * (p.v + 1) + w;
    const int32_t b = start[0], e = start[1];
    if (p.accumulate && b == e) continue;
    const int32_t *list = p.list + i * p.t;
    const TO *o = static_cast<const TO *>(p.src) + i * p.out_agent;
    TE *g = static_cast<TE *>(p.dst) + i * p.table_agent + w * p.table_row;
    for (int64_t c = lane; c < p.d; c += 32) {
      float acc = 0.f;
      for (int32_t j = b; j < e; ++j) acc += widen(o[list[j] * p.out_row + c]);
      acc *= p.scale;
      if (p.accumulate) acc += widen(g[c]);
      narrow(g + c, acc);
    }
  }
}

// Table rows per list block: at most kMaxBins (its counters then fill 128 KB), and so few that the blocks of
// all agents cover the GPU.
int32_t list_bins(int32_t n, int64_t v) {
  const int64_t blocks = std::max<int64_t>(ceil_div(v, kMaxBins), ceil_div(2 * 148, n));
  return (int32_t)std::max<int64_t>(1, ceil_div(v, blocks));
}

size_t round16(size_t bytes) { return (bytes + 15) / 16 * 16; }

bool embed_args_ok(int32_t n, int64_t t, int64_t v, int64_t d, int64_t table_agent, int64_t table_row,
                   int64_t tokens_agent, int64_t out_agent, int64_t out_row, int32_t table_type,
                   int32_t tokens_type, int32_t out_type) {
  return n >= 1 && n <= 65535 && t >= 0 && t < ((int64_t)1 << 31) && v >= 1 && v < ((int64_t)1 << 31) && d >= 1 &&
         table_agent >= 0 && table_row >= d && tokens_agent >= 0 && out_agent >= 0 && out_row >= 0 &&
         is_type(table_type) && is_index(tokens_type) && is_type(out_type);
}

int grid_of(int64_t rows) {
  return (int)std::min<int64_t>(ceil_div(rows, kLookupThreads / 32), (int64_t)sm_count() * 8);
}

template <typename TE, typename TO> void launch_lookup(const EmbedArgs &p, bool i64, cudaStream_t s) {
  const int g = grid_of((int64_t)p.n * p.t);
  if (i64) embed_lookup_kernel<TE, TO, int64_t><<<g, kLookupThreads, 0, s>>>(p);
  else embed_lookup_kernel<TE, TO, int32_t><<<g, kLookupThreads, 0, s>>>(p);
}

template <typename TE, typename TO> void launch_grad(const EmbedArgs &p, cudaStream_t s) {
  embed_grad_kernel<TE, TO><<<grid_of((int64_t)p.n * p.v), kLookupThreads, 0, s>>>(p);
}

template <typename TI> cudaError_t launch_list(const EmbedArgs &p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(token_list_kernel<TI>),
                                            sizeof(int32_t) * kListWarps * kMaxBins, &done);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)ceil_div(p.v, p.bins), (unsigned)p.n);
  token_list_kernel<TI><<<grid, kListThreads, sizeof(int32_t) * kListWarps * p.bins, s>>>(p);
  return cudaGetLastError();
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
  const bool i64 = tokens_type == DSGD_I64;
  if (table_type == DSGD_F32) {
    if (out_type == DSGD_F32) launch_lookup<float, float>(p, i64, s);
    else launch_lookup<float, bf16>(p, i64, s);
  } else {
    if (out_type == DSGD_F32) launch_lookup<bf16, float>(p, i64, s);
    else launch_lookup<bf16, bf16>(p, i64, s);
  }
  return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

extern "C" size_t dsgd_embed_workspace_bytes(int32_t n, int64_t t, int64_t v, int64_t d) {
  if (!embed_args_ok(n, t, v, d, 0, d, 0, 0, d, DSGD_F32, DSGD_I32, DSGD_F32)) return 0;
  return round16(sizeof(int32_t) * (size_t)n * (size_t)(v + 1)) + round16(sizeof(int32_t) * (size_t)n * (size_t)t);
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
  if (!workspace || workspace_bytes < dsgd_embed_workspace_bytes(n, t, v, d) || (uintptr_t)workspace % 16)
    return CECA_ERR_WORKSPACE;
  EmbedArgs p{};
  p.src = dout; p.dst = dE; p.tokens = tokens;
  p.t = t; p.v = v; p.d = d; p.n = n;
  p.table_agent = agent_stride; p.table_row = row_stride; p.tokens_agent = tokens_stride;
  p.out_agent = out_agent_stride; p.out_row = out_row_stride; p.scale = scale; p.accumulate = accumulate != 0;
  p.row_start = static_cast<int32_t *>(workspace);
  p.list = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + round16(sizeof(int32_t) * (size_t)n * (size_t)(v + 1)));
  p.bins = list_bins(n, v);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((tokens_type == DSGD_I64 ? launch_list<int64_t>(p, s) : launch_list<int32_t>(p, s)) != cudaSuccess)
    return CECA_ERR_CUDA;
  if (table_type == DSGD_F32) {
    if (out_type == DSGD_F32) launch_grad<float, float>(p, s);
    else launch_grad<float, bf16>(p, s);
  } else {
    if (out_type == DSGD_F32) launch_grad<bf16, float>(p, s);
    else launch_grad<bf16, bf16>(p, s);
  }
  return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}
