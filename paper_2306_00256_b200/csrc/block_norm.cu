// The end of a block and the start of the next, row by row, and its gradient.
//
//   h_out = h + s g(a) w_post y rho,  u = w_pre h_out r,  rho = 1 / rms(y),  r = 1 / rms(h_out)
//   D = dh_out + r (w_pre du - hn mean(hn w_pre du)),  hn = h_out r,  yn = y rho
//   dy = rho (e - yn mean(yn e)),  e = s g w_post D,  da = s g'(a) w_post yn D
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "block_norm.cuh"
#include "tma.h"

namespace ceca {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// The sum over a CTA, in one order.
__device__ __forceinline__ float cta_sum(float x) {
  __shared__ float part[kWarps];
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) x += part[i];
  return x;
}

// ---------------------------------------------------------------------------------------------- rows of any width
// What block_rows.cuh does not hold.  A CTA works on a row, channel by channel, and reads it once for each thing that it sums; the gradient's sums over rows
// are taken by a kernel of their own.  (2 x 2048 x 9000 bf16: 0.6 ms forward, 3.1 ms for the gradient.)

struct Gate {
  float g, slope;
};
struct Row {
  const BlockArgs &p;
  int64_t agent, row, h, y, gate;
  float scale;
  __device__ Row(const BlockArgs &p, int64_t i) : p(p), agent(i / p.t), row(i - agent * p.t) {
    if (p.kept) {
      h = y = gate = i * p.row_bytes;
    } else {
      h = place(p.h, agent, row);
      y = place(p.y, agent, row);
      gate = place(p.gate, agent, row);
    }
    scale = p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f;
  }
  __device__ float value(const dsgd_rows_t &x, int64_t at, int32_t type, int64_t c) const {
    if (!p.kept) return load(x.at, type, at + c);
    const uint8_t *q = static_cast<const uint8_t *>(x.at) + at;
    return (float)(int8_t)q[c] * step8(q[p.d + c / kBlock8]);
  }
  __device__ float h_at(int64_t c) const { return value(p.h, h, p.stream_type, c); }
  __device__ float y_at(int64_t c) const { return value(p.y, y, p.act_type, c); }
  __device__ float gate_at(int64_t c) const { return value(p.gate, gate, p.act_type, c); }
  __device__ Gate g(int64_t c) const {
    if (!p.gate.at) return {1.f, 0.f};
    const Gates x = gates_of(all<2>(gate_at(c)), p.silu);
    return {x.g.x, x.slope.x};
  }
  __device__ float w_pre(int64_t c) const { return load(p.w_pre, p.weights_type, agent * p.w_pre_stride + c); }
  __device__ float w_post(int64_t c) const { return load(p.w_post, p.weights_type, agent * p.w_post_stride + c); }
  __device__ float out(int64_t c, float rho) const {
    return p.y.at ? fmaf(scale * g(c).g * w_post(c), y_at(c) * rho, h_at(c)) : h_at(c);
  }
};

__device__ void keep(const BlockArgs &p, uint8_t *kept, int64_t i, int64_t c, float v) {   // by whole warps, c = 32 k + lane
  const uint32_t e = exponent8(__reduce_max_sync(0xffffffffu, magnitude(v)));
  uint8_t *to = kept + i * p.row_bytes;
  if (c < p.d) to[c] = (uint8_t)(int8_t)hold8(v, scale8(e));
  if (c % kBlock8 == 0 && c < p.d) to[p.d + c / kBlock8] = (uint8_t)e;
  const int64_t behind = p.d + blocks8(p.d);
  if (c < kBlock8 && behind + c < p.row_bytes) to[behind + c] = 0;
}

__global__ void __launch_bounds__(kThreads) wide_kernel(const BlockArgs p) {
  for (int64_t i = blockIdx.x; i < p.n * p.t; i += gridDim.x) {
    const Row x(p, i);
    const auto squares = [&](auto value, float unit) {
      float s = 0.f;
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
        const float v = value(c) * unit;
        s = fmaf(v, v, s);
      }
      return cta_sum(s);
    };
    const auto norm = [&](auto value) {
      const float sum = squares(value, 1.f);
      return sum == INFINITY ? inverse_rms_beyond(squares(value, kLess), 1.f / (float)p.d) : inverse_rms(sum, 1.f / (float)p.d, p.eps);
    };
    const float rho = p.y.at ? norm([&](int64_t c) { return x.y_at(c); }) : 0.f;
    const float r = p.w_pre ? norm([&](int64_t c) { return x.out(c, rho); }) : 0.f;
    if (threadIdx.x == 0 && p.stats) {
      p.stats[2 * i] = rho;
      p.stats[2 * i + 1] = r;
    }
    const int64_t ho = place(p.h_out, x.agent, x.row), u = place(p.u, x.agent, x.row);
    for (int64_t c = threadIdx.x; c - threadIdx.x % 32 < p.d; c += kThreads) {   // (whole warps)
      const bool in = c < p.d;
      const float v = in ? x.out(c, rho) : 0.f;
      if (p.h8) keep(p, p.h8, i, c, in ? x.h_at(c) : 0.f);
      if (p.y8) keep(p, p.y8, i, c, in ? x.y_at(c) : 0.f);
      if (p.gate8) keep(p, p.gate8, i, c, in ? x.gate_at(c) : 0.f);
      __syncwarp();
      if (!in) continue;
      if (p.y.at) store(p.h_out.at, p.stream_type, ho + c, v);
      if (p.w_pre) store(p.u.at, p.act_type, u + c, v * r * x.w_pre(c));
    }
  }
}

// What the gradient of a row is made of, channel by channel.
struct Slopes {
  const Row &x;
  float rho, r;
  int64_t du, dho;
  __device__ Slopes(const Row &x, int64_t i) : x(x), rho(x.p.stats[2 * i]), r(x.p.stats[2 * i + 1]), du(place(x.p.du, x.agent, x.row)), dho(place(x.p.dh_out, x.agent, x.row)) {}
  __device__ float hn(int64_t c) const { return x.out(c, rho) * r; }
  __device__ float up(int64_t c) const { return load(x.p.du.at, x.p.act_type, du + c); }
  __device__ float dh(int64_t c, float mean) const {
    const float past = x.p.dh_out.at ? load(x.p.dh_out.at, x.p.stream_type, dho + c) : 0.f;
    return x.p.w_pre ? fmaf(r, fmaf(-hn(c), mean, x.w_pre(c) * up(c)), past) : past;
  }
};

__global__ void __launch_bounds__(kThreads) wide_means_kernel(const BlockArgs p) {
  for (int64_t i = blockIdx.x; i < p.n * p.t; i += gridDim.x) {
    const Row x(p, i);
    const Slopes s(x, i);
    float a = 0.f, b = 0.f;
    if (p.w_pre) {
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads) a = fmaf(s.hn(c), x.w_pre(c) * s.up(c), a);
      a = cta_sum(a) / (float)p.d;
    }
    if (p.y.at) {
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads) b = fmaf(x.y_at(c) * s.rho, x.scale * x.g(c).g * x.w_post(c) * s.dh(c, a), b);
      b = cta_sum(b) / (float)p.d;
    }
    if (threadIdx.x == 0) p.means[i] = make_float2(a, b);
  }
}

// One channel a thread, part_rows rows of an agent a CTA.
__global__ void __launch_bounds__(kThreads) wide_sums_kernel(const BlockArgs p) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t q = blockIdx.y; q < (int64_t)p.n * p.part_count; q += gridDim.y) {
    const int64_t agent = q / p.part_count, part = q - agent * p.part_count;
    float a = 0.f, b = 0.f, w = 0.f;
    if (c < p.d) {
      for (int64_t row = part * p.part_rows; row < min(p.t, (part + 1) * p.part_rows); ++row) {
        const int64_t i = agent * p.t + row;
        const Row x(p, i);
        const Slopes s(x, i);
        if (p.w_pre) a = fmaf(s.hn(c), s.up(c), a);
        if (p.y.at) {
          b = fmaf(x.y_at(c) * s.rho, x.g(c).g * s.dh(c, p.means[i].x), b);
          w = x.w_post(c);
        }
      }
      p.parts[(q * 2) * p.d + c] = a;
      p.parts[(q * 2 + 1) * p.d + c] = b;
    }
    if (p.dscale) {
      const float s = cta_sum(b * w);
      if (threadIdx.x == 0) p.scale_parts[agent * p.scale_count + part * gridDim.x + blockIdx.x] = s;
    }
  }
}

__global__ void __launch_bounds__(kThreads) wide_grad_kernel(const BlockArgs p) {
  for (int64_t i = blockIdx.x; i < p.n * p.t; i += gridDim.x) {
    const Row x(p, i);
    const Slopes s(x, i);
    const float2 mean = p.means[i];
    const int64_t dh = place(p.dh, x.agent, x.row), dy = place(p.dy, x.agent, x.row), da = place(p.dgate, x.agent, x.row);
    for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
      const float v = s.dh(c, mean.x);
      float out = 0.f, turn = 0.f;
      if (p.y.at) {
        const Gate g = x.g(c);
        const float yn = x.y_at(c) * s.rho, e = x.scale * x.w_post(c) * v;
        out = s.rho * fmaf(-yn, mean.y, g.g * e);
        turn = g.slope * yn * e;
      }
      store(p.dh.at, p.stream_type, dh + c, v);
      if (p.y.at) store(p.dy.at, p.act_type, dy + c, out);
      if (p.gate.at) store(p.dgate.at, p.act_type, da + c, turn);
    }
  }
}

// The parts of the weights' gradients, in the order of the rows.
constexpr int kJoiners = 32;   // warps at most: as many parts are on their way at a time, and more by unrolling
int joiners_of(int64_t parts) { return parts <= 8 ? 4 : parts <= 32 ? 8 : kJoiners; }
__global__ void __launch_bounds__(32 * kJoiners) finish_kernel(const BlockArgs p) {
  __shared__ float halves[2][kJoiners][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, joiners = blockDim.x >> 5;
  const int64_t agent = blockIdx.y, c = (int64_t)blockIdx.x * 32 + lane;
  float a = 0.f, b = 0.f;
  after_first();   // (without rows, of the caller's own kernels, which may have written the scale)
  const float scale = p.part_count == 0 ? 0.f : p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f;
  if (c < p.d)
#pragma unroll 8
    for (int q = warp; q < p.part_count; q += joiners) {
      const float *part = p.parts + ((agent * p.part_count + q) * 2) * p.d + c;
      a += part[0];
      b += part[p.d];
    }
  halves[0][warp][lane] = a;
  halves[1][warp][lane] = b;
  __syncthreads();
  const auto put = [&](void *to, int64_t at, float v) {
    if (p.accumulate) v += load(to, p.weights_type, at);
    store(to, p.weights_type, at, v);
  };
  if (warp < 2 && c < p.d) {
    float s = 0.f;
#pragma unroll 4
    for (int i = 0; i < joiners; ++i) s += halves[warp][i][lane];
    if (warp == 0 && p.dw_pre) put(p.dw_pre, agent * p.dw_pre_stride + c, s);
    if (warp == 1 && p.dw_post) put(p.dw_post, agent * p.dw_post_stride + c, scale * s);
  }
  if (warp == 2 && blockIdx.x == 0 && p.dscale) {
    double s = 0.;
    for (int q = lane; q < p.scale_count; q += 32) s += (double)p.scale_parts[agent * p.scale_count + q];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) put(p.dscale, agent * p.dscale_stride, (float)s);
  }
}


constexpr int64_t kMost = ((int64_t)1 << 31) - 1024;

struct Sizes {
  int64_t part_rows, part_count, column_blocks;
};
Sizes sizes_of(int64_t n, int64_t t, int64_t d) {
  Sizes z;
  z.column_blocks = ceil_div(d, kThreads);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(ceil_div(t, 8), ceil_div(1184, n * z.column_blocks)));
  z.part_rows = std::max<int64_t>(1, ceil_div(t, want));
  z.part_count = ceil_div(t, z.part_rows);
  return z;
}

bool sizes_ok(int32_t n, int64_t t, int64_t d) { return n >= 1 && n <= 65535 && t >= 0 && t < kMost && d >= 1 && d < kMost; }
bool rows_ok(const dsgd_rows_t &x, int64_t d) { return !x.at || (x.row_stride >= d && x.agent_stride >= 0); }
// (two agents' rows in one place would be written by both)
bool out_ok(const dsgd_rows_t &x, int32_t n, int64_t d) { return rows_ok(x, d) && (!x.at || n == 1 || x.agent_stride >= d); }

// Rows in registers, by types and alignment.  A bf16 stream with fp32 activations, which no model here has, is read and written one by one wherever its rows
// start (8 x 4096 x 2048, silu: 208 us forward, 733 for the gradient; the other way round, in words, 168 and 261).
cudaError_t rows(const BlockArgs &p, bool grad, cudaStream_t s) {
  bool words = p.d % 8 == 0;
  for (const dsgd_rows_t *x : {&p.h, &p.y, &p.gate}) words = words && (p.kept || on_words(*x, x == &p.h ? p.stream_type : p.act_type));
  for (const dsgd_rows_t *x : {&p.h_out, &p.dh_out, &p.dh}) words = words && on_words(*x, p.stream_type);
  for (const dsgd_rows_t *x : {&p.u, &p.du, &p.dy, &p.dgate}) words = words && on_words(*x, p.act_type);
  if (p.stream_type == DSGD_F32 && p.act_type == DSGD_F32) return words ? block_rows_f32(p, grad, s) : block_odd_rows_f32(p, grad, s);
  if (p.stream_type == DSGD_F32) return words ? block_rows_mixed(p, grad, s) : block_odd_rows_mixed(p, grad, s);
  if (p.act_type == DSGD_BF16) return words ? block_rows_bf16(p, grad, s) : block_odd_rows_bf16(p, grad, s);
  return block_odd_rows_any(p, grad, s);
}

ceca_status_t status(cudaError_t e) { return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA; }

}  // namespace

// At least four rows a group where there are many (a part costs as much as two rows in memory), one where there are few: 16 rows of 2048 bf16 channels
// take 7.1 us so, 10.3 with four a group, and 256 rows 10.9 with four, 12.6 with one.  Parts are counted by 148 SMs, not by the device's: the workspace's
// size is asked for without one.
int64_t block_grad_parts(int64_t n, int64_t t, int64_t d) {
  const Shape z = grad_shape_of(d);
  const int64_t groups = groups_of(z.group), few = std::min<int64_t>(ceil_div(t, groups), 32);
  return std::max<int64_t>(1, std::min(148 * (int64_t)resident_grad(z.group) / n, std::max(few, ceil_div(t, 4 * groups))));
}

cudaError_t finish_block_grad(const BlockArgs &p, cudaStream_t s) {
  return launch_after(finish_kernel, p, dim3((unsigned)ceil_div(p.d, 32), (unsigned)p.n), 32 * joiners_of(p.part_count), 0, s);
}

}  // namespace ceca

using namespace ceca;

extern "C" ceca_status_t dsgd_block_norm(dsgd_rows_t h, dsgd_rows_t y, dsgd_rows_t gate, const void *w_pre, const void *w_post,
                                         const void *scale, int64_t w_pre_stride, int64_t w_post_stride, int64_t scale_stride,
                                         dsgd_rows_t h_out, dsgd_rows_t u, float *stats, void *h8, void *y8, void *gate8, int32_t n,
                                         int64_t t, int64_t d, int32_t stream_type, int32_t act_type, int32_t weights_type,
                                         int32_t gate_act, float eps, void *stream) {
  if (!sizes_ok(n, t, d) || !is_type(stream_type) || !is_type(act_type) || !is_type(weights_type) || (gate_act != DSGD_GATE_SIGMOID && gate_act != DSGD_GATE_SILU) ||
      !(eps > 0.f) || !std::isfinite(eps) || w_pre_stride < 0 || w_post_stride < 0 || scale_stride < 0 || !rows_ok(h, d) || !rows_ok(y, d) ||
      !rows_ok(gate, d) || !out_ok(h_out, n, d) || !out_ok(u, n, d))
    return CECA_ERR_INVALID_ARG;
  if (t == 0) return CECA_OK;
  if (!h.at || (!y.at && !w_pre) || (y.at && (!w_post || !h_out.at)) || (gate.at && !y.at) || (w_pre && !u.at) || (y8 && !y.at) || (gate8 && !gate.at))
    return CECA_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(h8) | reinterpret_cast<uintptr_t>(y8) | reinterpret_cast<uintptr_t>(gate8)) & 15) || (reinterpret_cast<uintptr_t>(stats) & 7))
    return CECA_ERR_ALIGNMENT;
  BlockArgs p{};
  p.h = h; p.y = y; p.gate = gate; p.h_out = h_out; p.u = u;
  p.w_pre = w_pre; p.w_post = w_post; p.scale = scale;
  p.w_pre_stride = w_pre_stride; p.w_post_stride = w_post_stride; p.scale_stride = scale_stride;
  p.stats = stats; p.h8 = static_cast<uint8_t *>(h8); p.y8 = static_cast<uint8_t *>(y8); p.gate8 = static_cast<uint8_t *>(gate8);
  p.t = t; p.d = d; p.row_bytes = kept_row_bytes(d); p.n = n;
  p.stream_type = stream_type; p.act_type = act_type; p.weights_type = weights_type; p.silu = gate_act == DSGD_GATE_SILU; p.eps = eps;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d <= kWidest) return status(rows(p, false, s));
  wide_kernel<<<(unsigned)std::min<int64_t>(n * t, (int64_t)sm_count() * 8), kThreads, 0, s>>>(p);
  return status(cudaGetLastError());
}

extern "C" size_t dsgd_block_norm_workspace_bytes(int32_t n, int64_t t, int64_t d) {
  if (!sizes_ok(n, t, d)) return 0;
  if (d <= kWidest) return (4 * (size_t)n * block_grad_parts(n, t, d) * part_floats(d) + 15) / 16 * 16;
  const Sizes z = sizes_of(n, t, d);
  return 8 * (size_t)n * t + 4 * (size_t)n * z.part_count * (2 * (size_t)d + z.column_blocks);
}

extern "C" ceca_status_t dsgd_block_norm_grad(dsgd_rows_t h, dsgd_rows_t y, dsgd_rows_t gate, int32_t kept, const void *w_pre,
                                              const void *w_post, const void *scale, int64_t w_pre_stride, int64_t w_post_stride,
                                              int64_t scale_stride, const float *stats, dsgd_rows_t du, dsgd_rows_t dh_out, dsgd_rows_t dh,
                                              dsgd_rows_t dy, dsgd_rows_t dgate, void *dw_pre, void *dw_post, void *dscale,
                                              int64_t dw_pre_stride, int64_t dw_post_stride, int64_t dscale_stride, int32_t accumulate,
                                              int32_t n, int64_t t, int64_t d, int32_t stream_type, int32_t act_type, int32_t weights_type,
                                              int32_t gate_act, void *workspace, size_t workspace_bytes, void *stream) {
  const dsgd_rows_t none{};
  if (!sizes_ok(n, t, d) || !is_type(stream_type) || !is_type(act_type) || !is_type(weights_type) || (gate_act != DSGD_GATE_SIGMOID && gate_act != DSGD_GATE_SILU) ||
      w_pre_stride < 0 || w_post_stride < 0 || scale_stride < 0 || !rows_ok(kept ? none : h, d) || !rows_ok(kept ? none : y, d) ||
      !rows_ok(kept ? none : gate, d) || du.agent_stride < 0 || du.row_stride < 0 || dh_out.agent_stride < 0 || dh_out.row_stride < 0 ||
      !out_ok(dh, n, d) || !out_ok(dy, n, d) || !out_ok(dgate, n, d) || (t > 0 && !y.at && !w_pre) || (gate.at && !y.at) || (y.at && (!w_post || !dw_post)) ||
      (w_pre && !dw_pre) || (dw_pre && dw_pre_stride < (n > 1 ? d : 0)) || (dw_post && dw_post_stride < (n > 1 ? d : 0)) ||
      (dscale && dscale_stride < (n > 1 ? 1 : 0)))
    return CECA_ERR_INVALID_ARG;
  if (t > 0 && (!h.at || !stats || (w_pre && !du.at) || !dh.at || (y.at && !dy.at) || (gate.at && !dgate.at))) return CECA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(stats) & 7) != 0) return CECA_ERR_ALIGNMENT;
  if (kept && ((reinterpret_cast<uintptr_t>(h.at) | reinterpret_cast<uintptr_t>(y.at) | reinterpret_cast<uintptr_t>(gate.at)) & 15))
    return CECA_ERR_ALIGNMENT;
  const size_t need = dsgd_block_norm_workspace_bytes(n, t, d);
  if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15))) return CECA_ERR_WORKSPACE;
  BlockArgs p{};
  p.h = h; p.y = y; p.gate = gate; p.du = du; p.dh_out = dh_out; p.dh = dh; p.dy = dy; p.dgate = dgate;
  p.w_pre = w_pre; p.w_post = w_post; p.scale = scale; p.dw_pre = dw_pre; p.dw_post = dw_post; p.dscale = dscale;
  p.w_pre_stride = w_pre_stride; p.w_post_stride = w_post_stride; p.scale_stride = scale_stride;
  p.dw_pre_stride = dw_pre_stride; p.dw_post_stride = dw_post_stride; p.dscale_stride = dscale_stride;
  p.stats = const_cast<float *>(stats);
  p.t = t; p.d = d; p.row_bytes = kept_row_bytes(d); p.n = n; p.kept = kept != 0; p.accumulate = accumulate != 0;
  p.stream_type = stream_type; p.act_type = act_type; p.weights_type = weights_type; p.silu = gate_act == DSGD_GATE_SILU;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  p.means = static_cast<float2 *>(workspace);
  if (d <= kWidest && t > 0) return status(rows(p, true, s));
  const Sizes z = sizes_of(n, t, d);
  p.part_rows = z.part_rows;
  p.part_count = (int32_t)z.part_count;
  p.scale_count = (int32_t)(z.part_count * z.column_blocks);
  p.parts = reinterpret_cast<float *>(p.means + n * t);
  p.scale_parts = p.parts + (size_t)n * z.part_count * 2 * d;
  if (t > 0) {
    const unsigned rows = (unsigned)std::min<int64_t>(n * t, (int64_t)sm_count() * 8);
    wide_means_kernel<<<rows, kThreads, 0, s>>>(p);
    wide_sums_kernel<<<dim3((unsigned)z.column_blocks, (unsigned)std::min<int64_t>(n * z.part_count, 65535)), kThreads, 0, s>>>(p);
    wide_grad_kernel<<<rows, kThreads, 0, s>>>(p);
  }
  return status(finish_block_grad(p, s));
}
