// The gradient of the end of a block and the start of the next, for rows that a group of threads holds in registers.
//
// As the forward kernel: every part_count-th row of an agent a group, the next rows on their way through a ring in shared memory.  With q = s g w_post yn
// (what the block added), f = w_pre du and t = dh_out + r f, a row needs three sums at once: A = hn f, B = q t, C = q hn; then
//   m = A / d,  dh = t - r m hn,  mean(yn e) = (B - r m C) / d.
// The weights' gradients are summed over the group's rows in registers, and written once, to be joined by a second kernel.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "block_norm.cuh"
#include "tma.h"

namespace ceca {
namespace {

constexpr int kSms = 148;   // parts are counted by this, not by the device's own number: the workspace's size is asked for without one

template <int G> __device__ __forceinline__ float3 group_sums(float3 x, float4 (*part)[G / 32], int turn) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    x.x += __shfl_xor_sync(0xffffffffu, x.x, o);
    x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
    x.z += __shfl_xor_sync(0xffffffffu, x.z, o);
  }
  if (G == 32) return x;
  if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = make_float4(x.x, x.y, x.z, 0.f);
  __syncthreads();
  x = make_float3(0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < G / 32; ++i) {
    const float4 v = part[turn][i];
    x.x += v.x;
    x.y += v.y;
    x.z += v.z;
  }
  return x;
}

template <int G, int PASSES, bool WORDS>
__global__ void __launch_bounds__(G == 32 ? 128 : G, G == 32 ? 4 : 512 / G) block_grad_kernel(const __grid_constant__ BlockArgs p) {
  using X = Place<G, PASSES, WORDS>;
  using L = Lay<G, PASSES, WORDS>;
  extern __shared__ uint4 ring[];
  __shared__ float4 part[2][G / 32];
  constexpr int kGroups = G == 32 ? 4 : 1;
  const int rank = G == 32 ? threadIdx.x & 31 : threadIdx.x, group = G == 32 ? threadIdx.x >> 5 : 0, d = (int)p.d;
  const int64_t agent = blockIdx.x / p.part_count, cta = blockIdx.x - agent * p.part_count;
  const int64_t first = cta * kGroups + group, hop = (int64_t)p.part_count * kGroups;
  const bool y = p.y.at != nullptr, gated = p.gate.at != nullptr, u = p.w_pre != nullptr, past = p.dh_out.at != nullptr;
  uint8_t *mine = reinterpret_cast<uint8_t *>(ring) + (size_t)group * p.stages * p.stage_bytes;
  const uint32_t mine32 = (uint32_t)__cvta_generic_to_shared(mine);
  const int sb = p.stream_type == DSGD_BF16 ? 2 : 4, ab = p.act_type == DSGD_BF16 ? 2 : 4;
  const int32_t held_s = p.kept ? 2 : p.stream_type, held_a = p.kept ? 2 : p.act_type;
  const auto row_of = [&](const dsgd_rows_t &x, int64_t row, int bytes) { return static_cast<const uint8_t *>(x.at) + place(x, agent, row) * bytes; };
  const auto held_row = [&](const dsgd_rows_t &x, int64_t row, int bytes) {
    return p.kept ? static_cast<const uint8_t *>(x.at) + (agent * p.t + row) * p.row_bytes : row_of(x, row, bytes);
  };
  const int off_y = p.room[0], off_g = off_y + p.room[1], off_u = off_g + p.room[2], off_p = off_u + p.room[3];
  const auto bring = [&](int64_t row, int stage) {
    if (row < p.t) {
      const uint32_t to = mine32 + stage * p.stage_bytes;
      if (y || u) X::copy(to, held_row(p.h, row, sb), held_s, d, rank);
      if (y) X::copy(to + off_y, held_row(p.y, row, ab), held_a, d, rank);
      if (gated) X::copy(to + off_g, held_row(p.gate, row, ab), held_a, d, rank);
      if (u) X::copy(to + off_u, row_of(p.du, row, ab), p.act_type, d, rank);
      if (past) X::copy(to + off_p, row_of(p.dh_out, row, sb), p.stream_type, d, rank);
    }
    copies_end();
  };
  for (int i = 0; i + 1 < p.stages; ++i) bring(first + i * hop, i);
  const float scale = p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f;
  Pairs8 wq[PASSES], wp[PASSES];   // scale w_post, w_pre
  Pairs8 sum_pre[PASSES], sum_post[PASSES];
#pragma unroll
  for (int j = 0; j < PASSES; ++j) {
#pragma unroll
    for (int k = 0; k < 4; ++k) sum_pre[j].v[k] = sum_post[j].v[k] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = L::channel(rank, j, e);
      (e & 1 ? wq[j].v[e / 2].y : wq[j].v[e / 2].x) = y && c < d ? scale * load(p.w_post, p.weights_type, agent * p.w_post_stride + c) : 0.f;
      (e & 1 ? wp[j].v[e / 2].y : wp[j].v[e / 2].x) = u && c < d ? load(p.w_pre, p.weights_type, agent * p.w_pre_stride + c) : 0.f;
    }
  }
  const float over_d = 1.f / (float)p.d;
  int stage = 0, turn = 0;
  for (int64_t row = first; row < p.t; row += hop) {
    if (p.stages > 1) bring(row + (p.stages - 1) * hop, stage == 0 ? p.stages - 1 : stage - 1);
    else bring(row, 0);
    const float2 st = *reinterpret_cast<const float2 *>(p.stats + 2 * (agent * p.t + row));
    const Val<2> rho = all<2>(st.x), r = all<2>(st.y);
    copies_but(p.stages - 1);
    if (!WORDS) {
      if (G == 32) __syncwarp();
      else __syncthreads();
    }
    const uint8_t *at = mine + stage * p.stage_bytes;
    stage = stage + 1 == p.stages ? 0 : stage + 1;
    const auto pad = [&](const dsgd_rows_t &x, int bytes, bool held) {
      return WORDS || (held && p.kept) ? 0 : (int)(reinterpret_cast<uintptr_t>(row_of(x, row, bytes)) & 15);
    };
    Pairs8 hn[PASSES], t[PASSES], yn[PASSES], g[PASSES], slope[PASSES];
    Val<2> a{0.f, 0.f}, b{0.f, 0.f}, c{0.f, 0.f};
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      hn[j] = X::read(at, pad(p.h, sb, true), held_s, d, rank, j);
      if (y) yn[j] = X::read(at + off_y, pad(p.y, ab, true), held_a, d, rank, j);
      if (gated) g[j] = X::read(at + off_g, pad(p.gate, ab, true), held_a, d, rank, j);
      Pairs8 du;
      if (u) du = X::read(at + off_u, pad(p.du, ab, false), p.act_type, d, rank, j);
      if (past) t[j] = X::read(at + off_p, pad(p.dh_out, sb, false), p.stream_type, d, rank, j);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (!past) t[j].v[k] = {0.f, 0.f};
        Val<2> q{0.f, 0.f};
        if (y) {
          yn[j].v[k] = mul(yn[j].v[k], rho);
          q = mul(wq[j].v[k], yn[j].v[k]);
          if (gated) {
            const Gate x = gate_of(g[j].v[k].x, p.silu), z = gate_of(g[j].v[k].y, p.silu);
            g[j].v[k] = {x.g, z.g};
            slope[j].v[k] = {x.slope, z.slope};
            q = mul(q, g[j].v[k]);
          }
        }
        if (u) {
          hn[j].v[k] = mul(add(hn[j].v[k], q), r);
          const Val<2> f = mul(wp[j].v[k], du.v[k]);
          a = fma(hn[j].v[k], f, a);
          t[j].v[k] = fma(r, f, t[j].v[k]);
          c = fma(q, hn[j].v[k], c);
          sum_pre[j].v[k] = fma(hn[j].v[k], du.v[k], sum_pre[j].v[k]);
        }
        b = fma(q, t[j].v[k], b);
      }
    }
    const float3 s = group_sums<G>(make_float3(a.x + a.y, b.x + b.y, c.x + c.y), part, turn);
    turn ^= 1;
    const float rm = u ? st.y * s.x * over_d : 0.f, my = (s.y - rm * s.z) * over_d;
    uint8_t *dh = static_cast<uint8_t *>(p.dh.at) + place(p.dh, agent, row) * sb;
    uint8_t *dy = static_cast<uint8_t *>(p.dy.at) + place(p.dy, agent, row) * ab;
    uint8_t *da = static_cast<uint8_t *>(p.dgate.at) + place(p.dgate, agent, row) * ab;
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      Pairs8 oy, oa;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (u) t[j].v[k] = fma(all<2>(-rm), hn[j].v[k], t[j].v[k]);
        if (y) {
          const Val<2> e = mul(wq[j].v[k], t[j].v[k]), gy = gated ? mul(g[j].v[k], yn[j].v[k]) : yn[j].v[k];
          oy.v[k] = mul(rho, fma(all<2>(-my), yn[j].v[k], gated ? mul(g[j].v[k], e) : e));
          if (gated) oa.v[k] = mul(mul(slope[j].v[k], yn[j].v[k]), e);
          sum_post[j].v[k] = fma(gy, t[j].v[k], sum_post[j].v[k]);
        }
      }
      X::write(dh, p.stream_type, t[j], d, rank, j);
      if (y) X::write(dy, p.act_type, oy, d, rank, j);
      if (gated) X::write(da, p.act_type, oa, d, rank, j);
    }
    if (!WORDS && G == 32) __syncwarp();   // (of larger groups all have met since they read the place)
  }
  copies_but(0);
  follow_early();
  // the group's sums; those of a CTA's groups are joined in their order
  const int64_t q = agent * p.part_count + cta;
  float *to = p.parts + 2 * q * p.d;
  float dot = 0.f;
#pragma unroll
  for (int j = 0; j < PASSES; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = L::channel(rank, j, e);
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
    for (int e = 0; e < 8; ++e) {
      const int c = L::channel(rank, 0, e);
      if (c >= d) continue;
      all_of[(2 * group) * d + c] = e & 1 ? sum_pre[0].v[e / 2].y : sum_pre[0].v[e / 2].x;
      all_of[(2 * group + 1) * d + c] = e & 1 ? sum_post[0].v[e / 2].y : sum_post[0].v[e / 2].x;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * d; c += 32 * kGroups) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) x += all_of[2 * i * d + c];
      to[c] = x;
    }
  }
  if (p.dscale) {
    const float3 s = group_sums<G>(make_float3(dot, 0.f, 0.f), part, turn);
    if (rank == 0) p.scale_parts[q * kGroups + group] = s.x;
  }
}

// CTAs of an SM
int64_t resident(int64_t d) { return group_of(d) == 32 ? 4 : 512 / group_of(d); }

template <int G, int PASSES, bool WORDS> cudaError_t launch(BlockArgs p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  auto kernel = block_grad_kernel<G, PASSES, WORDS>;
  constexpr int kGroups = G == 32 ? 4 : 1, threads = G == 32 ? 128 : G;
  cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), 220 << 10, &done);
  if (e != cudaSuccess) return e;
  const auto room = [&](const dsgd_rows_t &x, int32_t type) {
    if (!x.at) return 0;
    if (type == 2) return WORDS ? 12 * G * PASSES : (int)kept_row_bytes(p.d);
    return WORDS ? 16 * G * PASSES * (type == DSGD_BF16 ? 1 : 2) : (int)((p.d * type_bytes(type) + 47) / 16 * 16);
  };
  p.room[0] = room(p.h, p.kept ? 2 : p.stream_type);
  p.room[1] = room(p.y, p.kept ? 2 : p.act_type);
  p.room[2] = room(p.gate, p.kept ? 2 : p.act_type);
  p.room[3] = p.w_pre ? room(p.du, p.act_type) : 0;
  p.room[4] = room(p.dh_out, p.stream_type);
  p.stage_bytes = p.room[0] + p.room[1] + p.room[2] + p.room[3] + p.room[4];
  p.stages = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, (int64_t)(200 << 10) / (resident(p.d) * kGroups * p.stage_bytes)));
  const size_t bytes = std::max((size_t)p.stages * p.stage_bytes * kGroups, kGroups > 1 ? kGroups * 2 * sizeof(float) * (size_t)p.d : 0);
  if (bytes > (220 << 10)) return cudaErrorInvalidConfiguration;
  p.part_count = (int32_t)block_grad_parts(p.n, p.t, p.d);
  p.scale_count = p.part_count * kGroups;
  p.parts = reinterpret_cast<float *>(p.means);   // the workspace
  p.scale_parts = p.parts + (size_t)p.n * p.part_count * 2 * p.d;
  kernel<<<(unsigned)(p.n * p.part_count), threads, bytes, s>>>(p);
  e = cudaGetLastError();
  return e == cudaSuccess ? finish_block_grad(p, s) : e;
}

}  // namespace

// At least four rows a group: a part costs as much as two rows in memory.
int64_t block_grad_parts(int64_t n, int64_t t, int64_t d) {
  const int64_t groups = group_of(d) == 32 ? 4 : 1;
  return std::max<int64_t>(1, std::min(kSms * resident(d) / n, ceil_div(t, 4 * groups)));
}

cudaError_t launch_block_grad_rows(BlockArgs p, bool words, cudaStream_t s) {
  const auto by = [&](auto g, auto passes) {
    constexpr int G = decltype(g)::value, P = decltype(passes)::value;
    return words ? launch<G, P, true>(p, s) : launch<G, P, false>(p, s);
  };
  using One = std::integral_constant<int, 1>;
  switch (group_of(p.d)) {
    case 32: return by(std::integral_constant<int, 32>(), One());
    case 64: return by(std::integral_constant<int, 64>(), One());
    case 128: return by(std::integral_constant<int, 128>(), One());
    case 256: return by(std::integral_constant<int, 256>(), One());
    default: return p.d <= 4096 ? by(std::integral_constant<int, 512>(), One()) : by(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
  }
}

}  // namespace ceca
