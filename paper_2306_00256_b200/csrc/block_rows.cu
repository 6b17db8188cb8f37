// The end of a block and the start of the next for rows that a group of threads holds in registers.
//
// A CTA (or, of rows up to 256 channels, each of its four warps) takes every part_count-th row of an agent.  The next rows are copied to a
// ring in shared memory while one is computed on, so that loads are always under way; the weights stay in registers.  Two sums over the
// group a row: y^2, then h_out^2.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "block_norm.cuh"
#include "tma.h"

namespace ceca {
namespace {

template <int G, int PASSES, bool WORDS>
__global__ void __launch_bounds__(G == 32 ? 128 : G) block_kernel(const __grid_constant__ BlockArgs p) {
  using X = Place<G, PASSES, WORDS>;
  using L = Lay<G, PASSES, WORDS>;
  extern __shared__ uint4 ring[];
  __shared__ float part[2][G / 32];
  constexpr int kGroups = G == 32 ? 4 : 1;
  const int rank = G == 32 ? threadIdx.x & 31 : threadIdx.x, group = G == 32 ? threadIdx.x >> 5 : 0, d = (int)p.d;
  const int64_t ctas = p.part_count / kGroups, agent = blockIdx.x / ctas;
  const int64_t first = (blockIdx.x - agent * ctas) * kGroups + group;
  const bool y = p.y.at != nullptr, gated = p.gate.at != nullptr, u = p.w_pre != nullptr;
  uint8_t *mine = reinterpret_cast<uint8_t *>(ring) + (size_t)group * p.stages * p.stage_bytes;
  const uint32_t mine32 = (uint32_t)__cvta_generic_to_shared(mine);
  const int sb = p.stream_type == DSGD_BF16 ? 2 : 4, ab = p.act_type == DSGD_BF16 ? 2 : 4;
  const auto row_of = [&](const dsgd_rows_t &x, int64_t row, int bytes) { return static_cast<const uint8_t *>(x.at) + place(x, agent, row) * bytes; };
  const auto bring = [&](int64_t row, int stage) {
    if (row < p.t) {
      uint32_t to = mine32 + stage * p.stage_bytes;
      X::copy(to, row_of(p.h, row, sb), p.stream_type, d, rank);
      if (y) X::copy(to + p.room[0], row_of(p.y, row, ab), p.act_type, d, rank);
      if (gated) X::copy(to + p.room[0] + p.room[1], row_of(p.gate, row, ab), p.act_type, d, rank);
    }
    copies_end();
  };
  for (int i = 0; i + 1 < p.stages; ++i) bring(first + (int64_t)i * p.part_count, i);
  const float scale = p.scale ? load(p.scale, p.weights_type, agent * p.scale_stride) : 1.f;
  Pairs8 wq[PASSES], wp[PASSES];   // scale w_post, w_pre
#pragma unroll
  for (int j = 0; j < PASSES; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = L::channel(rank, j, e);
      (e & 1 ? wq[j].v[e / 2].y : wq[j].v[e / 2].x) = y && c < d ? scale * load(p.w_post, p.weights_type, agent * p.w_post_stride + c) : 0.f;
      (e & 1 ? wp[j].v[e / 2].y : wp[j].v[e / 2].x) = u && c < d ? load(p.w_pre, p.weights_type, agent * p.w_pre_stride + c) : 0.f;
    }
  int stage = 0;
  for (int64_t row = first; row < p.t; row += p.part_count) {
    if (p.stages > 1) {
      bring(row + (int64_t)(p.stages - 1) * p.part_count, stage == 0 ? p.stages - 1 : stage - 1);
    } else {
      bring(row, 0);
    }
    copies_but(p.stages - 1);
    if (!WORDS) {
      if (G == 32) __syncwarp();
      else __syncthreads();
    }
    const uint8_t *at = mine + stage * p.stage_bytes;
    stage = stage + 1 == p.stages ? 0 : stage + 1;
    const auto pad = [&](const dsgd_rows_t &x, int bytes) { return WORDS ? 0 : (int)(reinterpret_cast<uintptr_t>(row_of(x, row, bytes)) & 15); };
    const int64_t i = agent * p.t + row;
    Pairs8 h[PASSES];
    float rho = 0.f;
#pragma unroll
    for (int j = 0; j < PASSES; ++j) {
      h[j] = X::read(at, pad(p.h, sb), p.stream_type, d, rank, j);
      if (p.h8) X::keep(p.h8 + i * p.row_bytes, h[j], d, rank, j);
    }
    if (p.h8) X::keep_end(p.h8 + i * p.row_bytes, d, rank);
    if (y) {
      Pairs8 a[PASSES];
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        a[j] = X::read(at + p.room[0], pad(p.y, ab), p.act_type, d, rank, j);
        if (p.y8) X::keep(p.y8 + i * p.row_bytes, a[j], d, rank, j);
      }
      if (p.y8) X::keep_end(p.y8 + i * p.row_bytes, d, rank);
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
      rho = inverse_rms(group_sum<G>(squares(1.f), part, 0), p.d, p.eps, [&](float unit) {
        if (G > 32) __syncthreads();
        return group_sum<G>(squares(unit), part, 0);
      });
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
        Pairs8 g;
        if (gated) {
          g = X::read(at + p.room[0] + p.room[1], pad(p.gate, ab), p.act_type, d, rank, j);
          if (p.gate8) X::keep(p.gate8 + i * p.row_bytes, g, d, rank, j);
#pragma unroll
          for (int k = 0; k < 4; ++k) g.v[k] = {gate_of(g.v[k].x, p.silu).g, gate_of(g.v[k].y, p.silu).g};
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const Val<2> by = gated ? mul(wq[j].v[k], g.v[k]) : wq[j].v[k];
          h[j].v[k] = fma(by, mul(a[j].v[k], all<2>(rho)), h[j].v[k]);
        }
      }
      if (p.gate8) X::keep_end(p.gate8 + i * p.row_bytes, d, rank);
      uint8_t *to = static_cast<uint8_t *>(p.h_out.at) + place(p.h_out, agent, row) * sb;
#pragma unroll
      for (int j = 0; j < PASSES; ++j) X::write(to, p.stream_type, h[j], d, rank, j);
    }
    float r = 0.f;
    if (u) {
      const auto squares = [&](float unit) {
        Pairs8 s{};
#pragma unroll
        for (int j = 0; j < PASSES; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const Val<2> v = unit == 1.f ? h[j].v[k] : mul(h[j].v[k], all<2>(unit));
            s.v[k] = fma(v, v, s.v[k]);
          }
        return total(s);
      };
      r = inverse_rms(group_sum<G>(squares(1.f), part, 1), p.d, p.eps, [&](float unit) {
        if (G > 32) __syncthreads();
        return group_sum<G>(squares(unit), part, 1);
      });
      uint8_t *to = static_cast<uint8_t *>(p.u.at) + place(p.u, agent, row) * ab;
#pragma unroll
      for (int j = 0; j < PASSES; ++j) {
#pragma unroll
        for (int k = 0; k < 4; ++k) h[j].v[k] = mul(mul(h[j].v[k], all<2>(r)), wp[j].v[k]);
        X::write(to, p.act_type, h[j], d, rank, j);
      }
    }
    if (p.stats && rank == 0) *reinterpret_cast<float2 *>(p.stats + 2 * i) = make_float2(rho, r);
    if (!WORDS || !y || !u) {   // the place is written again only when everybody has read it, and a sum's when everybody has it
      if (G == 32) __syncwarp();
      else __syncthreads();
    }
  }
  copies_but(0);
}

template <int G, int PASSES, bool WORDS> cudaError_t launch(BlockArgs p, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  auto kernel = block_kernel<G, PASSES, WORDS>;
  constexpr int kGroups = G == 32 ? 4 : 1, threads = G == 32 ? 128 : G;
  cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), 220 << 10, &done);
  if (e != cudaSuccess) return e;
  const auto room = [&](const dsgd_rows_t &x, int32_t type) {
    if (!x.at) return 0;
    return WORDS ? 16 * G * PASSES * (type == DSGD_BF16 ? 1 : 2) : (int)((p.d * type_bytes(type) + 47) / 16 * 16);
  };
  p.room[0] = room(p.h, p.stream_type);
  p.room[1] = room(p.y, p.act_type);
  p.room[2] = room(p.gate, p.act_type);
  p.stage_bytes = p.room[0] + p.room[1] + p.room[2];
  // rows on their way: enough for the SM's share of what the memory delivers within a load's latency
  const int64_t resident = std::max(1, std::min(2048 / threads, 65536 / (threads * 72 * PASSES)));
  p.stages = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, (int64_t)(200 << 10) / (resident * kGroups * p.stage_bytes)));
  if ((int64_t)p.stages * p.stage_bytes * kGroups > (220 << 10)) return cudaErrorInvalidConfiguration;
  const int64_t most = std::max<int64_t>(1, (int64_t)sm_count() * resident / p.n) * kGroups;
  p.part_count = (int32_t)(std::min(most, ceil_div(p.t, kGroups) * kGroups));
  kernel<<<(unsigned)(p.n * (p.part_count / kGroups)), threads, (size_t)p.stages * p.stage_bytes * kGroups, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_block_rows(BlockArgs p, bool words, cudaStream_t s) {
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
