// Gated linear recurrence over a sequence and its gradient.
//
//   a = sigmoid(f),  h_s = keep_s h_{s-1} + (1 - a_s) x_s          (keep = a, or 0 where a document begins)
//   l_s = dh_s + keep_{s+1} l_{s+1},  dx_s = (1 - a_s) l_s,  df_s = a_s (1 - a_s) l_s (p_s - x_s),  dh0 = keep_0 l_0
//
// with p_s the state before step s (0 where a document begins).  States are carried in fp32.
//
// A run of steps maps the state before it to the state after it by h -> A h + H, and two such maps in a row are
// one again, so a sequence is cut into tiles of kTileSteps steps, a tile into the kSteps steps of each warp (lanes are
// channels): every thread finds its own (A, H), the warps exchange theirs through shared memory, and each thread
// runs its steps once more from the state that reaches it.  x and f are read once and h is written once.  Where the
// channels alone do not fill the GPU, a cluster of CTAs takes consecutive tiles of the same channels and
// exchanges the tiles' maps through distributed shared memory, all composed in the order of the steps: the
// result does not depend on timing.  The gradient runs the same way from the end, with c_s = keep_s l_s in place of
// the state, and finds the states again from the marks that the forward call kept at the start of each tile.
//
// A document's first step ends what comes before it even when that is an infinity or a NaN, which no product with
// zero does: the A of a run that contains such a step is set to kCut, and a map with A = kCut is the constant H.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ceca.h"
#include "tma.h"
#include "values.h"

namespace ceca {
namespace {

namespace cg = cooperative_groups;

constexpr int kSteps = 8;                       // steps of a thread
constexpr int kTileWarps = 8;
constexpr int kTileThreads = 32 * kTileWarps;
constexpr int kTileSteps = kSteps * kTileWarps; // and the distance between two marks
constexpr int kMaxCluster = 16;
constexpr int kFewSteps = 16;                   // sequences up to here: one thread per channel
constexpr float kCut = -1.f;

struct RecurArgs {
  const void *x, *f, *dh;
  const float *h0, *dh_last;
  const uint8_t *starts;
  void *h, *dx, *df;
  float *h_last, *dh0;
  float *marks;
  int64_t t, d, n_marks;
  int64_t x_seq, x_step, f_seq, f_step, h_seq, h_step, dh_seq, dh_step, dx_seq, dx_step, df_seq, df_step;
  int32_t blocks;   // channel blocks per sequence
  int32_t cluster;  // CTAs along the steps
};

// C adjacent channels of one step, as stored.
template <typename T, int C> struct Slice;
template <> struct Slice<float, 1> { float v; };
template <> struct Slice<float, 2> { float2 v; };
template <> struct Slice<bf16, 1> { bf16 v; };
template <> struct Slice<bf16, 2> { uint32_t v; };
__device__ __forceinline__ void unpack(const Slice<float, 1> &s, float *o) { o[0] = s.v; }
__device__ __forceinline__ void unpack(const Slice<float, 2> &s, float *o) { o[0] = s.v.x; o[1] = s.v.y; }
__device__ __forceinline__ void unpack(const Slice<bf16, 1> &s, float *o) { o[0] = __bfloat162float(s.v); }
__device__ __forceinline__ void unpack(const Slice<bf16, 2> &s, float *o) {
  o[0] = __uint_as_float(s.v << 16);   // a bf16 is the upper half of the fp32 of the same value
  o[1] = __uint_as_float(s.v & 0xffff0000u);
}
__device__ __forceinline__ void pack(const float *o, Slice<float, 1> *s) { s->v = o[0]; }
__device__ __forceinline__ void pack(const float *o, Slice<float, 2> *s) { s->v = make_float2(o[0], o[1]); }
__device__ __forceinline__ void pack(const float *o, Slice<bf16, 1> *s) { s->v = __float2bfloat16_rn(o[0]); }
__device__ __forceinline__ void pack(const float *o, Slice<bf16, 2> *s) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(o[0], o[1]);
  s->v = *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// a = sigmoid(f) and na = sigmoid(-f), each to a few ulp of itself: with e = exp(-f), a = 1 / (1 + e) and na = e a.
// The exponent stops at 126, where e and its reciprocal are both still normal numbers and na rounds to 1; the
// saturating subtraction then makes a exactly 0 and changes no a above 2^-100.
__device__ __forceinline__ void gates(float f, float *a, float *na) {
  const float e = ex2(fminf(f * -1.4426950408889634f, 126.f));
  const float r = rcp(1.f + e);
  *na = e * r;
  *a = __saturatef(r - 0x1p-125f);
}

template <bool STARTS> __device__ __forceinline__ float follow(float A, float H, float carry) {
  return STARTS && A < 0.f ? H : fmaf(A, carry, H);
}

// What the warps of a tile, and the tiles of a cluster, tell one another: the map of a run, per channel.
template <int C> struct Exchange {
  float warp_a[2][kTileWarps][32 * C], warp_h[2][kTileWarps][32 * C];
  float tile_a[2][kMaxCluster][32 * C], tile_h[2][kMaxCluster][32 * C];
};

// The thread's map enters the exchange; on return `carry` (what reaches the first run of the group of tiles) has
// become what reaches the group after this one, `into_tile` what reaches this tile and `into` what reaches this thread's
// run.  `order` is the warp's place in the direction of the recurrence.  One block barrier, and one cluster barrier
// where there is a cluster; `buf` alternates, so that what is still read is not overwritten.
template <int C, bool STARTS, bool CLUSTER>
__device__ __forceinline__ void join(Exchange<C> &ex, int buf, int order, int rank, int ranks, const float *A,
                                     const float *H, float *carry, float *into_tile, float *into) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    ex.warp_a[buf][order][lane * C + c] = A[c];
    ex.warp_h[buf][order][lane * C + c] = H[c];
  }
  __syncthreads();
  if (CLUSTER) {
    if (threadIdx.x < 32 * C) {
      float ta = 1.f, th = 0.f;
      for (int w = 0; w < kTileWarps; ++w) {
        const float wa = ex.warp_a[buf][w][threadIdx.x], wh = ex.warp_h[buf][w][threadIdx.x];
        th = follow<STARTS>(wa, wh, th);
        ta = STARTS && (wa < 0.f || ta < 0.f) ? kCut : ta * wa;
      }
      cg::cluster_group cl = cg::this_cluster();
      for (int r = 0; r < ranks; ++r) {
        cl.map_shared_rank(&ex.tile_a[buf][rank][0], r)[threadIdx.x] = ta;
        cl.map_shared_rank(&ex.tile_h[buf][rank][0], r)[threadIdx.x] = th;
      }
    }
    cg::this_cluster().sync();
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float v = carry[c], at = v;
    if (CLUSTER) {
      for (int r = 0; r < ranks; ++r) {
        if (r == rank) at = v;
        v = follow<STARTS>(ex.tile_a[buf][r][lane * C + c], ex.tile_h[buf][r][lane * C + c], v);
      }
      carry[c] = v;
    }
    into_tile[c] = v = at;
    for (int w = 0; w < kTileWarps; ++w) {
      if (w == order) {
        into[c] = v;
        if (CLUSTER) break;
      }
      v = follow<STARTS>(ex.warp_a[buf][w][lane * C + c], ex.warp_h[buf][w][lane * C + c], v);
    }
    if (!CLUSTER) carry[c] = v;
  }
}

template <typename T, int C, bool STARTS, bool CLUSTER>
__global__ void __launch_bounds__(kTileThreads, 3) recurrence_kernel(const RecurArgs p) {
  using S = Slice<T, C>;
  __shared__ Exchange<C> ex;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ranks = CLUSTER ? p.cluster : 1;
  const int rank = CLUSTER ? (int)(blockIdx.x % ranks) : 0;
  const int64_t which = blockIdx.x / ranks;
  const int64_t i = which / p.blocks;
  const int64_t c0 = (which - i * p.blocks) * (32 * C) + lane * C;
  const bool live = c0 < p.d;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c0;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c0;
  T *h = static_cast<T *>(p.h) + i * p.h_seq + c0;
  const uint8_t *starts = STARTS ? p.starts + i * p.t : nullptr;

  float carry[C];
#pragma unroll
  for (int c = 0; c < C; ++c) carry[c] = live && p.h0 ? p.h0[i * p.d + c0 + c] : 0.f;
  S xr[kSteps], fr[kSteps];
  auto fetch = [&](int64_t tile) {
    const int64_t s0 = tile * kTileSteps + warp * kSteps;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
      if (live && s0 + j < p.t) {
        xr[j] = *reinterpret_cast<const S *>(x + (s0 + j) * p.x_step);
        fr[j] = *reinterpret_cast<const S *>(f + (s0 + j) * p.f_step);
      }
  };
  if (CLUSTER) cg::this_cluster().sync();   // every CTA runs before anybody writes into its shared memory
  fetch(rank);
  int buf = 0;
  for (int64_t first = 0; first < p.n_marks; first += ranks, buf ^= 1) {
    const int64_t tile = first + rank;
    const int64_t s0 = tile * kTileSteps + warp * kSteps;
    float a[kSteps][C], b[kSteps][C], A[C], H[C];
    uint32_t cuts = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) { A[c] = 1.f; H[c] = 0.f; }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const bool in = live && s0 + j < p.t;
      float xv[C], fv[C];
      unpack(xr[j], xv);
      unpack(fr[j], fv);
      const bool cut = STARTS && s0 + j < p.t && starts[s0 + j] != 0;
      if (STARTS) cuts |= (uint32_t)cut << j;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float na;
        gates(fv[c], &a[j][c], &na);
        b[j][c] = na * xv[c];
        if (!in) { a[j][c] = 1.f; b[j][c] = 0.f; }   // steps beyond the end change nothing
        H[c] = cut ? b[j][c] : fmaf(a[j][c], H[c], b[j][c]);
        A[c] = STARTS && (cut || A[c] < 0.f) ? kCut : A[c] * a[j][c];
      }
    }
    fetch(tile + ranks);
    float into_tile[C], v[C];
    join<C, STARTS, CLUSTER>(ex, buf, warp, rank, ranks, A, H, carry, into_tile, v);
    if (p.marks && warp == 0 && live && tile < p.n_marks) {
#pragma unroll
      for (int c = 0; c < C; ++c) p.marks[(i * p.n_marks + tile) * p.d + c0 + c] = into_tile[c];
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = STARTS && (cuts >> j & 1) ? b[j][c] : fmaf(a[j][c], v[c], b[j][c]);
      if (live && s0 + j < p.t) pack(v, reinterpret_cast<S *>(h + (s0 + j) * p.h_step));
    }
  }
  if (p.h_last && live && rank == 0 && warp == 0) {
#pragma unroll
    for (int c = 0; c < C; ++c) p.h_last[i * p.d + c0 + c] = carry[c];
  }
}

template <typename T, int C, bool STARTS, bool CLUSTER>
__global__ void __launch_bounds__(kTileThreads, 2) recurrence_grad_kernel(const RecurArgs p) {
  using S = Slice<T, C>;
  __shared__ Exchange<C> back;
  __shared__ float fore_a[2][kTileWarps][32 * C], fore_h[2][kTileWarps][32 * C];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ranks = CLUSTER ? p.cluster : 1;
  const int rank = CLUSTER ? (int)(blockIdx.x % ranks) : 0;
  const int64_t which = blockIdx.x / ranks;
  const int64_t i = which / p.blocks;
  const int64_t c0 = (which - i * p.blocks) * (32 * C) + lane * C;
  const bool live = c0 < p.d;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c0;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c0;
  const T *dh = static_cast<const T *>(p.dh) + i * p.dh_seq + c0;
  T *dx = static_cast<T *>(p.dx) + i * p.dx_seq + c0;
  T *df = static_cast<T *>(p.df) + i * p.df_seq + c0;
  const uint8_t *starts = STARTS ? p.starts + i * p.t : nullptr;

  float carry[C];   // c of the step after the group of tiles
#pragma unroll
  for (int c = 0; c < C; ++c) carry[c] = live && p.dh_last ? p.dh_last[i * p.d + c0 + c] : 0.f;
  S xr[kSteps], fr[kSteps], gr[kSteps];
  float mark[C];
  auto fetch = [&](int64_t tile) {   // a tile before the first has no step that is in range
    const int64_t s0 = tile * kTileSteps + warp * kSteps;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
      if (live && tile >= 0 && s0 + j < p.t) {
        xr[j] = *reinterpret_cast<const S *>(x + (s0 + j) * p.x_step);
        fr[j] = *reinterpret_cast<const S *>(f + (s0 + j) * p.f_step);
        gr[j] = *reinterpret_cast<const S *>(dh + (s0 + j) * p.dh_step);
      }
#pragma unroll
    for (int c = 0; c < C; ++c) mark[c] = live && tile >= 0 ? p.marks[(i * p.n_marks + tile) * p.d + c0 + c] : 0.f;
  };
  if (CLUSTER) cg::this_cluster().sync();
  fetch(p.n_marks - 1 - rank);
  int buf = 0;
  for (int64_t first = 0; first < p.n_marks; first += ranks, buf ^= 1) {
    const int64_t tile = p.n_marks - 1 - first - rank;
    const int64_t s0 = tile * kTileSteps + warp * kSteps;
    float a[kSteps][C], na[kSteps][C], A[C], H[C], L[C];
    float xv[kSteps][C], g[kSteps][C], from[C];
    uint32_t cuts = 0, ins = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) { A[c] = 1.f; H[c] = 0.f; L[c] = 0.f; from[c] = mark[c]; }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const bool in = live && tile >= 0 && s0 + j < p.t;
      float fv[C];
      unpack(xr[j], xv[j]);
      unpack(fr[j], fv);
      unpack(gr[j], g[j]);
      ins |= (uint32_t)in << j;
      const bool cut = STARTS && in && starts[s0 + j] != 0;
      if (STARTS) cuts |= (uint32_t)cut << j;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        gates(fv[c], &a[j][c], &na[j][c]);
        if (!in) { a[j][c] = 1.f; na[j][c] = 0.f; xv[j][c] = 0.f; g[j][c] = 0.f; }
        const float b = na[j][c] * xv[j][c];
        H[c] = cut ? b : fmaf(a[j][c], H[c], b);
        A[c] = STARTS && (cut || A[c] < 0.f) ? kCut : A[c] * a[j][c];
      }
    }
    fetch(tile - ranks);
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j)
#pragma unroll
      for (int c = 0; c < C; ++c) L[c] = STARTS && (cuts >> j & 1) ? 0.f : a[j][c] * (g[j][c] + L[c]);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      fore_a[buf][warp][lane * C + c] = A[c];
      fore_h[buf][warp][lane * C + c] = H[c];
    }
    float unused[C], l[C];
    join<C, STARTS, CLUSTER>(back, buf, kTileWarps - 1 - warp, rank, ranks, A, L, carry, unused, l);
    float before[kSteps][C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float v = from[c];
      for (int w = 0; w < kTileWarps; ++w) if (w < warp) v = follow<STARTS>(fore_a[buf][w][lane * C + c], fore_h[buf][w][lane * C + c], v);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        before[j][c] = STARTS && (cuts >> j & 1) ? 0.f : v;
        v = fmaf(a[j][c], before[j][c], na[j][c] * xv[j][c]);
        if (STARTS && (cuts >> j & 1)) v = na[j][c] * xv[j][c];
      }
    }
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
      float ox[C], of[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float lj = g[j][c] + l[c];
        const float n = na[j][c] * lj;
        ox[c] = n;
        of[c] = a[j][c] * n * (before[j][c] - xv[j][c]);
        l[c] = STARTS && (cuts >> j & 1) ? 0.f : a[j][c] * lj;
      }
      if (ins >> j & 1) {
        pack(ox, reinterpret_cast<S *>(dx + (s0 + j) * p.dx_step));
        pack(of, reinterpret_cast<S *>(df + (s0 + j) * p.df_step));
      }
    }
  }
  if (p.dh0 && live && rank == 0 && warp == 0) {
#pragma unroll
    for (int c = 0; c < C; ++c) p.dh0[i * p.d + c0 + c] = carry[c];
  }
}

// Few steps: a thread takes C channels of one sequence through all of them.  A single new token is this form.
template <typename T, int C> __global__ void __launch_bounds__(256) recurrence_few_kernel(const RecurArgs p, int64_t total) {
  using S = Slice<T, C>;
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= total) return;
  const int64_t per = p.d / C, i = k / per, c0 = (k - i * per) * C;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c0;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c0;
  T *ho = static_cast<T *>(p.h) + i * p.h_seq + c0;
  float h[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    h[c] = p.h0 ? p.h0[i * p.d + c0 + c] : 0.f;
    if (p.marks) p.marks[i * p.d + c0 + c] = h[c];   // at most kFewSteps steps have one mark
  }
#pragma unroll 4
  for (int64_t s = 0; s < p.t; ++s) {
    float xv[C], fv[C];
    unpack(*reinterpret_cast<const S *>(x + s * p.x_step), xv);
    unpack(*reinterpret_cast<const S *>(f + s * p.f_step), fv);
    const bool cut = p.starts && p.starts[i * p.t + s] != 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float a, na;
      gates(fv[c], &a, &na);
      const float b = na * xv[c];
      h[c] = cut ? b : fmaf(a, h[c], b);
    }
    pack(h, reinterpret_cast<S *>(ho + s * p.h_step));
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (p.h_last) p.h_last[i * p.d + c0 + c] = h[c];
}

__global__ void __launch_bounds__(256) recurrence_empty_kernel(const float *from, float *to, int64_t count) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k < count) to[k] = from ? from[k] : 0.f;
}

ceca_status_t done() { return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA; }

// t = 0: the state goes through unchanged (in place it is there already).
ceca_status_t pass_through(const float *from, float *to, int64_t count, cudaStream_t s) {
  if (!to || to == from) return CECA_OK;
  recurrence_empty_kernel<<<(unsigned)ceil_div(count, 256), 256, 0, s>>>(from, to, count);
  return done();
}

bool sizes_ok(int64_t b, int64_t t, int64_t d, int32_t type) {
  constexpr int64_t big = (int64_t)1 << 31;
  return b >= 1 && b < big && d >= 1 && d < big && b * ceil_div(d, 32) < big / kMaxCluster && t >= 0 && t < big && is_type(type);
}

bool strides_ok(int64_t d, int64_t seq, int64_t step) { return seq >= 0 && step >= d; }

// Whether pairs of channels can be loaded together: d even, every step of the tensor on a boundary of a pair.
bool pairs(const void *base, int64_t seq, int64_t step, int32_t type) {
  return (uintptr_t)base % (2 * type_bytes(type)) == 0 && seq % 2 == 0 && step % 2 == 0;
}

template <typename T, int C, bool STARTS, bool CLUSTER> cudaError_t launch(const RecurArgs &p, bool grad, int64_t b, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(b * p.blocks * p.cluster));
  cfg.blockDim = dim3(kTileThreads);
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim = {(unsigned)p.cluster, 1, 1};
  if (CLUSTER) { cfg.attrs = &at; cfg.numAttrs = 1; }
  auto kernel = grad ? recurrence_grad_kernel<T, C, STARTS, CLUSTER> : recurrence_kernel<T, C, STARTS, CLUSTER>;
  if (CLUSTER && p.cluster > 8) {   // more CTAs than every GPU has to offer together: allowed on this one
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T, int C> cudaError_t launch_tiles(const RecurArgs &p, bool grad, int64_t b, cudaStream_t s) {
  if (p.cluster > 1) return p.starts ? launch<T, C, true, true>(p, grad, b, s) : launch<T, C, false, true>(p, grad, b, s);
  return p.starts ? launch<T, C, true, false>(p, grad, b, s) : launch<T, C, false, false>(p, grad, b, s);
}

// CTAs along the steps: as many as there are tiles for, until two CTAs per SM are there.
int cluster_of(int64_t ctas, int64_t tiles) {
  int s = 1;
  while (s < kMaxCluster && s < tiles && ctas * s * 2 <= 2 * (int64_t)sm_count()) s *= 2;
  return s;
}

template <typename T, int C> cudaError_t run(RecurArgs p, bool grad, int64_t b, cudaStream_t s) {
  if (!grad && p.t <= kFewSteps) {
    const int64_t total = b * (p.d / C);
    recurrence_few_kernel<T, C><<<(unsigned)ceil_div(total, 256), 256, 0, s>>>(p, total);
    return cudaGetLastError();
  }
  p.blocks = (int32_t)ceil_div(p.d, 32 * C);
  p.cluster = cluster_of(b * p.blocks, p.n_marks);
  return launch_tiles<T, C>(p, grad, b, s);
}

ceca_status_t run_any(const RecurArgs &p, bool grad, bool two, int32_t type, int64_t b, cudaStream_t s) {
  cudaError_t e;
  if (type == DSGD_F32) e = two ? run<float, 2>(p, grad, b, s) : run<float, 1>(p, grad, b, s);
  else e = two ? run<bf16, 2>(p, grad, b, s) : run<bf16, 1>(p, grad, b, s);
  return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" int64_t dsgd_recurrence_marks(int64_t t) { return t <= 0 ? 0 : ceil_div(t, kTileSteps); }

extern "C" ceca_status_t dsgd_recurrence(const void *x, const void *f, const float *h0, const uint8_t *starts,
                                         void *h, float *h_last, float *marks, int64_t b, int64_t t, int64_t d,
                                         int64_t x_seq_stride, int64_t x_step_stride, int64_t f_seq_stride,
                                         int64_t f_step_stride, int64_t h_seq_stride, int64_t h_step_stride,
                                         int32_t type, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || !strides_ok(d, h_seq_stride, h_step_stride) ||
      (t > 0 && (!x || !f || !h || (b > 1 && h_seq_stride == 0))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(h0, h_last, b * d, s);
  RecurArgs p{};
  p.x = x; p.f = f; p.h0 = h0; p.starts = starts; p.h = h; p.h_last = h_last; p.marks = marks;
  p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.h_seq = h_seq_stride; p.h_step = h_step_stride;
  const bool two = d % 2 == 0 && pairs(x, x_seq_stride, x_step_stride, type) && pairs(f, f_seq_stride, f_step_stride, type) &&
                   pairs(h, h_seq_stride, h_step_stride, type);
  return run_any(p, false, two, type, b, s);
}

extern "C" ceca_status_t dsgd_recurrence_grad(const void *x, const void *f, const void *dh, const float *marks,
                                              const uint8_t *starts, const float *dh_last, void *dx, void *df,
                                              float *dh0, int64_t b, int64_t t, int64_t d, int64_t x_seq_stride,
                                              int64_t x_step_stride, int64_t f_seq_stride, int64_t f_step_stride,
                                              int64_t dh_seq_stride, int64_t dh_step_stride, int64_t dx_seq_stride,
                                              int64_t dx_step_stride, int64_t df_seq_stride, int64_t df_step_stride,
                                              int32_t type, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || dh_seq_stride < 0 || dh_step_stride < 0 ||
      !strides_ok(d, dx_seq_stride, dx_step_stride) || !strides_ok(d, df_seq_stride, df_step_stride) ||
      (t > 0 && (!x || !f || !dh || !marks || !dx || !df || (b > 1 && (dx_seq_stride == 0 || df_seq_stride == 0)))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(dh_last, dh0, b * d, s);
  RecurArgs p{};
  p.x = x; p.f = f; p.dh = dh; p.marks = const_cast<float *>(marks); p.starts = starts; p.dh_last = dh_last;
  p.dx = dx; p.df = df; p.dh0 = dh0;
  p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.dh_seq = dh_seq_stride; p.dh_step = dh_step_stride; p.dx_seq = dx_seq_stride; p.dx_step = dx_step_stride;
  p.df_seq = df_seq_stride; p.df_step = df_step_stride;
  const bool two = d % 2 == 0 && pairs(x, x_seq_stride, x_step_stride, type) && pairs(f, f_seq_stride, f_step_stride, type) &&
                   pairs(dh, dh_seq_stride, dh_step_stride, type) && pairs(dx, dx_seq_stride, dx_step_stride, type) &&
                   pairs(df, df_seq_stride, df_step_stride, type);
  return run_any(p, true, two, type, b, s);
}
