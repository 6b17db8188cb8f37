// Gated linear recurrence over a sequence and its gradient.
//
//   a = sigmoid(f),  h_s = keep_s h_{s-1} + (1 - a_s) x_s          (keep = a, or 0 where a document begins)
//   l_s = dh_s + keep_{s+1} l_{s+1},  dx_s = (1 - a_s) l_s,  df_s = a_s (1 - a_s) l_s (p_s - x_s),  dh0 = keep_0 l_0
//
// with p_s the state before step s (0 where a document begins).  States are carried in fp32.
//
// A run of steps maps the state before it to the state after it by h -> A h + H, and two such maps in a row are
// one again, so a sequence is cut into tiles of kTileSteps steps, a tile into one run of steps per warp (lanes are
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

constexpr int kTileSteps = 64;    // and the distance between two marks
constexpr int kMaxCluster = 16;
constexpr int kFewSteps = 16;     // sequences up to here: one thread per channel
constexpr float kCut = -1.f;
// Warps of a CTA; each takes kTileSteps / warps steps of a tile.  The forward call holds 2 fp32 values per element and
// prefetches its inputs, the gradient 3: these are what leaves 16 warps an SM without spilling.
constexpr int kWarps = 4, kGradWarps = 8;

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

// C adjacent channels in fp32; two are computed on together (f32x2).
template <int C> struct Val;
template <> struct Val<1> { float x; };
template <> struct Val<2> { float x, y; };
__device__ __forceinline__ uint64_t bits(Val<2> v) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
  return r;
}
__device__ __forceinline__ Val<2> halves(uint64_t r) {
  Val<2> v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ __forceinline__ Val<1> mul(Val<1> a, Val<1> b) { return {a.x * b.x}; }
__device__ __forceinline__ Val<1> add(Val<1> a, Val<1> b) { return {a.x + b.x}; }
__device__ __forceinline__ Val<1> sub(Val<1> a, Val<1> b) { return {a.x - b.x}; }
__device__ __forceinline__ Val<1> fma(Val<1> a, Val<1> b, Val<1> c) { return {fmaf(a.x, b.x, c.x)}; }
__device__ __forceinline__ Val<2> mul(Val<2> a, Val<2> b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return halves(r);
}
__device__ __forceinline__ Val<2> add(Val<2> a, Val<2> b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
  return halves(r);
}
__device__ __forceinline__ Val<2> fma(Val<2> a, Val<2> b, Val<2> c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
  return halves(r);
}
__device__ __forceinline__ Val<2> sub(Val<2> a, Val<2> b) { return fma(b, Val<2>{-1.f, -1.f}, a); }
template <int C> __device__ __forceinline__ Val<C> all(float v);
template <> __device__ __forceinline__ Val<1> all<1>(float v) { return {v}; }
template <> __device__ __forceinline__ Val<2> all<2>(float v) { return {v, v}; }
__device__ __forceinline__ Val<1> read(const float *p, Val<1>) { return {*p}; }
__device__ __forceinline__ Val<2> read(const float *p, Val<2>) {   // shared memory, 8-byte aligned
  const float2 v = *reinterpret_cast<const float2 *>(p);
  return {v.x, v.y};
}
__device__ __forceinline__ void write(float *p, Val<1> v) { *p = v.x; }
__device__ __forceinline__ void write(float *p, Val<2> v) { *reinterpret_cast<float2 *>(p) = make_float2(v.x, v.y); }
// fp32 arrays of the caller, which need not be aligned for pairs
__device__ __forceinline__ Val<1> load(const float *p, Val<1>) { return {p[0]}; }
__device__ __forceinline__ Val<2> load(const float *p, Val<2>) { return {p[0], p[1]}; }
__device__ __forceinline__ void store(float *p, Val<1> v) { p[0] = v.x; }
__device__ __forceinline__ void store(float *p, Val<2> v) { p[0] = v.x; p[1] = v.y; }

// C adjacent channels of one step, as stored: at most 4 bytes.
template <typename T, int C> struct Slice;
template <> struct Slice<float, 1> {
  float v;
  __device__ __forceinline__ Val<1> value() const { return {v}; }
  __device__ __forceinline__ void set(Val<1> a) { v = a.x; }
};
template <> struct Slice<bf16, 1> {
  bf16 v;
  __device__ __forceinline__ Val<1> value() const { return {__bfloat162float(v)}; }
  __device__ __forceinline__ void set(Val<1> a) { v = __float2bfloat16_rn(a.x); }
};
template <> struct Slice<bf16, 2> {
  uint32_t v;
  __device__ __forceinline__ Val<2> value() const {   // a bf16 is the upper half of the fp32 of the same value
    return {__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)};
  }
  __device__ __forceinline__ void set(Val<2> a) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a.x, a.y);
    v = *reinterpret_cast<const uint32_t *>(&h);
  }
};

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
constexpr float kNegLog2e = -1.4426950408889634f, kLeast = 0x1p-125f;
__device__ __forceinline__ void gates(Val<1> f, Val<1> *a, Val<1> *na) {
  const float e = ex2(fminf(f.x * kNegLog2e, 126.f));
  const float r = rcp(1.f + e);
  na->x = e * r;
  a->x = __saturatef(r - kLeast);
}
__device__ __forceinline__ void gates(Val<2> f, Val<2> *a, Val<2> *na) {
  Val<2> e = mul(f, all<2>(kNegLog2e));
  e.x = ex2(fminf(e.x, 126.f));
  e.y = ex2(fminf(e.y, 126.f));
  Val<2> r = add(e, all<2>(1.f));
  r.x = rcp(r.x);
  r.y = rcp(r.y);
  *na = mul(e, r);
  a->x = __saturatef(r.x - kLeast);
  a->y = __saturatef(r.y - kLeast);
}

// A run's map applied to what comes into it, and the map of a run with one more map (wa, wh) after it.
template <bool STARTS> __device__ __forceinline__ Val<1> follow(Val<1> A, Val<1> H, Val<1> in) {
  const Val<1> v = fma(A, in, H);
  return STARTS && A.x < 0.f ? H : v;
}
template <bool STARTS> __device__ __forceinline__ Val<2> follow(Val<2> A, Val<2> H, Val<2> in) {
  Val<2> v = fma(A, in, H);
  if (STARTS && A.x < 0.f) v = H;   // a document begins for all channels at once
  return v;
}
template <bool STARTS, int C> __device__ __forceinline__ Val<C> through(Val<C> A, Val<C> wa) {
  const Val<C> v = mul(A, wa);
  return STARTS && (A.x < 0.f || wa.x < 0.f) ? all<C>(kCut) : v;
}

// What the warps of a tile, and the tiles of a cluster, tell one another: the map of a run, per channel.
template <int C, int WARPS> struct Exchange {
  float warp_a[2][WARPS][32 * C], warp_h[2][WARPS][32 * C];
  float tile_a[2][kMaxCluster][32 * C], tile_h[2][kMaxCluster][32 * C];
};

// The thread's map enters the exchange; on return `carry` (what reaches the first run of the group of tiles) has
// become what reaches the group after this one, `into_tile` what reaches this tile and `into` what reaches this thread's
// run.  `order` is the warp's place in the direction of the recurrence.  One block barrier, and one cluster barrier
// where there is a cluster; `buf` alternates, so that what is still read is not overwritten.
template <int C, int WARPS, bool STARTS, bool CLUSTER>
__device__ __forceinline__ void join(Exchange<C, WARPS> &ex, int buf, int order, int rank, int ranks, Val<C> A, Val<C> H,
                                     Val<C> *carry, Val<C> *into_tile, Val<C> *into) {
  const int at = (threadIdx.x & 31) * C;
  write(&ex.warp_a[buf][order][at], A);
  write(&ex.warp_h[buf][order][at], H);
  __syncthreads();
  if (CLUSTER) {
    if (threadIdx.x < 32) {
      Val<C> ta = all<C>(1.f), th = all<C>(0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const Val<C> wa = read(&ex.warp_a[buf][w][at], A);
        th = follow<STARTS>(wa, read(&ex.warp_h[buf][w][at], A), th);
        ta = through<STARTS>(ta, wa);
      }
      cg::cluster_group cl = cg::this_cluster();
      for (int r = 0; r < ranks; ++r) {
        write(cl.map_shared_rank(&ex.tile_a[buf][rank][at], r), ta);
        write(cl.map_shared_rank(&ex.tile_h[buf][rank][at], r), th);
      }
    }
    cg::this_cluster().sync();
  }
  Val<C> v = *carry, mine = v;
  if (CLUSTER) {
    for (int r = 0; r < ranks; ++r) {
      if (r == rank) mine = v;
      v = follow<STARTS>(read(&ex.tile_a[buf][r][at], A), read(&ex.tile_h[buf][r][at], A), v);
    }
    *carry = v;
    v = mine;
  }
  *into_tile = v;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w == order) mine = v;
    v = follow<STARTS>(read(&ex.warp_a[buf][w][at], A), read(&ex.warp_h[buf][w][at], A), v);
  }
  *into = mine;
  if (!CLUSTER) *carry = v;
}

// Where a CTA works: the sequence, the channels of its lanes, its place in the cluster.  Lanes beyond d read the last
// channels and store nothing.
template <int C> struct Place {
  int64_t i, c0;
  int lane, warp, rank, ranks;
  bool live;
  __device__ __forceinline__ Place(const RecurArgs &p, bool cluster) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    ranks = cluster ? p.cluster : 1;
    const uint32_t which = cluster ? blockIdx.x / ranks : blockIdx.x;
    rank = cluster ? (int)(blockIdx.x - which * ranks) : 0;
    i = which / (uint32_t)p.blocks;
    c0 = (int64_t)(which - (uint32_t)i * p.blocks) * (32 * C) + lane * C;
    live = c0 < p.d;
    if (!live) c0 = p.d - C;
  }
};

// The steps [s0, s0 + N) of a stream; those outside [0, t) read as `beyond`.
template <typename T, int C, int N>
__device__ __forceinline__ void fetch(Slice<T, C> *to, const T *p, int64_t step, int64_t s0, int64_t t, float beyond) {
  if (s0 >= 0 && s0 + N <= t) {
    p += s0 * step;
#pragma unroll
    for (int j = 0; j < N; ++j, p += step) to[j] = *reinterpret_cast<const Slice<T, C> *>(p);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      to[j].set(all<C>(beyond));
      if (s0 + j >= 0 && s0 + j < t) to[j] = *reinterpret_cast<const Slice<T, C> *>(p + (s0 + j) * step);
    }
  }
}

// Steps beyond the end are read as a gate held open (f = +infinity: a = 1, na = 0) on zeros: they change nothing.
template <typename T, int C, bool STARTS, bool CLUSTER>
__global__ void __launch_bounds__(32 * kWarps, 4) recurrence_kernel(const RecurArgs p) {
  constexpr int N = kTileSteps / kWarps;
  using S = Slice<T, C>;
  using V = Val<C>;
  __shared__ Exchange<C, kWarps> ex;
  const Place<C> me(p, CLUSTER);
  const T *x = static_cast<const T *>(p.x) + me.i * p.x_seq + me.c0;
  const T *f = static_cast<const T *>(p.f) + me.i * p.f_seq + me.c0;
  T *h = static_cast<T *>(p.h) + me.i * p.h_seq + me.c0;
  const uint8_t *starts = STARTS ? p.starts + me.i * p.t : nullptr;

  V carry = p.h0 ? load(p.h0 + me.i * p.d + me.c0, V{}) : all<C>(0.f);
  S xr[N], fr[N];
  int cut = 0;
  auto next = [&](int64_t s0) {
    fetch<T, C, N>(xr, x, p.x_step, s0, p.t, 0.f);
    fetch<T, C, N>(fr, f, p.f_step, s0, p.t, INFINITY);
    if (STARTS) cut = me.lane < N && s0 + me.lane < p.t ? starts[s0 + me.lane] : 0;
  };
  if (CLUSTER) cg::this_cluster().sync();   // every CTA runs before anybody writes into its shared memory
  int64_t tile = me.rank;
  next(tile * kTileSteps + me.warp * N);
  for (int buf = 0; tile - me.rank < p.n_marks; tile += me.ranks, buf ^= 1) {
    const int64_t s0 = tile * kTileSteps + me.warp * N;
    const uint32_t cuts = STARTS ? __ballot_sync(0xffffffffu, cut != 0) : 0;
    V a[N], b[N], A = all<C>(1.f), H = all<C>(0.f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      V na;
      gates(fr[j].value(), &a[j], &na);
      b[j] = mul(na, xr[j].value());
      H = fma(a[j], H, b[j]);
      A = mul(A, a[j]);
      if (STARTS && (cuts >> j & 1)) H = b[j];
    }
    if (STARTS && cuts) A = all<C>(kCut);
    next(s0 + me.ranks * kTileSteps);
    V into_tile, v;
    join<C, kWarps, STARTS, CLUSTER>(ex, buf, me.warp, me.rank, me.ranks, A, H, &carry, &into_tile, &v);
    if (p.marks && me.warp == 0 && me.live && tile < p.n_marks)
      store(p.marks + (me.i * p.n_marks + tile) * p.d + me.c0, into_tile);
    T *o = h + s0 * p.h_step;
    if (s0 + N <= p.t) {
#pragma unroll
      for (int j = 0; j < N; ++j, o += p.h_step) {
        v = fma(a[j], v, b[j]);
        if (STARTS && (cuts >> j & 1)) v = b[j];
        if (me.live) reinterpret_cast<S *>(o)->set(v);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j, o += p.h_step) {
        v = fma(a[j], v, b[j]);
        if (STARTS && (cuts >> j & 1)) v = b[j];
        if (me.live && s0 + j < p.t) reinterpret_cast<S *>(o)->set(v);
      }
    }
  }
  if (p.h_last && me.live && me.rank == 0 && me.warp == 0) store(p.h_last + me.i * p.d + me.c0, carry);
}

template <typename T, int C, bool STARTS, bool CLUSTER>
__global__ void __launch_bounds__(32 * kGradWarps, 2) recurrence_grad_kernel(const RecurArgs p) {
  constexpr int N = kTileSteps / kGradWarps;
  using S = Slice<T, C>;
  using V = Val<C>;
  __shared__ Exchange<C, kGradWarps> back;
  __shared__ float fore_h[2][kGradWarps][32 * C];   // the same runs' maps of the states; their A is back's
  const Place<C> me(p, CLUSTER);
  const T *x = static_cast<const T *>(p.x) + me.i * p.x_seq + me.c0;
  const T *f = static_cast<const T *>(p.f) + me.i * p.f_seq + me.c0;
  const T *dh = static_cast<const T *>(p.dh) + me.i * p.dh_seq + me.c0;
  T *dx = static_cast<T *>(p.dx) + me.i * p.dx_seq + me.c0;
  T *df = static_cast<T *>(p.df) + me.i * p.df_seq + me.c0;
  const uint8_t *starts = STARTS ? p.starts + me.i * p.t : nullptr;
  const float *marks = p.marks + me.i * p.n_marks * p.d + me.c0;

  V carry = p.dh_last ? load(p.dh_last + me.i * p.d + me.c0, V{}) : all<C>(0.f);   // c after the group of tiles
  S xr[N], fr[N], gr[N];
  V mark;
  int cut = 0;
  auto next = [&](int64_t s0, int64_t tile) {   // a tile before the first lies beyond the end as well
    fetch<T, C, N>(xr, x, p.x_step, s0, p.t, 0.f);
    fetch<T, C, N>(fr, f, p.f_step, s0, p.t, INFINITY);
    fetch<T, C, N>(gr, dh, p.dh_step, s0, p.t, 0.f);
    mark = tile >= 0 ? load(marks + tile * p.d, V{}) : all<C>(0.f);
    if (STARTS) cut = me.lane < N && s0 >= 0 && s0 + me.lane < p.t ? starts[s0 + me.lane] : 0;
  };
  if (CLUSTER) cg::this_cluster().sync();
  int64_t tile = p.n_marks - 1 - me.rank;
  next(tile * kTileSteps + me.warp * N, tile);
  const int order = kGradWarps - 1 - me.warp, at = me.lane * C;
  for (int buf = 0; tile + me.rank >= 0; tile -= me.ranks, buf ^= 1) {
    const int64_t s0 = tile * kTileSteps + me.warp * N;
    const uint32_t cuts = STARTS ? __ballot_sync(0xffffffffu, cut != 0) : 0;
    V a[N], na[N], A = all<C>(1.f), H = all<C>(0.f), L = all<C>(0.f), v = mark;
    S xs[N], gs[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      gates(fr[j].value(), &a[j], &na[j]);
      xs[j] = xr[j];
      gs[j] = gr[j];
      const V b = mul(na[j], xs[j].value());
      H = fma(a[j], H, b);
      A = mul(A, a[j]);
      if (STARTS && (cuts >> j & 1)) H = b;
    }
    if (STARTS && cuts) A = all<C>(kCut);
    next(s0 - me.ranks * kTileSteps, tile - me.ranks);
#pragma unroll
    for (int j = N - 1; j >= 0; --j) {
      L = mul(a[j], add(gs[j].value(), L));
      if (STARTS && (cuts >> j & 1)) L = all<C>(0.f);
    }
    write(&fore_h[buf][me.warp][at], H);
    V unused, l;
    join<C, kGradWarps, STARTS, CLUSTER>(back, buf, order, me.rank, me.ranks, A, L, &carry, &unused, &l);
#pragma unroll
    for (int w = 0; w < kGradWarps - 1; ++w)
      if (w < me.warp) v = follow<STARTS>(read(&back.warp_a[buf][kGradWarps - 1 - w][at], A), read(&fore_h[buf][w][at], A), v);
    V before[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      before[j] = v;
      const V b = mul(na[j], xs[j].value());
      v = fma(a[j], v, b);
      if (STARTS && (cuts >> j & 1)) {
        before[j] = all<C>(0.f);
        v = b;
      }
    }
    T *ox = dx + (s0 + N - 1) * p.dx_step, *of = df + (s0 + N - 1) * p.df_step;
    const int64_t left = tile < 0 ? 0 : p.t - s0;   // steps of the run that exist
#pragma unroll
    for (int j = N - 1; j >= 0; --j, ox -= p.dx_step, of -= p.df_step) {
      l = add(gs[j].value(), l);
      const V gx = mul(na[j], l), al = mul(a[j], l);
      const V gf = mul(mul(a[j], gx), sub(before[j], xs[j].value()));
      if (me.live && j < left) {
        reinterpret_cast<S *>(ox)->set(gx);
        reinterpret_cast<S *>(of)->set(gf);
      }
      l = STARTS && (cuts >> j & 1) ? all<C>(0.f) : al;
    }
  }
  if (p.dh0 && me.live && me.rank == 0 && me.warp == 0) store(p.dh0 + me.i * p.d + me.c0, carry);
}

// Few steps: a thread takes C channels of one sequence through all of them.  A single new token is this form.
template <typename T, int C> __global__ void __launch_bounds__(256) recurrence_few_kernel(const RecurArgs p, int64_t total) {
  using S = Slice<T, C>;
  using V = Val<C>;
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= total) return;
  const int64_t per = p.d / C, i = k / per, c0 = (k - i * per) * C;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c0;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c0;
  T *ho = static_cast<T *>(p.h) + i * p.h_seq + c0;
  V h = p.h0 ? load(p.h0 + i * p.d + c0, V{}) : all<C>(0.f);
  if (p.marks) store(p.marks + i * p.d + c0, h);   // so few steps have one mark
#pragma unroll 4
  for (int64_t s = 0; s < p.t; ++s) {
    const V xv = reinterpret_cast<const S *>(x + s * p.x_step)->value();
    const V fv = reinterpret_cast<const S *>(f + s * p.f_step)->value();
    V a, na;
    gates(fv, &a, &na);
    const V b = mul(na, xv);
    h = p.starts && p.starts[i * p.t + s] != 0 ? b : fma(a, h, b);
    reinterpret_cast<S *>(ho + s * p.h_step)->set(h);
  }
  if (p.h_last) store(p.h_last + i * p.d + c0, h);
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

// Whether two bf16 channels can be loaded together: every step of the tensor on a 4-byte boundary (and d even).
bool pairs(const void *base, int64_t seq, int64_t step) { return (uintptr_t)base % 4 == 0 && seq % 2 == 0 && step % 2 == 0; }

template <typename T, int C, bool STARTS, bool CLUSTER> cudaError_t launch(const RecurArgs &p, bool grad, int64_t b, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(b * p.blocks * p.cluster));
  cfg.blockDim = dim3(32 * (grad ? kGradWarps : kWarps));
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim = {(unsigned)p.cluster, 1, 1};
  if (CLUSTER) { cfg.attrs = &at; cfg.numAttrs = 1; }
  auto kernel = grad ? recurrence_grad_kernel<T, C, STARTS, CLUSTER> : recurrence_kernel<T, C, STARTS, CLUSTER>;
  if (CLUSTER && p.cluster > 8) {   // more CTAs together than every GPU has to offer: allowed on this one
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

// CTAs along the steps: as many as there are tiles for, until the SMs are full (4 CTAs of the forward kernel, 2 of the
// gradient's on each).
int cluster_of(int64_t ctas, int64_t tiles, bool grad) {
  const int64_t room = (int64_t)sm_count() * (grad ? 2 : 4) / ctas;
  return (int)std::max<int64_t>(1, std::min({room, tiles, (int64_t)kMaxCluster}));
}

template <typename T, int C> cudaError_t run(RecurArgs p, bool grad, int64_t b, cudaStream_t s) {
  if (!grad && p.t <= kFewSteps) {
    const int64_t total = b * (p.d / C);
    recurrence_few_kernel<T, C><<<(unsigned)ceil_div(total, 256), 256, 0, s>>>(p, total);
    return cudaGetLastError();
  }
  p.blocks = (int32_t)ceil_div(p.d, 32 * C);
  p.cluster = cluster_of(b * p.blocks, p.n_marks, grad);
  if (p.cluster > 1) return p.starts ? launch<T, C, true, true>(p, grad, b, s) : launch<T, C, false, true>(p, grad, b, s);
  return p.starts ? launch<T, C, true, false>(p, grad, b, s) : launch<T, C, false, false>(p, grad, b, s);
}

ceca_status_t run_any(const RecurArgs &p, bool grad, bool two, int32_t type, int64_t b, cudaStream_t s) {
  cudaError_t e;
  if (type == DSGD_F32) e = run<float, 1>(p, grad, b, s);
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
  const bool two = d % 2 == 0 && pairs(x, x_seq_stride, x_step_stride) && pairs(f, f_seq_stride, f_step_stride) &&
                   pairs(h, h_seq_stride, h_step_stride);
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
  const bool two = d % 2 == 0 && pairs(x, x_seq_stride, x_step_stride) && pairs(f, f_seq_stride, f_step_stride) &&
                   pairs(dh, dh_seq_stride, dh_step_stride) && pairs(dx, dx_seq_stride, dx_step_stride) &&
                   pairs(df, df_seq_stride, df_step_stride);
  return run_any(p, true, two, type, b, s);
}
