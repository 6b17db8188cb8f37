// The gradient of the gated linear recurrence (the mathematics and the split are in recurrence.cu): from the end of the
// sequence to its beginning, each tile first finding its runs' maps of both the states and of c_s = keep_s l_s, which
// share their A, then the states from the mark before it and c from the tiles after it.  The states are computed again
// rather than read: a mark of 4 bytes every 64 steps replaces a stream, and bf16 states would not be exact.  x and dh are
// read from shared memory where they are needed instead of being kept in registers: a, 1 - a and the differences take 96.
#include <algorithm>

#include "recurrence.cuh"

namespace ceca {
namespace {

// Shared memory of a CTA: the runs on their way, then the exchange.
template <int L, bool WIDE, int WARPS> struct Shared {
  static constexpr int kStages = 2;
  Run<L, WIDE> runs[WARPS][kStages][3];   // x, f and dh
  Exchange<L, WARPS> back;
  float fore_h[2][WARPS][32 * Lanes<L>::kVals];   // the runs' maps of the states; their A is back's
};

template <int L, bool WIDE, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS) recurrence_grad_kernel(const RecurArgs p) {
  using T = typename Lanes<L>::T;
  constexpr int C = Lanes<L>::kVals;
  using V = Val<C>;
  using Sh = Shared<L, WIDE, WARPS>;
  constexpr int kStages = Sh::kStages;
  static_assert(sizeof(Sh) <= kMaxShared);
  extern __shared__ __align__(16) char memory[];
  Sh &sh = *reinterpret_cast<Sh *>(memory);
  const Place<L> me(p);
  const T *x = static_cast<const T *>(p.x) + me.i * p.x_seq + me.first;
  const T *f = static_cast<const T *>(p.f) + me.i * p.f_seq + me.first;
  const T *dh = static_cast<const T *>(p.dh) + me.i * p.dh_seq + me.first;
  T *dx = static_cast<T *>(p.dx) + me.i * p.dx_seq + me.c0;
  T *df = static_cast<T *>(p.df) + me.i * p.df_seq + me.c0;
  const uint8_t *starts = p.starts ? p.starts + me.i * p.t : nullptr;
  const float *marks = p.marks + me.i * p.n_marks * p.d + me.c0;
  auto &mine = sh.runs[me.warp];

  constexpr int hop = WARPS * kRun;
  const int64_t first = me.seg * p.seg_tiles;
  int64_t tile = min(p.n_tiles, first + p.seg_tiles) - 1;
  int64_t s0 = tile * hop + me.warp * kRun;
  auto fetch = [&](int stage, int64_t from) {   // runs before the segment are not read
    from = from >= first * hop ? from : -1;
    mine[stage][0].fetch(x, p.x_step, from, p.t, me.width);
    mine[stage][1].fetch(f, p.f_step, from, p.t, me.width);
    mine[stage][2].fetch(dh, p.dh_step, from, p.t, me.width);
    copies_end();
  };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) fetch(k, s0 - k * hop);
  auto begins = [&](int64_t from) { return starts && me.lane < kRun && from >= 0 && from + me.lane < p.t ? (int)starts[from + me.lane] : 0; };
  int begin = begins(s0);
  V carry;   // c after the tile at hand
  if (p.segs > 1) carry = arriving<L, WARPS>(p, me, sh.back, p.segs - me.seg);
  else carry = p.dh_last ? load<L>(p.dh_last + me.i * p.d + me.c0, me.live) : all<C>(0.f);
  const int order = WARPS - 1 - me.warp, at = me.lane * C;
  int stage = 0, buf = 0;
  for (; tile >= first; --tile, s0 -= hop, buf ^= 1) {
    int ahead = stage + kStages - 1;
    ahead = ahead >= kStages ? ahead - kStages : ahead;
    __syncwarp();
    fetch(ahead, s0 - (kStages - 1) * hop);
    // the state before the marked group of runs that this one belongs to
    const int64_t group = s0 / kMarkSteps;
    V v = group < p.n_marks ? load<L>(marks + group * p.d, me.live) : all<C>(0.f);
    const uint32_t cuts = __ballot_sync(0xffffffffu, begin != 0);
    begin = begins(s0 - hop);
    copies_wait<kStages - 1>();
    __syncwarp();
    const Run<L, WIDE> &xr = mine[stage][0], &fr = mine[stage][1], &gr = mine[stage][2];
    stage = stage + 1 == kStages ? 0 : stage + 1;
    const int left = (int)max((int64_t)0, min((int64_t)kRun, p.t - s0));
    const Skew xk(x, p.x_step * sizeof(T), s0), fk(f, p.f_step * sizeof(T), s0), gk(dh, p.dh_step * sizeof(T), s0);
    auto xv = [&](int j) { return take<L>(xr.at(j, xk)); };
    auto gv = [&](int j) { return take<L>(gr.at(j, gk)); };
    V a[kRun], na[kRun], A = all<C>(1.f), H = all<C>(0.f), D = all<C>(0.f);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      gates(take<L>(fr.at(j, fk)), &a[j], &na[j]);
      A = mul(A, a[j]);
    }
    if (left < kRun) {   // steps beyond the end change nothing
      A = all<C>(1.f);
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        if (j >= left) { a[j] = all<C>(1.f); na[j] = all<C>(0.f); }
        A = mul(A, a[j]);
      }
    }
    if (cuts) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const V b = mul(na[j], xv(j));
        H = cuts >> j & 1 ? b : fma(a[j], H, b);
      }
#pragma unroll
      for (int j = kRun - 1; j >= 0; --j) D = cuts >> j & 1 ? all<C>(0.f) : mul(a[j], add(gv(j), D));
      A = all<C>(kCut);
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) H = fma(a[j], H, mul(na[j], xv(j)));
#pragma unroll
      for (int j = kRun - 1; j >= 0; --j) D = mul(a[j], add(gv(j), D));
    }
    write(&sh.fore_h[buf][me.warp][at], H);
    V l;
    join(sh.back, buf, order, A, D, &carry, &l);
    const int lead = me.warp / kMarkRuns * kMarkRuns;
#pragma unroll
    for (int w = 0; w < kMarkRuns - 1; ++w)
      if (lead + w < me.warp) v = follow(read(&sh.back.a[buf][WARPS - 1 - lead - w][at], A), read(&sh.fore_h[buf][lead + w][at], A), v);
    // q: the state before each step, less x
    V q[kRun];
    T *ox = dx + (s0 + kRun - 1) * p.dx_step, *of = df + (s0 + kRun - 1) * p.df_step;
    const auto give = [&](int j, V gx, V gf) {
      if (L == HALVES && left == kRun) {   // (spares two predicates a step)
        put<L>(ox, gx, me.live);
        put<L>(of, gf, me.live);
        ox -= p.dx_step;
        of -= p.df_step;
        return;
      }
      const Live in{me.live.x && j < left, me.live.y && j < left};
      put<L>(ox, gx, in);
      put<L>(of, gf, in);
      ox -= p.dx_step;
      of -= p.df_step;
    };
    if (cuts) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const V xj = xv(j), b = mul(na[j], xj);
        const bool cut = cuts >> j & 1;
        q[j] = sub(cut ? all<C>(0.f) : v, xj);
        v = cut ? b : fma(a[j], v, b);
      }
#pragma unroll
      for (int j = kRun - 1; j >= 0; --j) {
        l = add(gv(j), l);
        const V gx = mul(na[j], l), al = mul(a[j], l);
        give(j, gx, mul(mul(na[j], al), q[j]));
        l = cuts >> j & 1 ? all<C>(0.f) : al;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const V xj = xv(j);
        q[j] = sub(v, xj);
        v = fma(a[j], v, mul(na[j], xj));
      }
#pragma unroll
      for (int j = kRun - 1; j >= 0; --j) {
        l = add(gv(j), l);
        const V gx = mul(na[j], l);
        l = mul(a[j], l);
        give(j, gx, mul(mul(na[j], l), q[j]));
      }
    }
  }
  copies_wait<0>();
  if (p.dh0 && me.seg == 0 && me.warp == 0) store<L>(p.dh0 + me.i * p.d + me.c0, carry, me.live);
}

struct Backward {
  RecurArgs p;
  int64_t b;
  cudaStream_t s;
  // the most warps of a CTA that its shared memory has room for
  template <bool WIDE> static constexpr int most() { return WIDE ? 16 : 8; }
  template <bool WIDE> static constexpr int resident() { return WIDE ? 4 : 3; }   // CTAs of 4 warps on an SM
  template <int L, bool WIDE> cudaError_t maps() {
    static std::atomic<uint64_t> done{0};
    return launch_kernel(recurrence_map_kernel<L, WIDE, true>, p, b, 4, sizeof(MapShared<L, WIDE>), &done, false, s);
  }
  template <int L, bool WIDE, int WARPS> cudaError_t run() {
    static std::atomic<uint64_t> done{0};
    return launch_kernel(recurrence_grad_kernel<L, WIDE, WARPS>, p, b, WARPS, sizeof(Shared<L, WIDE, WARPS>), &done, p.segs > 1, s);
  }
};

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" ceca_status_t dsgd_recurrence_grad(const void *x, const void *f, const void *dh, const float *marks,
                                              const uint8_t *starts, const float *dh_last, void *dx, void *df,
                                              float *dh0, int64_t b, int64_t t, int64_t d, int64_t x_seq_stride,
                                              int64_t x_step_stride, int64_t f_seq_stride, int64_t f_step_stride,
                                              int64_t dh_seq_stride, int64_t dh_step_stride, int64_t dx_seq_stride,
                                              int64_t dx_step_stride, int64_t df_seq_stride, int64_t df_step_stride,
                                              int32_t type, void *workspace, size_t workspace_bytes, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || dh_seq_stride < 0 || dh_step_stride < 0 ||
      !strides_ok(d, dx_seq_stride, dx_step_stride) || !strides_ok(d, df_seq_stride, df_step_stride) ||
      (t > 0 && (!x || !f || !dh || !marks || !dx || !df || (b > 1 && (dx_seq_stride == 0 || df_seq_stride == 0)))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(dh_last, dh0, b * d, s);
  const size_t need = maps_bytes(b, t, d);
  if (need > 0 && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16)) return CECA_ERR_WORKSPACE;
  RecurArgs p{};
  p.maps_a = static_cast<float *>(workspace);
  p.x = x; p.f = f; p.dh = dh; p.marks = const_cast<float *>(marks); p.starts = starts; p.dh_last = dh_last;
  p.dx = dx; p.df = df; p.dh0 = dh0;
  p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.dh_seq = dh_seq_stride; p.dh_step = dh_step_stride; p.dx_seq = dx_seq_stride; p.dx_step = dx_step_stride;
  p.df_seq = df_seq_stride; p.df_step = df_step_stride;
  const int in = std::min({alignment(x, x_seq_stride, x_step_stride, type), alignment(f, f_seq_stride, f_step_stride, type),
                           alignment(dh, dh_seq_stride, dh_step_stride, type)});
  const int out = std::min(alignment(dx, dx_seq_stride, dx_step_stride, type), alignment(df, df_seq_stride, df_step_stride, type));
  return choose(Backward{p, b, s}, in, out, type);
}
