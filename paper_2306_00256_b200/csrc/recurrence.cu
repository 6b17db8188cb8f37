// Gated linear recurrence over a sequence and its gradient.
//
//   a = sigmoid(f),  h_s = keep_s h_{s-1} + (1 - a_s) x_s          (keep = a, or 0 where a document begins)
//   l_s = dh_s + keep_{s+1} l_{s+1},  dx_s = (1 - a_s) l_s,  df_s = a_s (1 - a_s) l_s (p_s - x_s),  dh0 = keep_0 l_0
//
// with p_s the state before step s (0 where a document begins).  States are carried in fp32.
//
// A run of steps maps the state before it to the state after it by h -> A h + H, and two such maps in a row are
// one again, so a sequence is cut into tiles and a tile into one run of kRun steps per warp (lanes are channels): every
// thread finds its own (A, H), the warps exchange theirs through shared memory, and each thread runs its steps once more
// from the state that reaches it.  x and f are read once and h is written once.  Where the channels alone do not
// fill the GPU, the sequences are cut into segments first, and another kernel finds the map of each.  All maps are
// composed in the order of the steps: the result does not depend on timing.  The gradient runs the same way from the
// end, with c_s = keep_s l_s in place of the state, and finds the states again from the marks that the forward call kept
// every kMarkSteps steps.
//
// Bytes bound it: 6 per element in bf16 forward, 10 for the gradient.  Lanes are channels so that the scan itself needs no
// shuffles, two bf16 channels to a lane so that it runs on f32x2 instructions, and runs are 16 steps because the exchange
// between warps costs the same for every run.  64 x 512 x 2048 bf16: forward 67 us (0.92 of the measured copy rate),
// gradient 128 us (0.80; 39 instructions an element, of which 12 are the gates and the two scans); in fp32 127 to 129 us (0.96)
// and 221 us (0.93).  8 x 4096 x 2048 bf16, 256 channel blocks and so CTAs of 8 warps, 256 of them on 296 places: 76 us (0.81) and
// 144 us (0.71), with documents' starts 79 and 146.  Few channels pay for the maps: 1 x 32768 x 1024 bf16 forward 66 us, of which 30
// are the first kernel.  Clusters of CTAs
// that exchanged the tiles' maps through distributed shared memory read everything once, but took 97 us there: their
// barrier was on the path from tile to tile.
//
// A document's first step ends what comes before it even when that is an infinity or a NaN, which no product with
// zero does: the A of a run that contains such a step is set to kCut, and a map with A = kCut is the constant H.
#include <algorithm>

#include "recurrence.cuh"

namespace ceca {
namespace {

constexpr int kFewSteps = 16;   // sequences up to here: one thread per channel

// Shared memory of a CTA: the runs on their way, then the exchange.
template <int L, bool WIDE, int WARPS> struct Shared {
  static constexpr int kStages = WARPS == 16 || !WIDE ? 2 : 3;
  Run<L, WIDE> runs[WARPS][kStages][2];   // x and f
  Exchange<L, WARPS> ex;
};

template <int L, bool WIDE, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS) recurrence_kernel(const RecurArgs p) {
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
  T *h = static_cast<T *>(p.h) + me.i * p.h_seq + me.c0;
  const uint8_t *starts = p.starts ? p.starts + me.i * p.t : nullptr;
  auto &mine = sh.runs[me.warp];

  constexpr int hop = WARPS * kRun;
  int64_t tile = me.seg * p.seg_tiles;
  const int64_t end = min(p.n_tiles, tile + p.seg_tiles), stop = min(p.t, end * hop);
  int64_t s0 = tile * hop + me.warp * kRun;   // the warp's run of the tile at hand
  auto begins = [&](int64_t from) { return starts && me.lane < kRun && from + me.lane < p.t ? (int)starts[from + me.lane] : 0; };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) {
    mine[k][0].fetch(x, p.x_step, s0 + k * hop, stop, me.width);
    mine[k][1].fetch(f, p.f_step, s0 + k * hop, stop, me.width);
    copies_end();
  }
  int begin = begins(s0);
  V carry;
  if (p.segs > 1) carry = arriving<L, WARPS>(p, me, sh.ex, me.seg + 1);
  else carry = p.h0 ? load<L>(p.h0 + me.i * p.d + me.c0, me.live) : all<C>(0.f);
  int stage = 0, buf = 0;
  for (; tile < end; ++tile, s0 += hop, buf ^= 1) {
    int ahead = stage + kStages - 1;
    ahead = ahead >= kStages ? ahead - kStages : ahead;
    __syncwarp();   // the run that is overwritten has been read by all lanes
    mine[ahead][0].fetch(x, p.x_step, s0 + (kStages - 1) * hop, stop, me.width);
    mine[ahead][1].fetch(f, p.f_step, s0 + (kStages - 1) * hop, stop, me.width);
    copies_end();
    const uint32_t cuts = __ballot_sync(0xffffffffu, begin != 0);
    begin = begins(s0 + hop);
    copies_wait<kStages - 1>();
    __syncwarp();
    const Run<L, WIDE> &xr = mine[stage][0], &fr = mine[stage][1];
    stage = stage + 1 == kStages ? 0 : stage + 1;
    const int left = (int)max((int64_t)0, min((int64_t)kRun, p.t - s0));   // steps of the run that exist
    V a[kRun], b[kRun], A = all<C>(1.f), H = all<C>(0.f);
    const Skew xk(x, p.x_step * sizeof(T), s0), fk(f, p.f_step * sizeof(T), s0);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      V na;
      gates(take<L>(fr.at(j, fk)), &a[j], &na);
      b[j] = mul(na, take<L>(xr.at(j, xk)));
    }
    if (left < kRun) {   // steps beyond the end change nothing
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (j >= left) { a[j] = all<C>(1.f); b[j] = all<C>(0.f); }
    }
    if (cuts) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) H = cuts >> j & 1 ? b[j] : fma(a[j], H, b[j]);
      A = all<C>(kCut);
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        H = fma(a[j], H, b[j]);
        A = mul(A, a[j]);
      }
    }
    V v;
    join(sh.ex, buf, me.warp, A, H, &carry, &v);
    if (p.marks && me.warp % kMarkRuns == 0 && s0 < p.t) store<L>(p.marks + (me.i * p.n_marks + s0 / kMarkSteps) * p.d + me.c0, v, me.live);
    T *o = h + s0 * p.h_step;
    if (left == kRun && !cuts) {
#pragma unroll
      for (int j = 0; j < kRun; ++j, o += p.h_step) {
        v = fma(a[j], v, b[j]);
        put<L>(o, v, me.live);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j, o += p.h_step) {
        v = cuts >> j & 1 ? b[j] : fma(a[j], v, b[j]);
        if (j < left) put<L>(o, v, me.live);
      }
    }
  }
  copies_wait<0>();
  if (p.h_last && me.seg == p.segs - 1 && me.warp == 0) store<L>(p.h_last + me.i * p.d + me.c0, carry, me.live);
}

// Few steps: a thread takes C channels of one sequence through all of them.  A single new token is this form.
template <int L> __global__ void __launch_bounds__(256) recurrence_few_kernel(const RecurArgs p, int64_t total) {
  using T = typename Lanes<L>::T;
  constexpr int C = Lanes<L>::kVals;
  using V = Val<C>;
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= total) return;
  const int64_t i = k / p.blocks, c = k - i * p.blocks;
  const int64_t c0 = L == HALVES ? (c & ~31) * 2 + (c & 31) : c * C;
  const Live live{c0 < p.d, L != F32 && c0 + Lanes<L>::kSecond < p.d};
  if (!live.x) return;
  const T *x = static_cast<const T *>(p.x) + i * p.x_seq + c0;
  const T *f = static_cast<const T *>(p.f) + i * p.f_seq + c0;
  T *ho = static_cast<T *>(p.h) + i * p.h_seq + c0;
  const int back = L == HALVES && !live.y ? -32 : 0;   // a lane without its second channel computes the first one twice
  auto both = [&](const T *q) {
    if constexpr (L == HALVES) return V{__bfloat162float(q[0]), __bfloat162float(q[32 + back])};
    else return take<L>(q);
  };
  V h = p.h0 ? load<L>(p.h0 + i * p.d + c0, live) : all<C>(0.f);
  if (p.marks) store<L>(p.marks + i * p.d + c0, h, live);   // so few steps have one mark
#pragma unroll 4
  for (int64_t s = 0; s < p.t; ++s) {
    const V xv = both(x + s * p.x_step), fv = both(f + s * p.f_step);
    V a, na;
    gates(fv, &a, &na);
    const V b = mul(na, xv);
    h = p.starts && p.starts[i * p.t + s] != 0 ? b : fma(a, h, b);
    put<L>(ho + s * p.h_step, h, live);
  }
  if (p.h_last) store<L>(p.h_last + i * p.d + c0, h, live);
}

struct Forward {
  RecurArgs p;
  int64_t b;
  cudaStream_t s;
  // the most warps of a CTA that its shared memory has room for
  template <bool WIDE> static constexpr int most() { return WIDE ? 16 : 8; }
  template <bool WIDE> static constexpr int resident() { return 4; }   // CTAs of 4 warps on an SM
  template <int L, bool WIDE> cudaError_t maps() {
    static std::atomic<uint64_t> done{0};
    return launch_kernel(recurrence_map_kernel<L, WIDE, false>, p, b, 4, sizeof(MapShared<L, WIDE>), &done, false, s);
  }
  template <int L, bool WIDE, int WARPS> cudaError_t run() {
    static std::atomic<uint64_t> done{0};
    return launch_kernel(recurrence_kernel<L, WIDE, WARPS>, p, b, WARPS, sizeof(Shared<L, WIDE, WARPS>), &done, p.segs > 1, s);
  }
};

template <int L> ceca_status_t run_few(RecurArgs p, int64_t b, cudaStream_t s) {
  p.blocks = (int32_t)(L == HALVES ? ceil_div(p.d, 64) * 32 : ceil_div(p.d, Lanes<L>::kVals));   // threads per sequence
  const int64_t total = b * p.blocks;
  recurrence_few_kernel<L><<<(unsigned)ceil_div(total, 256), 256, 0, s>>>(p, total);
  return done();
}

}  // namespace
}  // namespace ceca

using namespace ceca;

extern "C" int64_t dsgd_recurrence_marks(int64_t t) { return t <= 0 ? 0 : ceil_div(t, kMarkSteps); }

extern "C" size_t dsgd_recurrence_workspace_bytes(int64_t b, int64_t t, int64_t d) {
  return sizes_ok(b, t, d, DSGD_F32) && t > kFewSteps ? maps_bytes(b, t, d) : 0;
}

extern "C" ceca_status_t dsgd_recurrence(const void *x, const void *f, const float *h0, const uint8_t *starts,
                                         void *h, float *h_last, float *marks, int64_t b, int64_t t, int64_t d,
                                         int64_t x_seq_stride, int64_t x_step_stride, int64_t f_seq_stride,
                                         int64_t f_step_stride, int64_t h_seq_stride, int64_t h_step_stride,
                                         int32_t type, void *workspace, size_t workspace_bytes, void *stream) {
  if (!sizes_ok(b, t, d, type) || !strides_ok(d, x_seq_stride, x_step_stride) ||
      !strides_ok(d, f_seq_stride, f_step_stride) || !strides_ok(d, h_seq_stride, h_step_stride) ||
      (t > 0 && (!x || !f || !h || (b > 1 && h_seq_stride == 0))))
    return CECA_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t == 0) return pass_through(h0, h_last, b * d, s);
  const size_t need = dsgd_recurrence_workspace_bytes(b, t, d);
  if (need > 0 && (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16)) return CECA_ERR_WORKSPACE;
  RecurArgs p{};
  p.maps_a = static_cast<float *>(workspace);
  p.x = x; p.f = f; p.h0 = h0; p.starts = starts; p.h = h; p.h_last = h_last; p.marks = marks;
  p.t = t; p.d = d; p.n_marks = dsgd_recurrence_marks(t);
  p.x_seq = x_seq_stride; p.x_step = x_step_stride; p.f_seq = f_seq_stride; p.f_step = f_step_stride;
  p.h_seq = h_seq_stride; p.h_step = h_step_stride;
  const int in = std::min(alignment(x, x_seq_stride, x_step_stride, type), alignment(f, f_seq_stride, f_step_stride, type));
  const int out = alignment(h, h_seq_stride, h_step_stride, type);
  if (t <= kFewSteps)
    return type == DSGD_F32 ? run_few<F32>(p, b, s) : d % 2 == 0 && in >= 4 && out >= 4 ? run_few<PAIRS>(p, b, s) : run_few<HALVES>(p, b, s);
  return choose(Forward{p, b, s}, in, out, type);
}

