// Internal: what the two recurrence kernels share.  See recurrence.cu for the mathematics and the split.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "ceca.h"
#include "tma.h"
#include "values.h"

namespace ceca {
namespace {

constexpr int kRun = 16;          // steps of a warp's run
constexpr int kMarkSteps = 64;    // distance between two marks, kMarkRuns runs
constexpr int kMarkRuns = kMarkSteps / kRun;
constexpr int kMaxShared = 227 * 1024;
constexpr float kCut = -1.f;

struct RecurArgs {
  const void *x, *f, *dh;
  const float *h0, *dh_last;
  const uint8_t *starts;
  void *h, *dx, *df;
  float *h_last, *dh0;
  float *marks;
  float *maps_a, *maps_h;   // b x (segs + 1) x d: what reaches the first segment, then each segment's map
  int64_t t, d, n_marks, n_tiles, seg_tiles;
  int64_t x_seq, x_step, f_seq, f_step, h_seq, h_step, dh_seq, dh_step, dx_seq, dx_step, df_seq, df_step;
  int32_t blocks;   // channel blocks per sequence
  int32_t segs;     // segments of a sequence, of seg_tiles tiles each
};

// How a warp's 32 lanes hold the channels of a step, 128 bytes of them, and how these come and go.
//   F32:   one channel a lane
//   PAIRS: two adjacent bf16 channels a lane, every step on a 4-byte boundary
//   HALVES: bf16 channels lane and lane + 32; steps may begin on any element
enum Layout { F32, PAIRS, HALVES };
template <int L> struct Lanes {
  using T = bf16;
  static constexpr int kVals = 2, kChannels = 64, kFirst = L == PAIRS ? 2 : 1, kSecond = L == PAIRS ? 1 : 32;
};
template <> struct Lanes<F32> {
  using T = float;
  static constexpr int kVals = 1, kChannels = 32, kFirst = 1, kSecond = 0;
};

// The channels' values at `p`, which points at the lane's first one (in shared or global memory).
template <int L> __device__ __forceinline__ Val<Lanes<L>::kVals> take(const typename Lanes<L>::T *p) {
  if constexpr (L == F32) {
    return {*p};
  } else if constexpr (L == PAIRS) {   // a bf16 is the upper half of the fp32 of the same value
    const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
    return {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  } else {
    return {__bfloat162float(p[0]), __bfloat162float(p[32])};
  }
}
// Which of the lane's channels exist.
struct Live { bool x, y; };
template <int L> __device__ __forceinline__ void put(typename Lanes<L>::T *p, Val<Lanes<L>::kVals> v, Live live) {
  if constexpr (L == F32) {
    if (live.x) *p = v.x;
  } else if constexpr (L == PAIRS) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    if (live.x) *reinterpret_cast<__nv_bfloat162 *>(p) = h;
  } else {
    if (live.x) p[0] = __float2bfloat16_rn(v.x);
    if (live.y) p[32] = __float2bfloat16_rn(v.y);
  }
}
// fp32 arrays of the caller
template <int L> __device__ __forceinline__ Val<Lanes<L>::kVals> load(const float *p, Live live) {
  if constexpr (L == F32) return {live.x ? p[0] : 0.f};
  else return {live.x ? p[0] : 0.f, live.y ? p[Lanes<L>::kSecond] : 0.f};
}
template <int L> __device__ __forceinline__ void store(float *p, Val<Lanes<L>::kVals> v, Live live) {
  if (live.x) p[0] = v.x;
  if constexpr (L != F32)
    if (live.y) p[Lanes<L>::kSecond] = v.y;
}

// Asynchronous copies to shared memory; bytes beyond `have` become zeros and are not read.
__device__ __forceinline__ void copy16(uint32_t to, const void *from, int have) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(have) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Where the steps of a run begin between 16-byte boundaries: the first one, and how far it moves from step to step.
struct Skew {
  uint32_t first, step;
  __device__ __forceinline__ Skew(const void *p, int64_t step_bytes, int64_t s0)
      : first((uint32_t)(reinterpret_cast<uintptr_t>(p) + step_bytes * s0)), step((uint32_t)step_bytes) {}
  __device__ __forceinline__ uint32_t of(int j) const { return (first + j * step) & 15; }
};

// The kRun steps of one stream for one warp, brought by that warp itself: nobody else waits for them.  WIDE: every step
// begins on a 16-byte boundary.  Otherwise a step's 128 bytes are copied as the nine 16-byte words that hold them, and
// found at the step's skew; of a first word, what lies before the step is another channel's or another tensor's, in the
// same allocation (none begins inside such a word), and is not used.
template <int L, bool WIDE> struct Run {
  using T = typename Lanes<L>::T;
  static constexpr int kPitch = WIDE ? 128 : 144;
  alignas(16) char bytes[kRun * kPitch];

  // p: the stream's first channel of this warp at step 0; width: bytes of a step that exist from there on (up to 128).
  // Steps and channels that do not exist become zeros.
  __device__ __forceinline__ void fetch(const T *p, int64_t step, int64_t s0, int64_t t, int width) {
    const int lane = threadIdx.x & 31;
    const uint32_t to = smem_u32(bytes);
    const int left = s0 < 0 ? 0 : (int)max((int64_t)0, min((int64_t)kRun, t - s0));
    const int64_t hop = step * (int64_t)sizeof(T);
    const char *base = reinterpret_cast<const char *>(p) + s0 * hop;
    if constexpr (WIDE) {
      const int row = lane >> 3, col = (lane & 7) * 16;
      const char *from = base + row * hop + col;
      const uint32_t at = to + row * kPitch + col;
      if (left == kRun && width == 128) {
#pragma unroll
        for (int k = 0; k < kRun / 4; ++k) copy16(at + 4 * k * kPitch, from + 4 * k * hop);
      } else {
        const int have = max(0, min(16, width - col));
        for (int k = 0; k < kRun / 4; ++k) {
          const bool in = row + 4 * k < left && have > 0;
          copy16(at + 4 * k * kPitch, in ? from + 4 * k * hop : reinterpret_cast<const char *>(p), in ? have : 0);
        }
      }
    } else {
      const auto copy = [&](int k) {
        const int row = k / 9, col = (k - row * 9) * 16;
        const char *from = base + row * hop;
        const int skew = (int)(reinterpret_cast<uintptr_t>(from) & 15), have = min(16, width + skew - col);
        if (have > 0) copy16(to + row * kPitch + col, from - skew + col, have);
      };
      if (left == kRun) {
#pragma unroll
        for (int i = 0; i < kRun * 9 / 32; ++i) copy(lane + 32 * i);
        if (lane < kRun * 9 % 32) copy(lane + kRun * 9 / 32 * 32);
      } else {
#pragma unroll 1
        for (int k = lane; k < kRun * 9; k += 32) {
          if (k / 9 < left) copy(k);
          else *reinterpret_cast<uint4 *>(bytes + k * 16) = make_uint4(0, 0, 0, 0);
        }
      }
    }
  }
  // the lane's first channel of step j
  __device__ __forceinline__ const T *at(int j, const Skew &skew) const {
    return reinterpret_cast<const T *>(bytes + j * kPitch + (WIDE ? 0 : skew.of(j))) + (threadIdx.x & 31) * Lanes<L>::kFirst;
  }
};

// a = sigmoid(f) and na = sigmoid(-f): with e = exp(-f), a = 1 / (1 + e) and na = e a.  Each is within a few ulp of itself plus
// |f| ulp or so: the product f log2(e) is rounded before its exponential is taken, which is a choice (its low half would
// take two more instructions a gate, and where |f| is large enough to matter one of the two is next to 0 and the other next to 1).
// The exponent stops at 126, where e and its reciprocal are both still normal numbers and na rounds to 1; the
// subtraction then makes a exactly 0 and changes no a above 2^-101.  (a does not leave [0, 1]: the reciprocal of 1 is 1, that of
// 2^126 is 2^-126, and between them its last place does not reach beyond either.)  A NaN is not above 126 and goes
// through.
constexpr float kNegLog2e = -1.4426950408889634f, kLeast = 0x1p-126f;
__device__ __forceinline__ float least_or_nan(float x, float y) { return x > y ? y : x; }
__device__ __forceinline__ void gates(Val<1> f, Val<1> *a, Val<1> *na) {
  const float e = ex2(least_or_nan(f.x * kNegLog2e, 126.f));
  const float r = rcp(1.f + e);
  na->x = e * r;
  a->x = r - kLeast;
}
__device__ __forceinline__ void gates(Val<2> f, Val<2> *a, Val<2> *na) {
  Val<2> e = mul(f, all<2>(kNegLog2e));
  e.x = ex2(least_or_nan(e.x, 126.f));
  e.y = ex2(least_or_nan(e.y, 126.f));
  Val<2> r = add(e, all<2>(1.f));
  r.x = rcp(r.x);
  r.y = rcp(r.y);
  *na = mul(e, r);
  *a = add(r, all<2>(-kLeast));
}

// A run's map applied to what comes into it, and the map of a run with one more map (wa, wh) after it.
__device__ __forceinline__ Val<1> follow(Val<1> A, Val<1> H, Val<1> in) {
  const Val<1> v = fma(A, in, H);
  return A.x < 0.f ? H : v;
}
__device__ __forceinline__ Val<2> follow(Val<2> A, Val<2> H, Val<2> in) {
  Val<2> v = fma(A, in, H);
  if (A.x < 0.f) v = H;   // a document begins for all channels at once
  return v;
}
template <int C> __device__ __forceinline__ Val<C> through(Val<C> A, Val<C> wa) {
  const Val<C> v = mul(A, wa);
  return A.x < 0.f || wa.x < 0.f ? all<C>(kCut) : v;
}

// What the warps of a CTA tell one another: the map of a run, per channel.
template <int L, int WARPS> struct Exchange {
  float a[2][WARPS][32 * Lanes<L>::kVals], h[2][WARPS][32 * Lanes<L>::kVals];
};

// The thread's map enters the exchange; on return `carry` (what reaches the first run of the tile) has become what
// reaches the next tile, and `into` is what reaches this thread's run.  `order` is the warp's place in the direction
// of the recurrence.  One block barrier; `buf` alternates, so that what is still read is not overwritten.
template <int L, int WARPS, int C>
__device__ __forceinline__ void join(Exchange<L, WARPS> &ex, int buf, int order, Val<C> A, Val<C> H, Val<C> *carry, Val<C> *into) {
  const int at = (threadIdx.x & 31) * C;
  write(&ex.a[buf][order][at], A);
  write(&ex.h[buf][order][at], H);
  __syncthreads();
  Val<C> v = *carry, mine = v;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w == order) mine = v;
    v = follow(read(&ex.a[buf][w][at], A), read(&ex.h[buf][w][at], A), v);
  }
  *into = mine;
  *carry = v;
}

// Where a CTA works: the sequence, its first channel and the lanes' own, the segment.
template <int L> struct Place {
  int64_t i, first, c0;
  int lane, warp, seg, width;
  Live live;
  __device__ __forceinline__ explicit Place(const RecurArgs &p) {
    lane = threadIdx.x & 31;
    warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);   // one value for the warp, and known to be
    const uint32_t which = blockIdx.x / (uint32_t)p.segs;
    seg = (int)(blockIdx.x - which * p.segs);
    i = which / (uint32_t)p.blocks;
    first = (int64_t)(which - (uint32_t)i * p.blocks) * Lanes<L>::kChannels;
    c0 = first + lane * Lanes<L>::kFirst;
    live.x = c0 < p.d;
    live.y = L != F32 && c0 + Lanes<L>::kSecond < p.d;
    width = (int)min((int64_t)128, (p.d - first) * (int64_t)sizeof(typename Lanes<L>::T));
  }
  // the lane's place in entry k of the maps
  __device__ __forceinline__ int64_t map(const RecurArgs &p, int k) const { return (i * (p.segs + 1) + k) * p.d + c0; }
};

// What reaches a segment: the maps of all segments before it (in the direction of the recurrence), the warps each
// composing a part of them.  Takes the exchange's second buffer and one block barrier.
template <int L, int WARPS>
__device__ __forceinline__ Val<Lanes<L>::kVals> arriving(const RecurArgs &p, const Place<L> &me, Exchange<L, WARPS> &ex, int entries) {
  constexpr int C = Lanes<L>::kVals;
  using V = Val<C>;
  after_first();
  const int per = (entries + WARPS - 1) / WARPS, from = me.warp * per, to = min(entries, from + per);
  V A = all<C>(1.f), H = all<C>(0.f);
#pragma unroll 4
  for (int k = from; k < to; ++k) {
    const V wa = load<L>(p.maps_a + me.map(p, k), me.live), wh = load<L>(p.maps_h + me.map(p, k), me.live);
    H = follow(wa, wh, H);
    A = through(A, wa);
  }
  V none = all<C>(0.f), unused;
  join(ex, 1, me.warp, A, H, &none, &unused);
  return none;
}

// How far the steps of a tensor are aligned: 16, 4 or fewer bytes.
inline int alignment(const void *base, int64_t seq, int64_t step, int32_t type) {
  const int64_t e = type_bytes(type);
  const int64_t any = (int64_t)(uintptr_t)base | seq * e | step * e;
  return any % 16 == 0 ? 16 : any % 4 == 0 ? 4 : 2;
}

// How a call is split: the warps of a CTA and the segments of a sequence.  An SM holds 16 warps of the kernels that
// compute the outputs and wants at least 12, better in CTAs of 4 whose phases overlap.  Where there are too few channel
// blocks for that, a CTA gets 8 or 16 warps, up to `most`; where these do not do either, the sequences are cut into
// segments, as many as make `resident` CTAs of 4 warps for every SM, whose maps a first kernel finds (it reads two of the
// streams once more).
constexpr int64_t kSms = 148, kWanted = 12 * kSms, kMaxSegs = 128;
struct Split { int warps, segs; };
inline Split split(int64_t chains, int64_t t, int most, int resident) {
  const int64_t runs = ceil_div(t, kRun);
  for (int w = 4; w <= most; w *= 2)
    if (chains * w >= kWanted && w <= std::max<int64_t>(4, runs)) return {w, 1};
  return {4, (int)std::max<int64_t>(1, std::min({resident * kSms / chains, ceil_div(runs, 4), kMaxSegs}))};
}

inline cudaError_t launch_kernel(void (*kernel)(const RecurArgs), const RecurArgs &p, int64_t b, int warps, int bytes,
                                 std::atomic<uint64_t> *done, bool after, cudaStream_t s) {
  const cudaError_t e = set_max_shared_once(reinterpret_cast<const void *>(kernel), bytes, done);
  if (e != cudaSuccess) return e;
  const unsigned grid = (unsigned)(b * p.blocks * p.segs);
  if (after) return launch_after<RecurArgs>(kernel, p, dim3(grid), 32 * warps, bytes, s);
  kernel<<<grid, 32 * warps, bytes, s>>>(p);
  return cudaGetLastError();
}

// Calls `go` with the layout, the width of the copies and the warps that suit: go.template run<L, WIDE, WARPS>.
// `in`: the alignment that all inputs have, `out`: that of the outputs.
template <typename Go, int L, bool WIDE> cudaError_t choose_split(Go &go) {
  RecurArgs &p = go.p;
  p.blocks = (int32_t)ceil_div(p.d, Lanes<L>::kChannels);
  const Split s = split(go.b * p.blocks, p.t, Go::template most<WIDE>(), Go::template resident<WIDE>());
  p.n_tiles = ceil_div(p.t, s.warps * kRun);
  p.seg_tiles = ceil_div(p.n_tiles, s.segs);
  p.segs = (int32_t)ceil_div(p.n_tiles, p.seg_tiles);
  p.maps_h = p.maps_a + go.b * (p.segs + 1) * p.d;
  if (p.segs > 1) {
    const cudaError_t e = go.template maps<L, WIDE>();
    if (e != cudaSuccess) return e;
  }
  if constexpr (Go::template most<WIDE>() >= 16)
    if (s.warps == 16) return go.template run<L, WIDE, 16>();
  if constexpr (Go::template most<WIDE>() >= 8)
    if (s.warps == 8) return go.template run<L, WIDE, 8>();
  return go.template run<L, WIDE, 4>();
}
template <typename Go> ceca_status_t choose(Go go, int in, int out, int32_t type) {
  cudaError_t e;
  if (type == DSGD_F32) e = in == 16 ? choose_split<Go, F32, true>(go) : choose_split<Go, F32, false>(go);
  else if (go.p.d % 2 == 0 && in >= 4 && out >= 4) e = in == 16 ? choose_split<Go, PAIRS, true>(go) : choose_split<Go, PAIRS, false>(go);
  else e = choose_split<Go, HALVES, false>(go);
  return e == cudaSuccess ? CECA_OK : CECA_ERR_CUDA;
}

// Enough for every layout: the widest channel blocks and the fewest warps make the most segments.
inline size_t maps_bytes(int64_t b, int64_t t, int64_t d) {
  const int segs = split(b * ceil_div(d, 64), t, 4, 4).segs;
  return segs == 1 ? 0 : sizeof(float) * 2 * (size_t)b * (size_t)(segs + 1) * (size_t)d;
}

// The map of each segment.  A warp takes a quarter of it step by step; REVERSE: for c_s = keep_s (dh_s + c_{s+1}) from the end,
// with dh in x's place.  Entry 0 (of the maps in the direction of the recurrence) is what reaches the first segment.
template <int L, bool WIDE> struct MapShared {
  static constexpr int kStages = WIDE ? 3 : 2;   // so that four CTAs fit on an SM
  Run<L, WIDE> runs[4][kStages][2];
  Exchange<L, 4> ex;
};
template <int L, bool WIDE, bool REVERSE> __global__ void __launch_bounds__(128, 4) recurrence_map_kernel(const RecurArgs p) {
  using T = typename Lanes<L>::T;
  constexpr int C = Lanes<L>::kVals;
  using V = Val<C>;
  using Sh = MapShared<L, WIDE>;
  constexpr int kStages = Sh::kStages;
  static_assert(sizeof(Sh) <= kMaxShared);
  extern __shared__ __align__(16) char memory[];
  Sh &sh = *reinterpret_cast<Sh *>(memory);
  follow_early();
  const Place<L> me(p);
  const int64_t x_step = REVERSE ? p.dh_step : p.x_step;
  const T *x = (REVERSE ? static_cast<const T *>(p.dh) + me.i * p.dh_seq : static_cast<const T *>(p.x) + me.i * p.x_seq) + me.first;
  const T *f = static_cast<const T *>(p.f) + me.i * p.f_seq + me.first;
  const uint8_t *starts = p.starts ? p.starts + me.i * p.t : nullptr;
  auto &mine = sh.runs[me.warp];
  const int64_t runs = p.seg_tiles;   // of each warp
  const int64_t first = (me.seg * p.seg_tiles * 4 + me.warp * runs) * kRun;
  auto where = [&](int64_t k) { return first + (REVERSE ? runs - 1 - k : k) * kRun; };
  auto fetch = [&](int stage, int64_t k) {
    if (k < runs) {
      mine[stage][0].fetch(x, x_step, where(k), p.t, me.width);
      mine[stage][1].fetch(f, p.f_step, where(k), p.t, me.width);
    }
    copies_end();
  };
  auto begins = [&](int64_t k) {
    return starts && k < runs && me.lane < kRun && where(k) + me.lane < p.t ? (int)starts[where(k) + me.lane] : 0;
  };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) fetch(k, k);
  int begin = begins(0), stage = 0;
  bool cut = false;   // whether a document begins in what the warp has seen
  V A = all<C>(1.f), H = all<C>(0.f);
  for (int64_t k = 0; k < runs; ++k) {
    int ahead = stage + kStages - 1;
    ahead = ahead >= kStages ? ahead - kStages : ahead;
    __syncwarp();
    fetch(ahead, k + kStages - 1);
    const uint32_t cuts = __ballot_sync(0xffffffffu, begin != 0);
    begin = begins(k + 1);
    copies_wait<kStages - 1>();
    __syncwarp();
    const Run<L, WIDE> &xr = mine[stage][0], &fr = mine[stage][1];
    stage = stage + 1 == kStages ? 0 : stage + 1;
    const int64_t s0 = where(k);
    const int left = (int)max((int64_t)0, min((int64_t)kRun, p.t - s0));
    const Skew xk(x, x_step * sizeof(T), s0), fk(f, p.f_step * sizeof(T), s0);
    cut |= cuts != 0;
    auto step = [&](int j, bool begins_here) {
      V a, na;
      gates(take<L>(fr.at(j, fk)), &a, &na);
      const V xv = take<L>(xr.at(j, xk));
      if (REVERSE) H = begins_here ? all<C>(0.f) : mul(a, add(xv, H));
      else H = begins_here ? mul(na, xv) : fma(a, H, mul(na, xv));
      A = mul(A, a);
    };
    if (left == kRun && !cuts) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) step(REVERSE ? kRun - 1 - j : j, false);
    } else {
      for (int j = 0; j < left; ++j) {
        const int at = REVERSE ? left - 1 - j : j;
        step(at, cuts >> at & 1);
      }
    }
  }
  copies_wait<0>();
  const int order = REVERSE ? 3 - me.warp : me.warp, at = me.lane * C;
  write(&sh.ex.a[0][order][at], cut ? all<C>(kCut) : A);
  write(&sh.ex.h[0][order][at], H);
  __syncthreads();
  if (me.warp > 0) return;
  A = all<C>(1.f);
  H = all<C>(0.f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const V wa = read(&sh.ex.a[0][w][at], A);
    H = follow(wa, read(&sh.ex.h[0][w][at], A), H);
    A = through(A, wa);
  }
  const int entry = REVERSE ? p.segs - 1 - me.seg : me.seg;
  store<L>(p.maps_a + me.map(p, entry + 1), A, me.live);
  store<L>(p.maps_h + me.map(p, entry + 1), H, me.live);
  if (entry == 0) {
    const float *from = REVERSE ? p.dh_last : p.h0;
    store<L>(p.maps_a + me.map(p, 0), all<C>(kCut), me.live);
    store<L>(p.maps_h + me.map(p, 0), from ? load<L>(from + me.i * p.d + me.c0, me.live) : all<C>(0.f), me.live);
  }
}

__global__ void __launch_bounds__(256) recurrence_empty_kernel(const float *from, float *to, int64_t count) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k < count) to[k] = from ? from[k] : 0.f;
}

inline ceca_status_t done() { return cudaGetLastError() == cudaSuccess ? CECA_OK : CECA_ERR_CUDA; }

// t = 0: the state goes through unchanged (in place it is there already).
inline ceca_status_t pass_through(const float *from, float *to, int64_t count, cudaStream_t s) {
  if (!to || to == from) return CECA_OK;
  recurrence_empty_kernel<<<(unsigned)ceil_div(count, 256), 256, 0, s>>>(from, to, count);
  return done();
}

inline bool sizes_ok(int64_t b, int64_t t, int64_t d, int32_t type) {
  constexpr int64_t big = (int64_t)1 << 31;
  return b >= 1 && b < big && d >= 1 && d < big && b * ceil_div(d, 32) < big / 256 && t >= 0 && t < big && is_type(type);
}

inline bool strides_ok(int64_t d, int64_t seq, int64_t step) { return seq >= 0 && step >= d; }

}  // namespace
}  // namespace ceca
