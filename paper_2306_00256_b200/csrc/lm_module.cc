// Python module of the language-model operators: argument marshalling only, in C++ because a decoding step calls
// them for a few microseconds of work.  lm.py documents the functions.  Outputs that are not passed in, and
// workspaces, are allocated by torch on the stream that the call runs on.
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

#include <algorithm>
#include <optional>
#include <string>

#include "ceca.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

namespace {

void need(bool ok, const char *text) {
  if (!ok) throw py::value_error(text);
}

void check(ceca_status_t status, const char *where) {
  if (status == CECA_OK) return;
  const py::object error = py::module_::import("paper_2306_00256_b200.binding").attr("CecaError");
  PyErr_SetObject(error.ptr(), error((int)status, where).ptr());
  throw py::error_already_set();
}

// The type code and strides of a tensor whose last dimension is contiguous.  The stride of a dimension of one entry,
// which torch leaves arbitrary, is that of dense rows.
struct Rows {
  int32_t type;
  int64_t seq, step;
};
Rows rows(const Tensor &t, const char *name, bool index = false) {
  const auto type = t.scalar_type();
  const bool first = type == (index ? at::kInt : at::kFloat), second = type == (index ? at::kLong : at::kBFloat16);
  if (!first && !second) throw py::value_error(std::string(name) + (index ? " must be one of int32, int64" : " must be one of float32, bfloat16"));
  const int64_t dims = t.dim(), last = t.size(dims - 1);
  if (t.stride(dims - 1) != 1 && last > 1) throw py::value_error(std::string(name) + " must be contiguous in its last dimension");
  int64_t step = t.stride(dims - 2);
  if (t.size(dims - 2) <= 1 && step < last) step = last;
  return {second ? 1 : 0, dims > 2 ? t.stride(0) : step, step};
}

// fp32 (or bytes), contiguous, of the given shape
template <typename T = float> T *dense(const Tensor &t, const char *name, at::IntArrayRef shape, at::ScalarType type = at::kFloat) {
  if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
    throw py::value_error(std::string(name) + " must be a contiguous " + (type == at::kFloat ? "float32" : "uint8") + " tensor of the right shape");
  return static_cast<T *>(t.data_ptr());
}
template <typename T = float> T *dense(const Maybe &t, const char *name, at::IntArrayRef shape, at::ScalarType type = at::kFloat) {
  return t ? dense<T>(*t, name, shape, type) : nullptr;
}
const uint8_t *starts_of(const Maybe &t, at::IntArrayRef shape) {
  return t ? dense<uint8_t>(t->scalar_type() == at::kBool ? t->view(at::kByte) : *t, "starts", shape, at::kByte) : nullptr;
}

// Where the call runs: all tensors on the current device, and the stream, which torch allocates for as well.
struct Here {
  void *stream = nullptr;
  std::optional<c10::cuda::CUDAStreamGuard> guard;
  Here(const py::object &given, const Tensor &first) {
    need(first.is_cuda() && first.get_device() == c10::cuda::current_device(), "tensors must live in the current device's memory");
    if (given.is_none()) {
      stream = c10::cuda::getCurrentCUDAStream().stream();
      return;
    }
    const py::object raw = py::hasattr(given, "cuda_stream") ? given.attr("cuda_stream").cast<py::object>() : given;
    stream = reinterpret_cast<void *>(raw.cast<uintptr_t>());
    guard.emplace(stream ? c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), first.get_device())
                         : c10::cuda::getDefaultCUDAStream());
  }
  void also(const Tensor &first, const Tensor &t) const {
    need(t.is_cuda() && t.get_device() == first.get_device(), "tensors must live in the current device's memory");
  }
  void also(const Tensor &first, const Maybe &t) const {
    if (t) also(first, *t);
  }
};

Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor &like) { return at::empty(shape, like.options().dtype(type)); }

// The caller's workspace, or one allocated here where the sizes need it.
struct Workspace {
  Tensor held;
  void *at = nullptr;
  size_t bytes = 0;
  Workspace(const Maybe &given, size_t wanted, const Tensor &like) {
    if (given) {
      held = *given;
      need(held.is_contiguous(), "workspace must be contiguous");   // all memory from its first byte to its last is written
      bytes = (size_t)held.numel() * held.element_size();
    } else if (wanted) {
      held = empty({(int64_t)wanted}, at::kByte, like);
      bytes = wanted;
    } else {
      return;
    }
    at = held.data_ptr();
  }
};

Tensor embed_lookup(const Tensor &E, const Tensor &tokens, double scale, const Maybe &out, std::optional<at::ScalarType> out_dtype,
                    const py::object &stream) {
  need(E.dim() == 3 && tokens.dim() == 2 && tokens.size(0) == E.size(0), "E must be [n, v, d] and tokens [n, t]");
  const int64_t n = E.size(0), v = E.size(1), d = E.size(2), t = tokens.size(1);
  const Rows e = rows(E, "E"), w = rows(tokens, "tokens", true);
  const Here here(stream, E);
  here.also(E, tokens);
  here.also(E, out);
  need(!out || (out->sizes() == at::IntArrayRef({n, t, d}) && (!out_dtype || out->scalar_type() == *out_dtype)), "out must be [n, t, d] of out_dtype");
  const Tensor to = out ? *out : empty({n, t, d}, out_dtype.value_or(E.scalar_type()), E);
  const Rows o = rows(to, "out");
  check(dsgd_embed_lookup(E.data_ptr(), tokens.data_ptr(), to.data_ptr(), (int32_t)n, t, v, d, e.seq, e.step, w.step, o.seq, o.step,
                          e.type, w.type, o.type, (float)scale, here.stream),
        "dsgd_embed_lookup");
  return to;
}

Tensor embed_grad(const Tensor &dout, const Tensor &tokens, const Tensor &dE, double scale, bool accumulate, const Maybe &workspace,
                  const py::object &stream) {
  need(dE.dim() == 3 && tokens.dim() == 2 && tokens.size(0) == dE.size(0), "dE must be [n, v, d] and tokens [n, t]");
  const int64_t n = dE.size(0), v = dE.size(1), d = dE.size(2), t = tokens.size(1);
  need(dout.sizes() == at::IntArrayRef({n, t, d}), "dout must be [n, t, d]");
  const Rows e = rows(dE, "dE"), w = rows(tokens, "tokens", true), o = rows(dout, "dout");
  const Here here(stream, dE);
  here.also(dE, tokens);
  here.also(dE, dout);
  here.also(dE, workspace);
  const Workspace ws(workspace, dsgd_embed_workspace_bytes((int32_t)n, t, v, d), dE);
  check(dsgd_embed_grad(dout.data_ptr(), tokens.data_ptr(), dE.data_ptr(), (int32_t)n, t, v, d, e.seq, e.step, w.step, o.seq,
                        dout.stride(1), e.type, w.type, o.type, (float)scale, accumulate, ws.at, ws.bytes, here.stream),
        "dsgd_embed_grad");
  return dE;
}

py::tuple recurrence(const Tensor &x, const Tensor &f, const Maybe &h0, const Maybe &starts, const Maybe &h, const Maybe &h_last,
                     bool save, const Maybe &workspace, const py::object &stream) {
  need(x.dim() == 3 && f.sizes() == x.sizes() && f.scalar_type() == x.scalar_type(), "x and f must be [b, t, d] of one type");
  const int64_t b = x.size(0), t = x.size(1), d = x.size(2);
  const Rows rx = rows(x, "x"), rf = rows(f, "f");
  const Here here(stream, x);
  for (const Maybe *m : {&h0, &starts, &h, &h_last, &workspace}) here.also(x, *m);
  here.also(x, f);
  const float *p0 = dense(h0, "h0", {b, d});
  const uint8_t *ps = starts_of(starts, {b, t});
  need(!h || (h->sizes() == x.sizes() && h->scalar_type() == x.scalar_type()), "h must have the shape and type of x");
  const Tensor ho = h ? *h : empty({b, t, d}, x.scalar_type(), x), last = h_last ? *h_last : empty({b, d}, at::kFloat, x);
  const Rows rh = rows(ho, "h");
  float *pl = dense(last, "h_last", {b, d});
  Maybe marks;
  if (save) marks = empty({b, dsgd_recurrence_marks(t), d}, at::kFloat, x);
  const Workspace ws(workspace, dsgd_recurrence_workspace_bytes(b, t, d), x);
  check(dsgd_recurrence(x.data_ptr(), f.data_ptr(), p0, ps, ho.data_ptr(), pl, save ? static_cast<float *>(marks->data_ptr()) : nullptr, b, t, d,
                        rx.seq, rx.step, rf.seq, rf.step, rh.seq, rh.step, rx.type, ws.at, ws.bytes, here.stream),
        "dsgd_recurrence");
  return py::make_tuple(ho, last, marks);
}

py::tuple recurrence_grad(const Tensor &x, const Tensor &f, const Tensor &dh, const Tensor &marks, const Maybe &h0, const Maybe &starts,
                          const Maybe &dh_last, const Maybe &dx, const Maybe &df, const Maybe &dh0, const Maybe &workspace,
                          const py::object &stream) {
  need(x.dim() == 3 && f.sizes() == x.sizes() && dh.sizes() == x.sizes() && f.scalar_type() == x.scalar_type() &&
           dh.scalar_type() == x.scalar_type(),
       "x, f and dh must be [b, t, d] of one type");
  const int64_t b = x.size(0), t = x.size(1), d = x.size(2);
  const Rows rx = rows(x, "x"), rf = rows(f, "f"), rg = rows(dh, "dh");
  const Here here(stream, x);
  for (const Maybe *m : {&starts, &dh_last, &dx, &df, &dh0, &workspace}) here.also(x, *m);
  for (const Tensor *m : {&f, &dh, &marks}) here.also(x, *m);
  const float *pm = dense(marks, "marks", {b, dsgd_recurrence_marks(t), d});
  const uint8_t *ps = starts_of(starts, {b, t});
  const float *pl = dense(dh_last, "dh_last", {b, d});
  dense(h0, "h0", {b, d});
  for (const Maybe *m : {&dx, &df})
    need(!*m || ((*m)->sizes() == x.sizes() && (*m)->scalar_type() == x.scalar_type()), "dx and df must have the shape and type of x");
  const Tensor ox = dx ? *dx : empty({b, t, d}, x.scalar_type(), x), of = df ? *df : empty({b, t, d}, x.scalar_type(), x);
  const Tensor o0 = dh0 ? *dh0 : empty({b, d}, at::kFloat, x);
  const Rows rdx = rows(ox, "dx"), rdf = rows(of, "df");
  float *p0 = dense(o0, "dh0", {b, d});
  const Workspace ws(workspace, dsgd_recurrence_workspace_bytes(b, t, d), x);
  check(dsgd_recurrence_grad(x.data_ptr(), f.data_ptr(), dh.data_ptr(), pm, ps, pl, ox.data_ptr(), of.data_ptr(), p0, b, t, d, rx.seq,
                             rx.step, rf.seq, rf.step, rg.seq, rg.step, rdx.seq, rdx.step, rdf.seq, rdf.step, rx.type, ws.at, ws.bytes,
                             here.stream),
        "dsgd_recurrence_grad");
  return py::make_tuple(ox, of, o0);
}

// The loss alone, or with `grad` the pair of it and dz.
py::object distill(const Tensor &z, const Tensor &idx, const Tensor &t, const Maybe &teacher_lse, const Maybe &weight, double temperature,
                   const Maybe &loss, bool grad, const Maybe &dz, const py::object &stream) {
  need(z.dim() == 2 && idx.dim() == 2 && t.sizes() == idx.sizes() && idx.size(0) == z.size(0), "z must be [r, v], idx and t [r, k]");
  const int64_t r = z.size(0), v = z.size(1), k = idx.size(1);
  const Rows rz = rows(z, "z"), ri = rows(idx, "idx", true), rt = rows(t, "t");
  const Here here(stream, z);
  here.also(z, idx);
  here.also(z, t);
  for (const Maybe *m : {&teacher_lse, &weight, &loss, &dz}) here.also(z, *m);
  const float *pe = dense(teacher_lse, "teacher_lse", {r}), *pw = dense(weight, "weight", {r});
  const Tensor lo = loss ? *loss : empty({r}, at::kFloat, z);
  float *pl = dense(lo, "loss", {r});
  if (!grad) {
    check(dsgd_distill_loss(z.data_ptr(), idx.data_ptr(), t.data_ptr(), pe, pw, pl, r, v, k, rz.step, ri.step, rt.step, rz.type, ri.type, rt.type,
                            (float)temperature, here.stream),
          "dsgd_distill_loss");
    return py::cast(lo);
  }
  need(!dz || (dz->sizes() == z.sizes() && dz->scalar_type() == z.scalar_type()), "dz must have the shape and type of z");
  const Tensor g = dz ? *dz : empty({r, v}, z.scalar_type(), z);
  const Rows rg = rows(g, "dz");
  check(dsgd_distill_grad(z.data_ptr(), idx.data_ptr(), t.data_ptr(), pe, pw, pl, g.data_ptr(), r, v, k, rz.step, ri.step, rt.step, rg.step, rz.type,
                          ri.type, rt.type, (float)temperature, here.stream),
        "dsgd_distill_grad");
  return py::make_tuple(lo, g);
}

// An n x t x d tensor of one of the two types, or nothing.
struct Block {
  dsgd_rows_t at{};
  int32_t type = -1;
  Block() = default;
  Block(const Tensor &t, const char *name, at::IntArrayRef shape, int32_t as = -1) {
    if (t.sizes() != shape) throw py::value_error(std::string(name) + " must be [n, t, d]");
    const Rows r = rows(t, name);
    if (as >= 0 && r.type != as) throw py::value_error(std::string(name) + " has another type than it must have");
    at = {t.data_ptr(), r.seq, r.step};
    type = r.type;
  }
  Block(const Maybe &t, const char *name, at::IntArrayRef shape, int32_t as = -1) {
    if (t) *this = Block(*t, name, shape, as);
  }
};
at::ScalarType scalar_of(int32_t type) { return type ? at::kBFloat16 : at::kFloat; }

// Each agent's d weights (or its one, for d = 0), any stride between agents.
struct Weights {
  void *at = nullptr;
  int64_t stride = 0;
  Weights(const Maybe &t, const char *name, int64_t n, int64_t d, int32_t &type) {
    if (!t) return;
    const int32_t mine = t->scalar_type() == at::kBFloat16 ? 1 : 0;
    if (t->dim() != (d ? 2 : 1) || t->size(0) != n || (d && (t->size(1) != d || (d > 1 && t->stride(1) != 1))) ||
        (!mine && t->scalar_type() != at::kFloat) || (type >= 0 && type != mine))
      throw py::value_error(std::string(name) + " must be " + (d ? "[n, d], contiguous in d," : "[n]") + " in float32 or bfloat16, one type for all weights");
    type = mine;
    at = t->data_ptr();
    stride = n > 1 ? t->stride(0) : std::max<int64_t>(d, 1);
  }
};

Tensor kept_like(const Tensor &x) { return empty({x.size(0), x.size(1), dsgd_kept_row_bytes(x.size(2))}, at::kByte, x); }
// The rows of a kept tensor, n x t x bytes.
void *kept_of(const Tensor &t, const char *name, int64_t n, int64_t rows, int64_t d) {
  return dense<uint8_t>(t, name, {n, rows, dsgd_kept_row_bytes(d)}, at::kByte);
}

Tensor keep8(const Tensor &x, const Maybe &kept, const py::object &stream) {
  need(x.dim() == 3 && x.size(2) > 0, "x must be [n, t, d]");
  const Block b(x, "x", x.sizes());
  const Here here(stream, x);
  here.also(x, kept);
  const Tensor to = kept ? *kept : kept_like(x);
  check(dsgd_keep8(b.at, kept_of(to, "kept", x.size(0), x.size(1), x.size(2)), (int32_t)x.size(0), x.size(1), x.size(2), b.type, here.stream), "dsgd_keep8");
  return to;
}

Tensor bring8(const Tensor &kept, int64_t d, std::optional<at::ScalarType> dtype, const Maybe &x, const py::object &stream) {
  need(kept.dim() == 3 && d > 0, "kept must be [n, t, bytes], d at least 1");
  const int64_t n = kept.size(0), t = kept.size(1);
  const void *from = kept_of(kept, "kept", n, t, d);
  const Here here(stream, kept);
  here.also(kept, x);
  need(!x || !dtype || x->scalar_type() == *dtype, "x must be of dtype");
  const Tensor to = x ? *x : empty({n, t, d}, dtype.value_or(at::kFloat), kept);
  const Block b(to, "x", {n, t, d});
  check(dsgd_bring8(from, b.at, (int32_t)n, t, d, b.type, here.stream), "dsgd_bring8");
  return to;
}

py::tuple block_norm(const Tensor &h, const Maybe &y, const Maybe &w_pre, const Maybe &w_post, const Maybe &gate, int gate_act, const Maybe &scale,
                     double eps, const Maybe &h_out, const Maybe &u, bool save, bool keep, const py::object &stream) {
  need(h.dim() == 3, "h must be [n, t, d]");
  need(y || w_pre, "there must be y or w_pre");
  need(!y == !w_post && (!gate || y) && (!h_out || y) && (!u || w_pre), "y and w_post come together, a gate and h_out with y, u with w_pre");
  const int64_t n = h.size(0), t = h.size(1), d = h.size(2);
  const at::IntArrayRef shape = h.sizes();
  const Here here(stream, h);
  for (const Maybe *m : {&y, &w_pre, &w_post, &gate, &scale, &h_out, &u}) here.also(h, *m);
  const Block bh(h, "h", shape), by(y, "y", shape), bg(gate, "gate", shape, by.type);
  int32_t wt = -1;
  const Weights pre(w_pre, "w_pre", n, d, wt), post(w_post, "w_post", n, d, wt), sc(scale, "scale", n, 0, wt);
  Maybe ho = h_out, uo = u;
  if (y && !ho) ho = empty(shape, h.scalar_type(), h);
  int32_t act = by.type;
  if (act < 0) act = u ? (u->scalar_type() == at::kBFloat16 ? 1 : 0) : bh.type;
  if (w_pre && !uo) uo = empty(shape, scalar_of(act), h);
  const Block bo(ho, "h_out", shape, bh.type), bu(uo, "u", shape, act);
  Maybe stats, h8, y8, g8;
  if (save) stats = empty({n, t, 2}, at::kFloat, h);
  if (keep) {
    h8 = kept_like(h);
    if (y) y8 = kept_like(h);
    if (gate) g8 = kept_like(h);
  }
  const auto ptr = [](const Maybe &m) { return m ? m->data_ptr() : nullptr; };
  check(dsgd_block_norm(bh.at, by.at, bg.at, pre.at, post.at, sc.at, pre.stride, post.stride, sc.stride, bo.at, bu.at, static_cast<float *>(ptr(stats)),
                        ptr(h8), ptr(y8), ptr(g8), (int32_t)n, t, d, bh.type, act, wt, gate_act, (float)eps, here.stream),
        "dsgd_block_norm");
  return py::make_tuple(y ? ho : Maybe(h), uo, stats, keep ? py::object(py::make_tuple(h8, y8, g8)) : py::object(py::none()));
}

py::tuple block_norm_grad(const Tensor &h, const Maybe &y, const Maybe &w_pre, const Maybe &w_post, const Tensor &stats, const Maybe &du,
                          const Maybe &dh_out, const Maybe &gate, int gate_act, const Maybe &scale, const Maybe &dh, const Maybe &dy,
                          const Maybe &dgate, const Maybe &dw_pre, const Maybe &dw_post, const Maybe &dscale, bool accumulate, const Maybe &workspace,
                          const py::object &stream) {
  need(h.dim() == 3, "h must be [n, t, d]");
  need((y || w_pre) && !y == !w_post && (!gate || y) && !du == !w_pre && (du || dh_out),
       "y and w_post come together, a gate with y, du with w_pre; there must be y or w_pre, and du or dh_out");
  const int64_t n = h.size(0), t = h.size(1);
  const bool kept = h.scalar_type() == at::kByte;
  const Tensor &g = du ? *du : *dh_out;
  const at::IntArrayRef shape = g.sizes();
  need(g.dim() == 3 && shape[0] == n && shape[1] == t, "du and dh_out must be [n, t, d]");
  const int64_t d = shape[2];
  const Here here(stream, h);
  for (const Maybe *m : {&y, &w_pre, &w_post, &du, &dh_out, &gate, &scale, &dh, &dy, &dgate, &dw_pre, &dw_post, &dscale, &workspace}) here.also(h, *m);
  here.also(h, stats);
  const auto type_of = [](const Tensor &x) { return x.scalar_type() == at::kBFloat16 ? 1 : 0; };
  // the types of the stream and of the activations, from whatever there is of each
  const int32_t stream_type = !kept ? type_of(h) : dh_out ? type_of(*dh_out) : dh ? type_of(*dh) : type_of(*du);
  const int32_t act = du ? type_of(*du) : !kept && y ? type_of(*y) : dy ? type_of(*dy) : stream_type;
  Block bh, by, bg;
  if (kept) {
    bh.at.at = kept_of(h, "h", n, t, d);
    if (y) by.at.at = kept_of(*y, "y", n, t, d);
    if (gate) bg.at.at = kept_of(*gate, "gate", n, t, d);
  } else {
    bh = Block(h, "h", shape, stream_type);
    by = Block(y, "y", shape, act);
    bg = Block(gate, "gate", shape, act);
  }
  const Block bu(du, "du", shape, act), bo(dh_out, "dh_out", shape, stream_type);
  const auto strides = [](const Maybe &m, const Block &b) {   // 0 where the gradient is one row for all
    return m ? dsgd_rows_t{b.at.at, m->stride(0), m->stride(1)} : b.at;
  };
  int32_t wt = -1;
  const Weights pre(w_pre, "w_pre", n, d, wt), post(w_post, "w_post", n, d, wt), sc(scale, "scale", n, 0, wt);
  const auto ours = [&](const Maybe &given, bool wanted, at::IntArrayRef size, int32_t type) {
    return given ? given : wanted ? Maybe(empty(size, scalar_of(type), h)) : Maybe();
  };
  need((!dy || y) && (!dgate || gate) && (!dw_pre || w_pre) && (!dw_post || y) && (!dscale || scale), "a gradient of what is not there");
  need(!accumulate || ((!w_pre || dw_pre) && (!y || dw_post) && (!scale || !y || dscale)), "accumulate needs the gradients that are added to");
  const Maybe odh = ours(dh, true, shape, stream_type), ody = ours(dy, y.has_value(), shape, act), oda = ours(dgate, gate.has_value(), shape, act);
  const Maybe opre = ours(dw_pre, w_pre.has_value(), {n, d}, wt), opost = ours(dw_post, y.has_value(), {n, d}, wt),
              osc = ours(dscale, scale.has_value() && y.has_value(), {n}, wt);
  const Block rdh(odh, "dh", shape, stream_type), rdy(ody, "dy", shape, act), rda(oda, "dgate", shape, act);
  const Weights gpre(opre, "dw_pre", n, d, wt), gpost(opost, "dw_post", n, d, wt), gsc(osc, "dscale", n, 0, wt);
  const float *ps = dense(stats, "stats", {n, t, 2});
  const Workspace ws(workspace, dsgd_block_norm_workspace_bytes((int32_t)n, t, d), h);
  check(dsgd_block_norm_grad(bh.at, by.at, bg.at, kept, pre.at, post.at, sc.at, pre.stride, post.stride, sc.stride, ps, strides(du, bu),
                             strides(dh_out, bo), rdh.at, rdy.at, rda.at, gpre.at, gpost.at, gsc.at, gpre.stride, gpost.stride, gsc.stride, accumulate,
                             (int32_t)n, t, d, stream_type, act, wt, gate_act, ws.at, ws.bytes, here.stream),
        "dsgd_block_norm_grad");
  return py::make_tuple(odh, ody, oda, opre, opost, osc);
}

// One index a row, contiguous.
int32_t tokens_of(const Tensor &t, const char *name, int64_t count) {
  const bool wide = t.scalar_type() == at::kLong;
  if ((!wide && t.scalar_type() != at::kInt) || t.dim() != 1 || t.size(0) != count || !t.is_contiguous())
    throw py::value_error(std::string(name) + " must be a contiguous int32 or int64 tensor of the right size");
  return wide ? 1 : 0;
}

Tensor token_logprob(const Tensor &z, const Tensor &tokens, double temperature, const Maybe &logp, const Maybe &workspace, const py::object &stream) {
  need(z.dim() == 2, "z must be [r, v]");
  const int64_t r = z.size(0), v = z.size(1);
  const Rows rz = rows(z, "z");
  const int32_t ti = tokens_of(tokens, "tokens", r);
  const Here here(stream, z);
  here.also(z, tokens);
  for (const Maybe *m : {&logp, &workspace}) here.also(z, *m);
  const Tensor lo = logp ? *logp : empty({r}, at::kFloat, z);
  const Workspace ws(workspace, dsgd_token_workspace_bytes(r, v, 0), z);
  check(dsgd_token_logprob(z.data_ptr(), tokens.data_ptr(), dense(lo, "logp", {r}), r, v, rz.step, rz.type, ti, (float)temperature, ws.at, ws.bytes,
                           here.stream),
        "dsgd_token_logprob");
  return lo;
}

struct Turned {   // dz, given or like z
  Maybe dz;
  int64_t row = 0;
  void *at = nullptr;
  Turned(const Tensor &z, bool grad, const Maybe &given) {
    if (!grad) return;
    need(!given || (given->sizes() == z.sizes() && given->scalar_type() == z.scalar_type()), "dz must have the shape and type of z");
    dz = given ? *given : empty(z.sizes(), z.scalar_type(), z);
    row = rows(*dz, "dz").step;
    at = dz->data_ptr();
  }
};

// The loss alone, or with `grad` the pair of it and dz.
py::object policy(const Tensor &z, const Tensor &tokens, const Tensor &old_logp, const Tensor &advantage, const Maybe &ref_logp, const Maybe &weight,
                  double temperature, double clip_low, double clip_high, double kl, const Maybe &loss, const Maybe &logp, bool grad, const Maybe &dz,
                  const Maybe &workspace, const py::object &stream) {
  need(z.dim() == 2, "z must be [r, v]");
  const int64_t r = z.size(0), v = z.size(1);
  const Rows rz = rows(z, "z");
  const int32_t ti = tokens_of(tokens, "tokens", r);
  const Here here(stream, z);
  for (const Tensor *m : {&tokens, &old_logp, &advantage}) here.also(z, *m);
  for (const Maybe *m : {&ref_logp, &weight, &loss, &logp, &dz, &workspace}) here.also(z, *m);
  const float *po = dense(old_logp, "old_logp", {r}), *pa = dense(advantage, "advantage", {r}), *pr = dense(ref_logp, "ref_logp", {r}),
              *pw = dense(weight, "weight", {r});
  const Tensor lo = loss ? *loss : empty({r}, at::kFloat, z);
  float *pl = dense(lo, "loss", {r}), *pp = dense(logp, "logp", {r});
  const Turned g(z, grad, dz);
  const Workspace ws(workspace, dsgd_token_workspace_bytes(r, v, 0), z);
  if (!grad) {
    check(dsgd_policy_loss(z.data_ptr(), tokens.data_ptr(), po, pa, pr, pw, pl, pp, r, v, rz.step, rz.type, ti, (float)temperature, (float)clip_low,
                           (float)clip_high, (float)kl, ws.at, ws.bytes, here.stream),
          "dsgd_policy_loss");
    return py::cast(lo);
  }
  check(dsgd_policy_grad(z.data_ptr(), tokens.data_ptr(), po, pa, pr, pw, pl, pp, g.at, r, v, rz.step, g.row, rz.type, ti, (float)temperature,
                         (float)clip_low, (float)clip_high, (float)kl, ws.at, ws.bytes, here.stream),
        "dsgd_policy_grad");
  return py::make_tuple(lo, g.dz);
}

// (loss, logp), or with `grad` (loss, logp, dz).
py::tuple preference(const Tensor &z, const Tensor &tokens, const Tensor &bounds, const Maybe &ref_logp, const Maybe &weight, double temperature,
                     double beta, double smoothing, bool average, const Maybe &loss, const Maybe &logp, bool grad, const Maybe &dz,
                     const Maybe &workspace, const py::object &stream) {
  need(z.dim() == 2 && bounds.dim() == 1 && bounds.size(0) % 2 == 1, "z must be [r, v] and bounds [2 pairs + 1]");
  const int64_t r = z.size(0), v = z.size(1), pairs = bounds.size(0) / 2;
  const Rows rz = rows(z, "z");
  const int32_t ti = tokens_of(tokens, "tokens", r), tb = tokens_of(bounds, "bounds", 2 * pairs + 1);
  const Here here(stream, z);
  here.also(z, tokens);
  here.also(z, bounds);
  for (const Maybe *m : {&ref_logp, &weight, &loss, &logp, &dz, &workspace}) here.also(z, *m);
  const float *pr = dense(ref_logp, "ref_logp", {2 * pairs}), *pw = dense(weight, "weight", {pairs});
  const Tensor lo = loss ? *loss : empty({pairs}, at::kFloat, z), lp = logp ? *logp : empty({2 * pairs}, at::kFloat, z);
  float *pl = dense(lo, "loss", {pairs}), *pp = dense(lp, "logp", {2 * pairs});
  const Turned g(z, grad, dz);
  const Workspace ws(workspace, dsgd_token_workspace_bytes(r, v, pairs), z);
  if (!grad) {
    check(dsgd_preference_loss(z.data_ptr(), tokens.data_ptr(), bounds.data_ptr(), pr, pw, pl, pp, pairs, r, v, rz.step, rz.type, ti, tb,
                               (float)temperature, (float)beta, (float)smoothing, average, ws.at, ws.bytes, here.stream),
          "dsgd_preference_loss");
    return py::make_tuple(lo, lp);
  }
  check(dsgd_preference_grad(z.data_ptr(), tokens.data_ptr(), bounds.data_ptr(), pr, pw, pl, pp, g.at, pairs, r, v, rz.step, g.row, rz.type, ti, tb,
                             (float)temperature, (float)beta, (float)smoothing, average, ws.at, ws.bytes, here.stream),
        "dsgd_preference_grad");
  return py::make_tuple(lo, lp, g.dz);
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("embed_lookup", &embed_lookup);
  m.def("embed_grad", &embed_grad);
  m.def("recurrence", &recurrence);
  m.def("recurrence_grad", &recurrence_grad);
  m.def("distill", &distill);
  m.def("keep8", &keep8);
  m.def("bring8", &bring8);
  m.def("block_norm", &block_norm);
  m.def("block_norm_grad", &block_norm_grad);
  m.def("token_logprob", &token_logprob);
  m.def("policy", &policy);
  m.def("preference", &preference);
}
