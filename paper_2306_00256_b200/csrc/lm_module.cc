// Python module of the language-model operators: argument marshalling only, in C++ because a decoding step calls
// them for a few microseconds of work.  lm.py documents the functions.  Outputs that are not passed in, and
// workspaces, are allocated by torch on the stream that the call runs on.
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

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

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("embed_lookup", &embed_lookup);
  m.def("embed_grad", &embed_grad);
  m.def("recurrence", &recurrence);
  m.def("recurrence_grad", &recurrence_grad);
  m.def("distill", &distill);
}
