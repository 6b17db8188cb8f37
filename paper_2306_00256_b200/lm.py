"""ctypes binding of the language-model operators of include/ceca.h.  Argument marshalling only.

Outputs that are not passed in, and the workspace of dsgd_embed_grad, are allocated by torch on the stream
that the call runs on; everything else is as in binding.py: the current stream by default, ValueError for
tensors that do not fit, CecaError for what the library refuses."""
import contextlib

import torch

from .binding import _check, _stream, library

_TYPES = {torch.float32: 0, torch.bfloat16: 1}
_INDEX = {torch.int32: 0, torch.int64: 1}


def _on(stream):
    """The context in which torch allocates for work on `stream`."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream) or 0))
    return torch.cuda.stream(stream)


def _empty(shape, dtype, like, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _device(first, *others):
    """All tensors live on the current device: the launch goes to one of its streams."""
    _need(first.is_cuda and first.get_device() == torch.cuda.current_device(), "tensors must live in the current device's memory")
    for t in others:
        _need(t is None or t.get_device() == first.get_device(), "tensors must live in the current device's memory")


def _rows(t, name, types=_TYPES):
    """The type code of a tensor whose last dimension is contiguous."""
    code = types.get(t.dtype)
    _need(code is not None, "%s must be one of %s" % (name, ", ".join(str(k)[6:] for k in types)))
    _need(t.stride(-1) == 1 or t.shape[-1] == 1, "%s must be contiguous in its last dimension" % name)
    return code


def _step(t, dim):
    """The stride of a dimension; for one of a single entry, which torch leaves arbitrary, that of dense rows."""
    return t.stride(dim) if t.shape[dim] > 1 else max(t.stride(dim), t.shape[-1])


def _dense(t, name, shape, dtype=torch.float32):
    if t is not None:
        _need(t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous(),
              "%s must be a contiguous %s tensor of shape %s" % (name, str(dtype)[6:], tuple(shape)))


def _p(t):
    return None if t is None else t.data_ptr()


def _seq(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), 0)


def dsgd_embed_lookup(E, tokens, scale=1.0, out=None, out_dtype=None, stream=None):
    """out[i, s, :] = scale * E[i, tokens[i, s], :] for n agents' tables E [n, v, d] (float32 or bfloat16, any agent
    and row strides: a block of columns of X unflattened to [n, v, d] will do; an expanded first dimension
    is one table for all agents) and tokens [n, t] (int32 or int64).  A token outside [0, v) gives a zero row."""
    _need(E.dim() == 3 and tokens.dim() == 2 and tokens.shape[0] == E.shape[0], "E must be [n, v, d] and tokens [n, t]")
    (n, v, d), t = E.shape, tokens.shape[1]
    te, ti = _rows(E, "E"), _rows(tokens, "tokens", _INDEX)
    _device(E, tokens, out)
    if out is None:
        out = _empty((n, t, d), out_dtype or E.dtype, E, stream)
    _need(tuple(out.shape) == (n, t, d) and (out_dtype is None or out.dtype == out_dtype), "out must be [n, t, d] of out_dtype")
    to = _rows(out, "out")
    st = library().dsgd_embed_lookup(_p(E), _p(tokens), _p(out), n, t, v, d, _seq(E), _step(E, 1), tokens.stride(0),
                                     _seq(out), _step(out, 1), te, ti, to, float(scale), _stream(stream))
    _check(st, "dsgd_embed_lookup")
    return out


def dsgd_embed_workspace_bytes(n, t, v, d):
    return int(library().dsgd_embed_workspace_bytes(n, t, v, d))


def dsgd_embed_grad(dout, tokens, dE, scale=1.0, accumulate=False, workspace=None, stream=None):
    """The gradient of dsgd_embed_lookup: writes (or, with accumulate, adds) scale times the sum of dout's rows
    over each token's positions into dE [n, v, d], and returns it.  workspace: device memory of
    dsgd_embed_workspace_bytes(n, t, v, d) bytes, allocated here when it is None."""
    _need(dE.dim() == 3 and tokens.dim() == 2 and tokens.shape[0] == dE.shape[0], "dE must be [n, v, d] and tokens [n, t]")
    (n, v, d), t = dE.shape, tokens.shape[1]
    _need(tuple(dout.shape) == (n, t, d), "dout must be [n, t, d]")
    te, ti, to = _rows(dE, "dE"), _rows(tokens, "tokens", _INDEX), _rows(dout, "dout")
    _device(dE, tokens, dout, workspace)
    if workspace is None:
        workspace = _empty((dsgd_embed_workspace_bytes(n, t, v, d),), torch.uint8, dE, stream)
    st = library().dsgd_embed_grad(_p(dout), _p(tokens), _p(dE), n, t, v, d, _seq(dE), _step(dE, 1), tokens.stride(0),
                                   _seq(dout), dout.stride(1), te, ti, to, float(scale), int(bool(accumulate)),
                                   _p(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "dsgd_embed_grad")
    return dE


def dsgd_recurrence_marks(t):
    return int(library().dsgd_recurrence_marks(t))


def dsgd_recurrence_workspace_bytes(b, t, d):
    return int(library().dsgd_recurrence_workspace_bytes(b, t, d))


def _recurrence_workspace(workspace, x, stream):
    """(tensor or None, bytes): the caller's workspace, or one allocated here where the sizes need it."""
    if workspace is None:
        size = library().dsgd_recurrence_workspace_bytes(*x.shape)
        workspace = _empty((size,), torch.uint8, x, stream) if size else None
    return workspace, 0 if workspace is None else workspace.numel() * workspace.element_size()


def dsgd_recurrence(x, f, h0=None, starts=None, h=None, h_last=None, save=False, workspace=None, stream=None):
    """h[:, s] = keep * h[:, s-1] + (1 - sigmoid(f[:, s])) * x[:, s], keep = sigmoid(f[:, s]) or 0 where starts is set,
    for x, f [b, t, d] of one type (float32 or bfloat16).  h0: float32 [b, d]; starts: uint8 or bool [b, t].
    Returns (h, h_last, marks): h like x, h_last the float32 state after the last step, marks what
    dsgd_recurrence_grad starts from (None unless save).  One new token is t = 1 with h0 = h_last = the kept state.
    workspace: device memory of dsgd_recurrence_workspace_bytes(b, t, d) bytes, allocated here when it is None."""
    _need(x.dim() == 3 and f.shape == x.shape and f.dtype == x.dtype, "x and f must be [b, t, d] of one type")
    b, t, d = x.shape
    code = _rows(x, "x")
    _rows(f, "f")
    _dense(h0, "h0", (b, d))
    if starts is not None and starts.dtype == torch.bool:
        starts = starts.view(torch.uint8)
    _dense(starts, "starts", (b, t), torch.uint8)
    _device(x, f, h0, starts, h, h_last, workspace)
    if h is None:
        h = _empty((b, t, d), x.dtype, x, stream)
    _need(h.shape == x.shape and h.dtype == x.dtype, "h must have the shape and type of x")
    _rows(h, "h")
    if h_last is None:
        h_last = _empty((b, d), torch.float32, x, stream)
    _dense(h_last, "h_last", (b, d))
    marks = _empty((b, dsgd_recurrence_marks(t), d), torch.float32, x, stream) if save else None
    workspace, size = _recurrence_workspace(workspace, x, stream)
    st = library().dsgd_recurrence(_p(x), _p(f), _p(h0), _p(starts), _p(h), _p(h_last), _p(marks), b, t, d,
                                   _seq(x), _step(x, 1), _seq(f), _step(f, 1), _seq(h), _step(h, 1), code,
                                   _p(workspace), size, _stream(stream))
    _check(st, "dsgd_recurrence")
    return h, h_last, marks


def dsgd_recurrence_grad(x, f, dh, marks, h0=None, starts=None, dh_last=None, dx=None, df=None, dh0=None, workspace=None, stream=None):
    """The gradient of dsgd_recurrence at the same x, f, h0, starts, from the marks that it saved: returns
    (dx, df, dh0), dh0 float32 [b, d] with respect to the initial state, given or zero (h0 itself lies in the marks)."""
    _need(x.dim() == 3 and f.shape == x.shape == dh.shape and f.dtype == x.dtype == dh.dtype, "x, f and dh must be [b, t, d] of one type")
    b, t, d = x.shape
    code = _rows(x, "x")
    _rows(f, "f")
    _rows(dh, "dh")
    _dense(marks, "marks", (b, dsgd_recurrence_marks(t), d))
    _dense(dh_last, "dh_last", (b, d))
    if starts is not None and starts.dtype == torch.bool:
        starts = starts.view(torch.uint8)
    _dense(starts, "starts", (b, t), torch.uint8)
    _device(x, f, dh, marks, starts, dh_last, dx, df, dh0, workspace)
    dx = _empty((b, t, d), x.dtype, x, stream) if dx is None else dx
    df = _empty((b, t, d), x.dtype, x, stream) if df is None else df
    dh0 = _empty((b, d), torch.float32, x, stream) if dh0 is None else dh0
    _dense(h0, "h0", (b, d))
    _dense(dh0, "dh0", (b, d))
    for g, name in ((dx, "dx"), (df, "df")):
        _need(g.shape == x.shape and g.dtype == x.dtype, "%s must have the shape and type of x" % name)
        _rows(g, name)
    workspace, size = _recurrence_workspace(workspace, x, stream)
    st = library().dsgd_recurrence_grad(_p(x), _p(f), _p(dh), _p(marks), _p(starts), _p(dh_last), _p(dx), _p(df), _p(dh0),
                                        b, t, d, _seq(x), _step(x, 1), _seq(f), _step(f, 1), _seq(dh), _step(dh, 1),
                                        _seq(dx), _step(dx, 1), _seq(df), _step(df, 1), code, _p(workspace),
                                        size, _stream(stream))
    _check(st, "dsgd_recurrence_grad")
    return dx, df, dh0


def _distill_args(z, idx, t, teacher_lse, weight, loss, stream):
    _need(z.dim() == 2 and idx.dim() == 2 and idx.shape == t.shape and idx.shape[0] == z.shape[0],
          "z must be [r, v], idx and t [r, k]")
    r, v = z.shape
    codes = _rows(z, "z"), _rows(idx, "idx", _INDEX), _rows(t, "t")
    _dense(teacher_lse, "teacher_lse", (r,))
    _dense(weight, "weight", (r,))
    _device(z, idx, t, teacher_lse, weight, loss)
    if loss is None:
        loss = _empty((r,), torch.float32, z, stream)
    _dense(loss, "loss", (r,))
    return r, v, idx.shape[1], codes, loss


def dsgd_distill_loss(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, stream=None):
    """weight * KL(teacher || softmax(z / temperature)) of each row of z [r, v], the teacher being known by its top
    logits t [r, k] at the vocabulary entries idx [r, k] (an idx outside [0, v): fewer entries).  Without teacher_lse
    it is renormalised over them; with it, the mass it leaves is compared with the student's outside the top."""
    r, v, k, (tz, ti, tt), loss = _distill_args(z, idx, t, teacher_lse, weight, loss, stream)
    st = library().dsgd_distill_loss(_p(z), _p(idx), _p(t), _p(teacher_lse), _p(weight), _p(loss), r, v, k, _step(z, 0),
                                     _step(idx, 0), _step(t, 0), tz, ti, tt, float(temperature), _stream(stream))
    _check(st, "dsgd_distill_loss")
    return loss


def dsgd_distill_grad(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, dz=None, stream=None):
    """(loss, dz): dsgd_distill_loss and the gradient of its sum over rows with respect to z, in one pass.  dz may be z."""
    r, v, k, (tz, ti, tt), loss = _distill_args(z, idx, t, teacher_lse, weight, loss, stream)
    dz = _empty((r, v), z.dtype, z, stream) if dz is None else dz
    _need(dz.shape == z.shape and dz.dtype == z.dtype and dz.get_device() == z.get_device(), "dz must have the shape, type and device of z")
    _rows(dz, "dz")
    st = library().dsgd_distill_grad(_p(z), _p(idx), _p(t), _p(teacher_lse), _p(weight), _p(loss), _p(dz), r, v, k,
                                     _step(z, 0), _step(idx, 0), _step(t, 0), _step(dz, 0), tz, ti, tt, float(temperature),
                                     _stream(stream))
    _check(st, "dsgd_distill_grad")
    return loss, dz
