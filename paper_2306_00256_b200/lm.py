"""ctypes binding of the language-model operators of include/ceca.h.  Argument marshalling only.

Outputs that are not passed in, and workspaces, are allocated by torch on the stream that the call runs on;
everything else is as in binding.py: the current stream by default, ValueError for tensors that do not fit,
CecaError for what the library refuses.  A decoding step calls these for a few microseconds of work, so the
checks below read each property of a tensor once and build their messages only when they fail."""
import torch

from .binding import CecaError, library

_TYPES = {torch.float32: 0, torch.bfloat16: 1}
_INDEX = {torch.int32: 0, torch.int64: 1}
_F32, _U8, _BOOL = torch.float32, torch.uint8, torch.bool
_device_of_thread = torch._C._cuda_getDevice
_stream_of_device = torch._C._cuda_getCurrentRawStream


def _empty(shape, dtype, like, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream) or 0))
    with torch.cuda.stream(stream):   # torch hands memory out for one stream
        return torch.empty(shape, dtype=dtype, device=like.device)


def _like(t, dtype, stream):
    """An uninitialised dense tensor of t's shape; the short way where t says it all."""
    if stream is None and t.dtype == dtype and t.is_contiguous():
        return torch.empty_like(t)
    return _empty(t.shape, dtype, t, stream)


def _here(stream, first, *others):
    """The stream to launch on, as a number; all tensors must live on the current device."""
    device = first.get_device()
    if device < 0 or device != _device_of_thread():
        raise ValueError("tensors must live in the current device's memory")
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError("tensors must live in the current device's memory")
    return _stream_of_device(device) if stream is None else getattr(stream, "cuda_stream", stream)


def _rows(t, name, types=_TYPES):
    """(type code, strides) of a tensor whose last dimension is contiguous.  The stride of a dimension of one entry,
    which torch leaves arbitrary, is that of dense rows."""
    code, strides, shape = types.get(t.dtype), t.stride(), t.shape
    if code is None:
        raise ValueError("%s must be one of %s" % (name, ", ".join(str(k)[6:] for k in types)))
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    if len(shape) >= 2 and shape[-2] <= 1 and strides[-2] < shape[-1]:
        strides = strides[:-2] + (shape[-1], strides[-1])
    return code, strides


def _dense(t, name, shape, dtype=_F32):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, str(dtype)[6:], tuple(shape)))
    return t.data_ptr()


def _starts(starts, shape):
    if starts.dtype == _BOOL:
        starts = starts.view(_U8)
    return _dense(starts, "starts", shape, _U8)


def _workspace(bytes_of, sizes, workspace, like, stream):
    """(tensor or None, address, bytes): the caller's workspace, or one allocated here where the sizes need it."""
    if workspace is None:
        size = bytes_of(*sizes)
        if size == 0:
            return None, None, 0
        workspace = _empty(size, _U8, like, stream)
        return workspace, workspace.data_ptr(), size
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _check(status, where):
    if status != 0:
        raise CecaError(status, where)


def dsgd_embed_lookup(E, tokens, scale=1.0, out=None, out_dtype=None, stream=None):
    """out[i, s, :] = scale * E[i, tokens[i, s], :] for n agents' tables E [n, v, d] (float32 or bfloat16, any agent
    and row strides: a block of columns of X unflattened to [n, v, d] will do; an expanded first dimension
    is one table for all agents) and tokens [n, t] (int32 or int64).  A token outside [0, v) gives a zero row."""
    if E.dim() != 3 or tokens.dim() != 2 or tokens.shape[0] != E.shape[0]:
        raise ValueError("E must be [n, v, d] and tokens [n, t]")
    (n, v, d), t = E.shape, tokens.shape[1]
    (te, se), (ti, st) = _rows(E, "E"), _rows(tokens, "tokens", _INDEX)
    s = _here(stream, E, tokens, out)
    if out is None:
        out = _empty((n, t, d), out_dtype or E.dtype, E, stream)
    elif out.shape != (n, t, d) or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError("out must be [n, t, d] of out_dtype")
    to, so = _rows(out, "out")
    _check(library().dsgd_embed_lookup(E.data_ptr(), tokens.data_ptr(), out.data_ptr(), n, t, v, d, se[0], se[1], st[0], so[0],
                                       so[1], te, ti, to, scale, s), "dsgd_embed_lookup")
    return out


def dsgd_embed_workspace_bytes(n, t, v, d):
    return int(library().dsgd_embed_workspace_bytes(n, t, v, d))


def dsgd_embed_grad(dout, tokens, dE, scale=1.0, accumulate=False, workspace=None, stream=None):
    """The gradient of dsgd_embed_lookup: writes (or, with accumulate, adds) scale times the sum of dout's rows
    over each token's positions into dE [n, v, d], and returns it.  workspace: device memory of
    dsgd_embed_workspace_bytes(n, t, v, d) bytes, allocated here when it is None and the sizes need one."""
    if dE.dim() != 3 or tokens.dim() != 2 or tokens.shape[0] != dE.shape[0]:
        raise ValueError("dE must be [n, v, d] and tokens [n, t]")
    (n, v, d), t = dE.shape, tokens.shape[1]
    if dout.shape != (n, t, d):
        raise ValueError("dout must be [n, t, d]")
    (te, se), (ti, st), (to, so) = _rows(dE, "dE"), _rows(tokens, "tokens", _INDEX), _rows(dout, "dout")
    s = _here(stream, dE, tokens, dout, workspace)
    lib = library()
    workspace, pw, size = _workspace(lib.dsgd_embed_workspace_bytes, (n, t, v, d), workspace, dE, stream)
    _check(lib.dsgd_embed_grad(dout.data_ptr(), tokens.data_ptr(), dE.data_ptr(), n, t, v, d, se[0], se[1], st[0], so[0], so[1],
                               te, ti, to, scale, 1 if accumulate else 0, pw, size, s), "dsgd_embed_grad")
    return dE


def dsgd_recurrence_marks(t):
    return int(library().dsgd_recurrence_marks(t))


def dsgd_recurrence_workspace_bytes(b, t, d):
    return int(library().dsgd_recurrence_workspace_bytes(b, t, d))


def dsgd_recurrence(x, f, h0=None, starts=None, h=None, h_last=None, save=False, workspace=None, stream=None):
    """h[:, s] = keep * h[:, s-1] + (1 - sigmoid(f[:, s])) * x[:, s], keep = sigmoid(f[:, s]) or 0 where starts is set,
    for x, f [b, t, d] of one type (float32 or bfloat16).  h0: float32 [b, d]; starts: uint8 or bool [b, t].
    Returns (h, h_last, marks): h like x, h_last the float32 state after the last step, marks what
    dsgd_recurrence_grad starts from (None unless save).  One new token is t = 1 with h0 = h_last = the kept state.
    workspace: device memory of dsgd_recurrence_workspace_bytes(b, t, d) bytes, allocated here when it is None and the sizes need one."""
    shape, dtype = x.shape, x.dtype
    if len(shape) != 3 or f.shape != shape or f.dtype != dtype:
        raise ValueError("x and f must be [b, t, d] of one type")
    b, t, d = shape
    (code, sx), (_, sf) = _rows(x, "x"), _rows(f, "f")
    s = _here(stream, x, f, h0, starts, h, h_last, workspace)
    p0 = None if h0 is None else _dense(h0, "h0", (b, d))
    ps = None if starts is None else _starts(starts, (b, t))
    if h is None:
        h = _like(x, dtype, stream)
    elif h.shape != shape or h.dtype != dtype:
        raise ValueError("h must have the shape and type of x")
    sh = _rows(h, "h")[1]
    if h_last is None:
        h_last = _empty((b, d), _F32, x, stream) if h0 is None else _like(h0, _F32, stream)
        pl = h_last.data_ptr()
    else:
        pl = _dense(h_last, "h_last", (b, d))
    lib = library()
    marks = _empty((b, lib.dsgd_recurrence_marks(t), d), _F32, x, stream) if save else None
    workspace, pw, size = _workspace(lib.dsgd_recurrence_workspace_bytes, shape, workspace, x, stream)
    _check(lib.dsgd_recurrence(x.data_ptr(), f.data_ptr(), p0, ps, h.data_ptr(), pl, None if marks is None else marks.data_ptr(), b,
                               t, d, sx[0], sx[1], sf[0], sf[1], sh[0], sh[1], code, pw, size, s), "dsgd_recurrence")
    return h, h_last, marks


def dsgd_recurrence_grad(x, f, dh, marks, h0=None, starts=None, dh_last=None, dx=None, df=None, dh0=None, workspace=None, stream=None):
    """The gradient of dsgd_recurrence at the same x, f, h0, starts, from the marks that it saved: returns
    (dx, df, dh0), dh0 float32 [b, d] with respect to the initial state, given or zero (h0 itself lies in the marks)."""
    shape, dtype = x.shape, x.dtype
    if len(shape) != 3 or f.shape != shape or dh.shape != shape or f.dtype != dtype or dh.dtype != dtype:
        raise ValueError("x, f and dh must be [b, t, d] of one type")
    b, t, d = shape
    (code, sx), (_, sf), (_, sg) = _rows(x, "x"), _rows(f, "f"), _rows(dh, "dh")
    s = _here(stream, x, f, dh, marks, starts, dh_last, dx, df, dh0, workspace)
    lib = library()
    pm = _dense(marks, "marks", (b, lib.dsgd_recurrence_marks(t), d))
    ps = None if starts is None else _starts(starts, (b, t))
    pl = None if dh_last is None else _dense(dh_last, "dh_last", (b, d))
    if h0 is not None:
        _dense(h0, "h0", (b, d))
    outs = []
    for g, name in ((dx, "dx"), (df, "df")):
        if g is None:
            g = _like(x, dtype, stream)
        elif g.shape != shape or g.dtype != dtype:
            raise ValueError("%s must have the shape and type of x" % name)
        outs.append((g, _rows(g, name)[1]))
    (dx, sdx), (df, sdf) = outs
    if dh0 is None:
        dh0 = _empty((b, d), _F32, x, stream) if dh_last is None else _like(dh_last, _F32, stream)
        p0 = dh0.data_ptr()
    else:
        p0 = _dense(dh0, "dh0", (b, d))
    workspace, pw, size = _workspace(lib.dsgd_recurrence_workspace_bytes, shape, workspace, x, stream)
    _check(lib.dsgd_recurrence_grad(x.data_ptr(), f.data_ptr(), dh.data_ptr(), pm, ps, pl, dx.data_ptr(), df.data_ptr(), p0, b, t, d,
                                    sx[0], sx[1], sf[0], sf[1], sg[0], sg[1], sdx[0], sdx[1], sdf[0], sdf[1], code, pw, size, s),
           "dsgd_recurrence_grad")
    return dx, df, dh0


def _distill(z, idx, t, teacher_lse, weight, loss, dz, stream):
    """What the two calls share: (r, v, k, stream, type codes, row strides, addresses, loss)."""
    shape, top = z.shape, idx.shape
    if len(shape) != 2 or len(top) != 2 or t.shape != top or top[0] != shape[0]:
        raise ValueError("z must be [r, v], idx and t [r, k]")
    r, v = shape
    (tz, sz), (ti, si), (tt, st) = _rows(z, "z"), _rows(idx, "idx", _INDEX), _rows(t, "t")
    s = _here(stream, z, idx, t, teacher_lse, weight, loss, dz)
    pe = None if teacher_lse is None else _dense(teacher_lse, "teacher_lse", (r,))
    pw = None if weight is None else _dense(weight, "weight", (r,))
    if loss is None:
        loss = _empty(r, _F32, z, stream) if weight is None else _like(weight, _F32, stream)
        pl = loss.data_ptr()
    else:
        pl = _dense(loss, "loss", (r,))
    return (z.data_ptr(), idx.data_ptr(), t.data_ptr(), pe, pw, pl), (r, v, top[1], sz[0], si[0], st[0]), (tz, ti, tt), s, loss


def dsgd_distill_loss(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, stream=None):
    """weight * KL(teacher || softmax(z / temperature)) of each row of z [r, v], the teacher being known by its top
    logits t [r, k] at the vocabulary entries idx [r, k] (an idx outside [0, v): fewer entries).  Without teacher_lse
    it is renormalised over them; with it, the mass it leaves is compared with the student's outside the top."""
    at, sizes, types, s, loss = _distill(z, idx, t, teacher_lse, weight, loss, None, stream)
    _check(library().dsgd_distill_loss(*at, *sizes, *types, temperature, s), "dsgd_distill_loss")
    return loss


def dsgd_distill_grad(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, dz=None, stream=None):
    """(loss, dz): dsgd_distill_loss and the gradient of its sum over rows with respect to z, in one pass.  dz may be z."""
    at, sizes, types, s, loss = _distill(z, idx, t, teacher_lse, weight, loss, dz, stream)
    if dz is None:
        dz = _like(z, z.dtype, stream)
    elif dz.shape != z.shape or dz.dtype != z.dtype:
        raise ValueError("dz must have the shape and type of z")
    _check(library().dsgd_distill_grad(*at, dz.data_ptr(), *sizes, _rows(dz, "dz")[1][0], *types, temperature, s), "dsgd_distill_grad")
    return loss, dz
