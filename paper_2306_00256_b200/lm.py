"""The language-model operators of include/ceca.h on torch tensors.

The marshalling itself is C++ (csrc/lm_module.cc, built next to the library).  Outputs that are not passed
in, and workspaces, are allocated by torch on the stream that the call runs on; everything else is as in binding.py:
the current stream by default, ValueError for tensors that do not fit, CecaError for what the library refuses.

They build no graph for automatic differentiation: an input may have requires_grad, the outputs never do, and each gradient
is a call of its own (wrap the pair in a torch.autograd.Function where a graph is wanted)."""
import importlib.util
import os

from . import build as _build
from .binding import library

_module = None


def _load():
    global _module
    library()   # which the module links with
    path = _build.build_module() if (_build.module_is_stale() and os.environ.get("CECA_NO_BUILD") != "1") else _build.module_path()
    spec = importlib.util.spec_from_file_location(_build.MODULE_NAME, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    _module = module
    return module


def dsgd_embed_lookup(E, tokens, scale=1.0, out=None, out_dtype=None, stream=None):
    """out[i, s, :] = scale * E[i, tokens[i, s], :] for n agents' tables E [n, v, d] (float32 or bfloat16, any agent
    and row strides: a block of columns of X unflattened to [n, v, d] will do; an expanded first dimension
    is one table for all agents) and tokens [n, t] (int32 or int64).  A token outside [0, v) gives a zero row."""
    return (_module or _load()).embed_lookup(E, tokens, scale, out, out_dtype, stream)


def dsgd_embed_workspace_bytes(n, t, v, d):
    return int(library().dsgd_embed_workspace_bytes(n, t, v, d))


def dsgd_embed_grad(dout, tokens, dE, scale=1.0, accumulate=False, workspace=None, stream=None):
    """The gradient of dsgd_embed_lookup: writes (or, with accumulate, adds) scale times the sum of dout's rows
    over each token's positions into dE [n, v, d], and returns it.  workspace: device memory of
    dsgd_embed_workspace_bytes(n, t, v, d) bytes, allocated here when it is None and the sizes need one."""
    return (_module or _load()).embed_grad(dout, tokens, dE, scale, accumulate, workspace, stream)


def dsgd_recurrence_marks(t):
    return int(library().dsgd_recurrence_marks(t))


def dsgd_recurrence_workspace_bytes(b, t, d):
    return int(library().dsgd_recurrence_workspace_bytes(b, t, d))


def dsgd_recurrence(x, f, h0=None, starts=None, h=None, h_last=None, save=False, workspace=None, stream=None):
    """h[:, s] = keep * h[:, s-1] + (1 - sigmoid(f[:, s])) * x[:, s], keep = sigmoid(f[:, s]) or 0 where starts is set,
    for x, f [b, t, d] of one type (float32 or bfloat16).  h0: float32 [b, d]; starts: uint8 or bool [b, t].
    Returns (h, h_last, marks): h like x, h_last the float32 state after the last step, marks what
    dsgd_recurrence_grad starts from (None unless save).  One new token is t = 1 with h0 = h_last = the kept state.
    workspace: device memory of dsgd_recurrence_workspace_bytes(b, t, d) bytes, allocated here when it is None and
    the sizes need one."""
    return (_module or _load()).recurrence(x, f, h0, starts, h, h_last, save, workspace, stream)


def dsgd_recurrence_grad(x, f, dh, marks, h0=None, starts=None, dh_last=None, dx=None, df=None, dh0=None, workspace=None, stream=None):
    """The gradient of dsgd_recurrence at the same x, f, h0, starts, from the marks that it saved: returns
    (dx, df, dh0), dh0 float32 [b, d] with respect to the initial state, given or zero (h0 itself lies in the marks)."""
    return (_module or _load()).recurrence_grad(x, f, dh, marks, h0, starts, dh_last, dx, df, dh0, workspace, stream)


def dsgd_distill_loss(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, stream=None):
    """weight * KL(teacher || softmax(z / temperature)) of each row of z [r, v], the teacher being known by its top
    logits t [r, k] at the vocabulary entries idx [r, k] (an idx outside [0, v): fewer entries).  Without teacher_lse
    it is renormalised over them; with it, the mass it leaves is compared with the student's outside the top.  (Taken
    before t was rounded to fewer bits, it may leave the top more than all mass; loss and gradient go by the mass there is.)"""
    return (_module or _load()).distill(z, idx, t, teacher_lse, weight, temperature, loss, False, None, stream)


def dsgd_distill_grad(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, loss=None, dz=None, stream=None):
    """(loss, dz): dsgd_distill_loss and the gradient of its sum over rows with respect to z, in one pass.  dz may be z."""
    return (_module or _load()).distill(z, idx, t, teacher_lse, weight, temperature, loss, True, dz, stream)
