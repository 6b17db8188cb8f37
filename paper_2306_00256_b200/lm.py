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

GATE_SIGMOID, GATE_SILU = 0, 1

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


def dsgd_kept_row_bytes(d):
    return int(library().dsgd_kept_row_bytes(d))


def dsgd_keep8(x, kept=None, stream=None):
    """x [n, t, d] (float32 or bfloat16) in 8 bits with an exponent for every 32 channels: uint8 [n, t, dsgd_kept_row_bytes(d)].
    For activations that wait for the backward pass; dsgd_block_norm writes its inputs in this form by itself (keep8=True)."""
    return (_module or _load()).keep8(x, kept, stream)


def dsgd_bring8(kept, d, dtype=None, x=None, stream=None):
    """The values [n, t, d] that a kept tensor stands for, exactly, in dtype (float32 unless x says otherwise)."""
    return (_module or _load()).bring8(kept, d, dtype, x, stream)


def dsgd_block_norm(h, y, w_pre, w_post, gate=None, gate_act=GATE_SIGMOID, scale=None, eps=1e-6, h_out=None, u=None, save=False, keep8=False,
                    stream=None):
    """The end of a residual model's block and the start of the next, for n agents' rows [n, t, d]:
        h_out = h + scale * g(gate) * w_post * y / rms(y),   u = w_pre * h_out / rms(h_out)
    h (the residual stream) and h_out have one type, y (the block's output), gate and u one; w_pre, w_post [n, d] and scale [n] are each
    agent's (blocks of columns of X will do).  y = w_post = None leaves the first line out (a model's first norm), w_pre = None the second.
    g is the sigmoid of the gate (GATE_SIGMOID) or gate * sigmoid(gate) (GATE_SILU), 1 without one.
    Returns (h_out, u, stats, kept): stats (None unless save) and kept, with keep8 the kept forms of (h, y, gate), are what
    dsgd_block_norm_grad takes.  h_out may be h, and u may be y or gate."""
    return (_module or _load()).block_norm(h, y, w_pre, w_post, gate, gate_act, scale, eps, h_out, u, save, keep8, stream)


def dsgd_block_norm_workspace_bytes(n, t, d):
    return int(library().dsgd_block_norm_workspace_bytes(n, t, d))


def dsgd_block_norm_grad(h, y, w_pre, w_post, stats, du, dh_out=None, gate=None, gate_act=GATE_SIGMOID, scale=None, dh=None, dy=None,
                         dgate=None, dw_pre=None, dw_post=None, dscale=None, accumulate=False, workspace=None, stream=None):
    """The gradient of dsgd_block_norm from its stats and its inputs h, y and gate, whole or as it kept them in 8 bits: returns
    (dh, dy, dgate, dw_pre, dw_post, dscale), None for what is not there.  du and dh_out (0 when None) are the gradients with respect to u and
    h_out.  dw_pre, dw_post [n, d] and dscale [n] may be blocks of columns of G; with accumulate they are added to.  With kept inputs and no
    dh_out, dh has the type of du unless it is passed in."""
    return (_module or _load()).block_norm_grad(h, y, w_pre, w_post, stats, du, dh_out, gate, gate_act, scale, dh, dy, dgate, dw_pre, dw_post, dscale,
                                                accumulate, workspace, stream)


def dsgd_token_workspace_bytes(r, v, pairs=0):
    return int(library().dsgd_token_workspace_bytes(r, v, pairs))


def dsgd_token_logprob(z, tokens, temperature=1.0, logp=None, workspace=None, stream=None):
    """log softmax(z / temperature) of z [r, v] at each row's token (int32 or int64 [r]): float32 [r], 0 where the token is outside [0, v)."""
    return (_module or _load()).token_logprob(z, tokens, temperature, logp, workspace, stream)


def dsgd_policy_loss(z, tokens, old_logp, advantage, ref_logp=None, weight=None, temperature=1.0, clip_low=0.2, clip_high=0.2, kl=0.0, loss=None,
                     logp=None, workspace=None, stream=None):
    """weight * (-min(p A, clip(p, 1 - clip_low, 1 + clip_high) A) + kl * (exp(x) - 1 - x)) of each row, p = exp(l - old_logp) and
    x = ref_logp - l with l the log-probability of the row's token, A the advantage.  Rows without a token or with weight 0 have loss 0.
    logp: float32 [r], receives l."""
    return (_module or _load()).policy(z, tokens, old_logp, advantage, ref_logp, weight, temperature, clip_low, clip_high, kl, loss, logp, False, None,
                                       workspace, stream)


def dsgd_policy_grad(z, tokens, old_logp, advantage, ref_logp=None, weight=None, temperature=1.0, clip_low=0.2, clip_high=0.2, kl=0.0, loss=None,
                     logp=None, dz=None, workspace=None, stream=None):
    """(loss, dz): dsgd_policy_loss and the gradient of its sum over rows with respect to z.  dz may be z."""
    return (_module or _load()).policy(z, tokens, old_logp, advantage, ref_logp, weight, temperature, clip_low, clip_high, kl, loss, logp, True, dz,
                                       workspace, stream)


def dsgd_preference_loss(z, tokens, bounds, ref_logp=None, weight=None, temperature=1.0, beta=0.1, smoothing=0.0, average=False, loss=None, logp=None,
                         workspace=None, stream=None):
    """The preference loss of pairs of sequences packed into the rows of z [r, v]: sequence j is rows bounds[j] to bounds[j + 1] (int32 or
    int64 [2 pairs + 1]), 2p the preferred one of pair p.  With L the sum (or average) of its rows' log-probabilities and
    m = beta * ((L_2p - ref_2p) - (L_2p+1 - ref_2p+1)): weight * (-(1 - smoothing) log sigmoid(m) - smoothing log sigmoid(-m)).
    Returns (loss [pairs], logp [2 pairs]), logp being the L."""
    return (_module or _load()).preference(z, tokens, bounds, ref_logp, weight, temperature, beta, smoothing, average, loss, logp, False, None,
                                           workspace, stream)


def dsgd_preference_grad(z, tokens, bounds, ref_logp=None, weight=None, temperature=1.0, beta=0.1, smoothing=0.0, average=False, loss=None, logp=None,
                         dz=None, workspace=None, stream=None):
    """(loss, logp, dz): dsgd_preference_loss and the gradient of the sum of its losses with respect to z.  dz may be z."""
    return (_module or _load()).preference(z, tokens, bounds, ref_logp, weight, temperature, beta, smoothing, average, loss, logp, True, dz,
                                           workspace, stream)
