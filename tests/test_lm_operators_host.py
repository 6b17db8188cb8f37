"""The language-model operators without a GPU: the 64-bit statements against differences of themselves, and what
the library refuses before it launches anything."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import lm

RNG = np.random.default_rng


def _directional(fn, x, grad, seed, tol):
    u = RNG(seed).standard_normal(x.shape)
    h = 1e-5
    quot = (fn(x + h * u) - fn(x - h * u)) / (2 * h)
    assert abs(quot - (grad * u).sum()) <= tol * max(1.0, abs(quot))


@pytest.mark.parametrize("starts", [False, True])
def test_recurrence_statement_against_differences(starts):
    r = RNG(0)
    b, t, d = 2, 23, 5
    x, f, dh = (r.standard_normal((b, t, d)) for _ in range(3))
    h0, dl = r.standard_normal((b, d)), r.standard_normal((b, d))
    st = (r.random((b, t)) < 0.2).astype(np.uint8) if starts else None

    def loss(x, f, h0):
        out, _ = lm.recurrence(x, f, h0, st)
        return (out["h"][0] * dh).sum() + (out["last"][0] * dl).sum()

    g = lm.recurrence_grad(x, f, dh, h0, st, dl)
    _directional(lambda v: loss(v, f, h0), x, g["dx"][0], 1, 1e-8)
    _directional(lambda v: loss(x, v, h0), f, g["df"][0], 2, 1e-8)
    _directional(lambda v: loss(x, f, v), h0, g["dh0"][0], 3, 1e-8)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("temperature", [0.7, 1.0, 3.0])
def test_distillation_statement_against_differences(tail, temperature):
    r = RNG(4)
    z, t = r.standard_normal((3, 20)) * 2, r.standard_normal((3, 6))
    idx = np.stack([r.permutation(20)[:6] for _ in range(3)])
    idx[0, 2], idx[1, 0] = -1, idx[1, 5]
    lse = np.log(np.where(idx >= 0, np.exp(t / temperature), 0).sum(1)) + 0.3 if tail else None
    w = np.array([0.5, 2.0, 1.0])
    g = lm.distill(z, idx, t, lse, w, temperature)["dz"][0]
    _directional(lambda v: lm.distill(v, idx, t, lse, w, temperature)["loss"][0].sum(), z, g, 5, 1e-8)


def test_embedding_statement_is_its_own_transpose():
    r = RNG(6)
    tok = r.integers(-1, 9, (2, 30))
    E, dout = r.standard_normal((2, 8, 3)), r.standard_normal((2, 30, 3))
    out = lm.embed_lookup(E, tok, 1.5)[0]
    dE = lm.embed_grad(dout, tok, 8, 1.5)[0]
    assert abs((out * dout).sum() - (E * dE).sum()) < 1e-10


INVALID, WORKSPACE, UNSUPPORTED = 1, 5, 4
P = ctypes.c_void_p(4096)   # stands for device memory: every call here is refused before anything is launched


def _call(name, args, **change):
    args = dict(args)
    args.update(change)
    return getattr(ceca.library(), name)(*args.values())


LOOKUP = dict(E=P, tokens=P, out=P, n=2, t=4, v=8, d=16, agent=128, row=16, tok=4, o_agent=64, o_row=16, te=0, ti=0, to=0, scale=1.0, stream=None)
GRAD = dict(dout=P, tokens=P, dE=P, n=2, t=4, v=8, d=16, agent=128, row=16, tok=4, o_agent=64, o_row=16, te=0, ti=0, to=0, scale=1.0,
            acc=0, ws=P, size=1 << 20, stream=None)
RECUR = dict(x=P, f=P, h0=None, starts=None, h=P, last=P, marks=None, b=2, t=4, d=16, xs=64, xt=16, fs=64, ft=16, hs=64, ht=16, type=0, ws=None, size=0, stream=None)
RGRAD = dict(x=P, f=P, dh=P, marks=P, starts=None, dlast=None, dx=P, df=P, dh0=None, b=2, t=4, d=16, xs=64, xt=16, fs=64, ft=16, dhs=64, dht=16,
             dxs=64, dxt=16, dfs=64, dft=16, type=0, ws=None, size=0, stream=None)
LOSS = dict(z=P, idx=P, t=P, lse=None, w=None, loss=P, r=2, v=8, k=3, ldz=8, ldi=3, ldt=3, tz=0, ti=0, tt=0, temp=1.0, stream=None)
DGRAD = dict(z=P, idx=P, t=P, lse=None, w=None, loss=P, dz=P, r=2, v=8, k=3, ldz=8, ldi=3, ldt=3, lddz=8, tz=0, ti=0, tt=0, temp=1.0, stream=None)
BIG = 1 << 31


@pytest.mark.parametrize("change", [
    dict(E=None), dict(tokens=None), dict(out=None), dict(n=0), dict(n=-1), dict(t=-1), dict(t=BIG), dict(v=0), dict(v=BIG), dict(d=0), dict(agent=-1),
    dict(row=15), dict(tok=-1), dict(o_agent=-1), dict(o_row=15), dict(o_agent=0), dict(te=2), dict(ti=2), dict(to=-1)])
def test_lookup_refuses(change):
    assert _call("dsgd_embed_lookup", LOOKUP, **change) == INVALID


@pytest.mark.parametrize("change,status", [(c, INVALID) for c in [
    dict(dout=None), dict(tokens=None), dict(dE=None), dict(n=0), dict(t=-1), dict(t=BIG), dict(v=0), dict(v=BIG), dict(d=0), dict(agent=127), dict(agent=0),
    dict(row=15), dict(tok=-1), dict(o_row=-1), dict(te=2), dict(ti=-1), dict(to=9)]] + [
    (dict(t=4000, ws=None), WORKSPACE), (dict(t=4000, size=8), WORKSPACE), (dict(t=4000, ws=ctypes.c_void_p(4104)), WORKSPACE)])
def test_lookup_gradient_refuses(change, status):
    assert _call("dsgd_embed_grad", GRAD, **change) == status


@pytest.mark.parametrize("change", [
    dict(x=None), dict(f=None), dict(h=None), dict(b=0), dict(t=-1), dict(t=BIG), dict(d=0), dict(d=BIG), dict(xt=15), dict(ft=0), dict(ht=15), dict(xs=-1),
    dict(hs=0), dict(type=2)])
def test_recurrence_refuses(change):
    assert _call("dsgd_recurrence", RECUR, **change) == INVALID


@pytest.mark.parametrize("change", [
    dict(x=None), dict(f=None), dict(dh=None), dict(marks=None), dict(dx=None), dict(df=None), dict(b=0), dict(t=-1), dict(t=BIG), dict(d=0), dict(xt=15),
    dict(ft=1), dict(dht=-1), dict(dxt=15), dict(dft=15), dict(dxs=0), dict(dfs=0), dict(fs=-1), dict(type=-1)])
def test_recurrence_gradient_refuses(change):
    assert _call("dsgd_recurrence_grad", RGRAD, **change) == INVALID


@pytest.mark.parametrize("change", [
    dict(z=None), dict(idx=None), dict(t=None), dict(r=-1), dict(r=BIG), dict(v=0), dict(v=BIG), dict(k=-1), dict(k=4097), dict(ldz=7), dict(ldi=2), dict(ldt=2),
    dict(tz=2), dict(ti=2), dict(tt=2), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("inf")), dict(temp=float("nan"))])
def test_distillation_refuses(change):
    assert _call("dsgd_distill_loss", LOSS, **change) == INVALID
    assert _call("dsgd_distill_grad", DGRAD, **change) == INVALID


def test_distillation_refuses_outputs_that_are_missing_or_crossed():
    assert _call("dsgd_distill_loss", LOSS, loss=None) == INVALID
    assert _call("dsgd_distill_grad", DGRAD, dz=None) == INVALID
    assert _call("dsgd_distill_grad", DGRAD, lddz=7) == INVALID
    assert _call("dsgd_distill_grad", DGRAD, ldz=9, lddz=8) == UNSUPPORTED   # P is both z and dz


def test_recurrence_refuses_a_workspace_that_does_not_do():
    t, size = 5000, ceca.dsgd_recurrence_workspace_bytes(2, 5000, 16)
    assert size > 0 and size % 4 == 0
    for ws, have in ((None, 0), (P, size - 1), (ctypes.c_void_p(4104), size)):
        assert _call("dsgd_recurrence", RECUR, t=t, ws=ws, size=have) == WORKSPACE
        assert _call("dsgd_recurrence_grad", RGRAD, t=t, ws=ws, size=have) == WORKSPACE


def test_calls_without_work_succeed_without_a_device():
    assert _call("dsgd_embed_lookup", LOOKUP, t=0, out=None) == 0
    assert _call("dsgd_distill_loss", LOSS, r=0, z=None, loss=None) == 0


def test_sizes():
    assert [ceca.dsgd_recurrence_marks(t) for t in (-1, 0, 1)] == [0, 0, 1]
    assert ceca.dsgd_recurrence_marks(100000) > ceca.dsgd_recurrence_marks(1000) >= 1
    assert ceca.dsgd_recurrence_workspace_bytes(64, 1000, 2048) == 0 and ceca.dsgd_recurrence_workspace_bytes(1, 1, 64) == 0
    assert ceca.dsgd_recurrence_workspace_bytes(0, 100, 64) == 0
    assert ceca.dsgd_embed_workspace_bytes(2, 1000, 1000, 64) >= 4 * (2 * 1000 + 2 * 1001) and ceca.dsgd_embed_workspace_bytes(2, 1, 1000, 64) == 0
    for bad in ((0, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, BIG, 1, 1)):
        assert ceca.dsgd_embed_workspace_bytes(*bad) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros((2, 3, 4))
    tok = torch.zeros((2, 3), dtype=torch.int32)
    z, i = torch.zeros((2, 8)), torch.zeros((2, 3), dtype=torch.int64)
    for call in (lambda: ceca.dsgd_embed_lookup(x, tok), lambda: ceca.dsgd_embed_lookup(x.half(), tok), lambda: ceca.dsgd_embed_lookup(x, tok[:1]),
                 lambda: ceca.dsgd_embed_grad(x, tok, x[0]), lambda: ceca.dsgd_recurrence(x, x), lambda: ceca.dsgd_recurrence(x, x[:, :2]),
                 lambda: ceca.dsgd_recurrence(x.double(), x.double()), lambda: ceca.dsgd_recurrence(x.transpose(1, 2), x.transpose(1, 2)),
                 lambda: ceca.dsgd_recurrence(x, x, h0=torch.zeros(4)), lambda: ceca.dsgd_recurrence_grad(x, x, x, torch.zeros(1)),
                 lambda: ceca.dsgd_distill_loss(z, i, torch.zeros((2, 3))), lambda: ceca.dsgd_distill_loss(z, i.float(), torch.zeros((2, 3))),
                 lambda: ceca.dsgd_distill_grad(z, i, torch.zeros((2, 2)))):
        with pytest.raises(ValueError):
            call()
