"""The operators around a model's blocks and behind its logits without a GPU: the 64-bit statements against differences of
themselves, and what the library refuses before it launches anything."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import blocks
from paper_2306_00256_b200.binding import Rows

RNG = np.random.default_rng


def _directional(fn, x, grad, seed, tol):
    u = RNG(seed).standard_normal(x.shape)
    h = 1e-5
    quot = (fn(x + h * u) - fn(x - h * u)) / (2 * h)
    assert abs(quot - (grad * u).sum()) <= tol * max(1.0, abs(quot))


@pytest.mark.parametrize("gate", [None, blocks.SIGMOID, blocks.SILU])
@pytest.mark.parametrize("parts", ["both", "no y", "no w_pre"])
def test_block_norm_statement_against_differences(gate, parts):
    r = RNG(1)
    n, t, d = 2, 3, 37
    x = {k: r.standard_normal((n, t, d)) for k in ("h", "y", "gate")}
    x |= {k: 1 + 0.3 * r.standard_normal((n, d)) for k in ("w_pre", "w_post")}
    x["scale"] = r.standard_normal(n)
    du, dh_out = r.standard_normal((n, t, d)), r.standard_normal((n, t, d))
    act = gate or 0
    if gate is None or parts == "no y":
        x["gate"] = None
    if parts == "no y":
        x["y"] = x["w_post"] = x["scale"] = None
    if parts == "no w_pre":
        x["w_pre"] = None

    def loss(**change):
        a = {**x, **change}
        out = blocks.block_norm(a["h"], a["y"], a["w_pre"], a["w_post"], a["gate"], act, a["scale"], 1e-3)
        total = (out["u"][0] * du).sum() if "u" in out else 0.0
        return total + ((out["h"][0] if "h" in out else a["h"]) * dh_out).sum()

    stats = blocks.block_norm(x["h"], x["y"], x["w_pre"], x["w_post"], x["gate"], act, x["scale"], 1e-3)["stats"][0]
    g = blocks.block_norm_grad(x["h"], x["y"], x["w_pre"], x["w_post"], stats, du if x["w_pre"] is not None else None, dh_out, x["gate"], act, x["scale"])
    names = {"h": "dh", "y": "dy", "gate": "dgate", "w_pre": "dw_pre", "w_post": "dw_post", "scale": "dscale"}
    for i, (k, dk) in enumerate(names.items()):
        if x[k] is None:
            assert dk not in g
        else:
            _directional(lambda v: loss(**{k: v}), x[k], g[dk][0], 10 + i, 1e-8)


def _logits(seed, r, v):
    g = RNG(seed)
    tok = g.integers(0, v, r)
    tok[1] = -1
    return g.standard_normal((r, v)) * 2, tok


@pytest.mark.parametrize("temperature", [0.7, 2.0])
@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_statement_against_differences(temperature, kl):
    r, v = 9, 23
    z, tok = _logits(2, r, v)
    g = RNG(3)
    old = blocks.token_logprob(z, tok, temperature)[0] + np.array([0.4, 0, -0.4, 0.1, -0.1, 0.5, -0.5, 0.05, 0.3])
    adv, ref, w = g.standard_normal(r), old + 0.3 * g.standard_normal(r), g.random(r)
    w[4] = 0.0
    args = (old, adv, ref, w, temperature, 0.2, 0.3, kl)
    out = blocks.policy(z, tok, *args)
    assert (out["dz"][0][1] == 0).all() and (out["dz"][0][4] == 0).all()
    if not kl:   # a row whose ratio has left the corridor on the side of its advantage stays still
        assert (out["dz"][0][0] == 0).all() == (adv[0] < 0) and (out["dz"][0][2] == 0).all() == (adv[2] > 0)
    _directional(lambda x: blocks.policy(x, tok, *args)["loss"][0].sum(), z, out["dz"][0], 5, 1e-7)


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("smoothing", [0.0, 0.25])
def test_preference_statement_against_differences(average, smoothing):
    r, v = 14, 19
    z, tok = _logits(6, r, v)
    bounds = [0, 4, 6, 6, 12]
    ref = np.array([-9.0, -4.0, 1.0, -12.0])
    args = (bounds, ref, np.array([0.5, 2.0]), 0.8, 0.3, smoothing, average)
    out = blocks.preference(z, tok, *args)
    assert (out["dz"][0][12:] == 0).all()
    _directional(lambda x: blocks.preference(x, tok, *args)["loss"][0].sum(), z, out["dz"][0], 7, 1e-7)


def test_kept_statement_on_hand_cases():
    x = np.zeros((4, 33))
    x[0, 0], x[0, 1], x[0, 32] = 1.0, 1 / 128, -3.0      # steps of 1/64 and of 1/32
    x[1, :3] = 127.75, -127.75, 0.5                      # cut to 127 steps of 1; a half goes to the even number
    x[2, 5], x[2, 32] = np.inf, 2.0
    q, e, v = blocks.kept(x)
    assert list(e[0]) == [0, 1] and v[0, 0] == 1 and v[0, 1] == 0 and v[0, 32] == -3
    assert list(v[1, :3]) == [127, -127, 0] and e[1, 0] == 6
    assert np.isnan(v[2, :32]).all() and v[2, 32] == 2
    assert (v[3] == 0).all() and list(e[3]) == [-121, -121]
    assert blocks.kept_bytes(x).shape == (4, 48)


def test_kept_row_bytes():
    assert [ceca.dsgd_kept_row_bytes(d) for d in (-1, 0, 1, 14, 15, 32, 33, 2048)] == [0, 0, 16, 16, 16, 48, 48, 2112]


# ------------------------------------------------------------------------------------------- refusals

INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 1, 3, 4, 5
P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104)   # stands for device memory: every call here is refused before anything is launched
NONE = Rows(None, 0, 0)
BIG = 1 << 31


def R(agent=64, row=16, at=4096):
    return Rows(at, agent, row)


def _call(name, args, **change):
    args = dict(args)
    args.update(change)
    return getattr(ceca.library(), name)(*args.values())


KEEP = dict(x=R(), kept=P, n=2, t=4, d=16, type=0, stream=None)
BRING = dict(kept=P, x=R(), n=2, t=4, d=16, type=0, stream=None)
NORM = dict(h=R(), y=R(), gate=R(), w_pre=P, w_post=P, scale=P, wps=16, wqs=16, ss=1, h_out=R(), u=R(), stats=P, h8=P, y8=P, gate8=P, n=2, t=4, d=16,
            st=0, at=0, wt=0, act=0, eps=1e-6, stream=None)
NGRAD = dict(h=R(), y=R(), gate=R(), kept=0, w_pre=P, w_post=P, scale=P, wps=16, wqs=16, ss=1, stats=P, du=R(), dh_out=R(), dh=R(), dy=R(), dgate=R(),
             dw_pre=P, dw_post=P, dscale=P, dps=16, dqs=16, dss=1, acc=0, n=2, t=4, d=16, st=0, at=0, wt=0, act=0, ws=P, size=1 << 30, stream=None)
LOGP = dict(z=P, tok=P, logp=P, r=2, v=8, ldz=8, tz=0, ti=0, temp=1.0, ws=P, size=1 << 20, stream=None)
PLOSS = dict(z=P, tok=P, old=P, adv=P, ref=P, w=P, loss=P, logp=P, r=2, v=8, ldz=8, tz=0, ti=0, temp=1.0, low=0.2, high=0.2, kl=0.1, ws=P, size=1 << 20,
             stream=None)
PGRAD = dict(z=P, tok=P, old=P, adv=P, ref=P, w=P, loss=P, logp=P, dz=ODD, r=2, v=8, ldz=8, lddz=8, tz=0, ti=0, temp=1.0, low=0.2, high=0.2, kl=0.1, ws=P,
             size=1 << 20, stream=None)
QLOSS = dict(z=P, tok=P, bounds=P, ref=P, w=P, loss=P, logp=P, pairs=1, r=2, v=8, ldz=8, tz=0, ti=0, tb=0, temp=1.0, beta=0.1, smooth=0.0, avg=0, ws=P,
             size=1 << 20, stream=None)
QGRAD = dict(z=P, tok=P, bounds=P, ref=P, w=P, loss=P, logp=P, dz=ODD, pairs=1, r=2, v=8, ldz=8, lddz=8, tz=0, ti=0, tb=0, temp=1.0, beta=0.1, smooth=0.0,
             avg=0, ws=P, size=1 << 20, stream=None)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change", [dict(x=NONE), dict(kept=None), dict(n=0), dict(n=65536), dict(t=-1), dict(t=BIG), dict(d=0), dict(d=BIG),
                                    dict(x=R(row=15)), dict(x=R(agent=-1)), dict(type=2)])
def test_keeping_refuses(change):
    assert _call("dsgd_keep8", KEEP, **change) == INVALID
    assert _call("dsgd_bring8", BRING, **change) == INVALID


def test_keeping_refuses_odd_places_and_agents_in_one():
    assert _call("dsgd_keep8", KEEP, kept=ODD) == ALIGNMENT and _call("dsgd_bring8", BRING, kept=ODD) == ALIGNMENT
    assert _call("dsgd_bring8", BRING, x=R(agent=0)) == INVALID


COMMON = [dict(h=NONE), dict(w_post=None), dict(n=0), dict(n=65536), dict(t=-1), dict(t=BIG), dict(d=0), dict(d=BIG), dict(st=2), dict(at=-1), dict(wt=3), dict(act=2),
          dict(h=R(row=15)), dict(y=R(row=8)), dict(gate=R(row=0)), dict(y=R(agent=-1)), dict(y=NONE), dict(wps=-1), dict(wqs=-1), dict(ss=-1)]


@pytest.mark.parametrize("change", COMMON + [
    dict(h_out=NONE), dict(u=NONE), dict(h_out=R(row=15)), dict(u=R(agent=0)), dict(h_out=R(agent=15)), dict(eps=0.0), dict(eps=-1.0), dict(eps=INF), dict(eps=NAN),
    dict(gate=NONE), dict(y=NONE, gate=NONE, w_pre=None)])
def test_block_norm_refuses(change):
    assert _call("dsgd_block_norm", NORM, **change) == INVALID


@pytest.mark.parametrize("change", COMMON + [
    dict(stats=None), dict(du=NONE), dict(dh=NONE), dict(dy=NONE), dict(dgate=NONE), dict(dw_pre=None), dict(dw_post=None), dict(dh=R(row=15)), dict(dy=R(agent=0)),
    dict(dgate=R(agent=-1)), dict(du=R(row=-1)), dict(dh_out=R(agent=-1)), dict(dps=15), dict(dqs=0), dict(dss=0), dict(y=NONE, gate=NONE, w_pre=None)])
def test_block_norm_gradient_refuses(change):
    assert _call("dsgd_block_norm_grad", NGRAD, **change) == INVALID


def test_block_norm_refuses_places_that_do_not_do():
    for k in ("h8", "y8", "gate8"):
        assert _call("dsgd_block_norm", NORM, **{k: ODD}) == ALIGNMENT
    for name, args in (("dsgd_block_norm", NORM), ("dsgd_block_norm_grad", NGRAD)):
        assert _call(name, args, stats=ctypes.c_void_p(4100)) == ALIGNMENT
    for k in ("h", "y", "gate"):
        assert _call("dsgd_block_norm_grad", NGRAD, kept=1, **{k: R(at=4104)}) == ALIGNMENT
    size = ceca.dsgd_block_norm_workspace_bytes(2, 4, 16)
    assert size > 0
    for ws, have in ((None, 0), (P, size - 1), (ODD, size)):
        assert _call("dsgd_block_norm_grad", NGRAD, ws=ws, size=have) == WORKSPACE
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1, 0), (65536, 1, 1), (1, BIG, 1)):
        assert ceca.dsgd_block_norm_workspace_bytes(*bad) == 0


TOKEN = [dict(z=None), dict(tok=None), dict(r=-1), dict(r=1 << 28), dict(v=0), dict(v=BIG), dict(ldz=7), dict(tz=2), dict(ti=2), dict(temp=0.0), dict(temp=-1.0),
         dict(temp=INF), dict(temp=NAN)]


@pytest.mark.parametrize("change", TOKEN + [dict(logp=None)])
def test_log_probability_refuses(change):
    assert _call("dsgd_token_logprob", LOGP, **change) == INVALID


@pytest.mark.parametrize("change", TOKEN + [dict(old=None), dict(adv=None), dict(loss=None), dict(low=-0.1), dict(low=1.1), dict(low=NAN), dict(high=-1.0), dict(high=INF),
                                            dict(kl=-1.0), dict(kl=INF), dict(kl=NAN)])
def test_policy_loss_refuses(change):
    assert _call("dsgd_policy_loss", PLOSS, **change) == INVALID
    assert _call("dsgd_policy_grad", PGRAD, **change) == INVALID


@pytest.mark.parametrize("change", TOKEN + [dict(bounds=None), dict(loss=None), dict(pairs=-1), dict(pairs=1 << 27), dict(tb=2), dict(beta=INF), dict(beta=NAN), dict(smooth=-0.1),
                                            dict(smooth=1.5), dict(smooth=NAN)])
def test_preference_loss_refuses(change):
    assert _call("dsgd_preference_loss", QLOSS, **change) == INVALID
    assert _call("dsgd_preference_grad", QGRAD, **change) == INVALID


@pytest.mark.parametrize("name,args", [("dsgd_policy_grad", PGRAD), ("dsgd_preference_grad", QGRAD)])
def test_gradients_refuse_outputs_that_are_missing_or_crossed(name, args):
    assert _call(name, args, dz=None) == INVALID and _call(name, args, lddz=7) == INVALID
    assert _call(name, args, dz=P, ldz=9, lddz=8) == UNSUPPORTED


def test_losses_refuse_a_workspace_that_does_not_do():
    assert ceca.dsgd_token_workspace_bytes(2, 8) == 0 < ceca.dsgd_token_workspace_bytes(2, 8, 1)
    size = ceca.dsgd_token_workspace_bytes(2, 9000, 1)
    assert size >= ceca.dsgd_token_workspace_bytes(2, 9000) > 0
    for ws, have in ((None, 0), (ODD, size)):
        for name, args in (("dsgd_token_logprob", LOGP), ("dsgd_policy_loss", PLOSS), ("dsgd_policy_grad", PGRAD), ("dsgd_preference_loss", QLOSS),
                           ("dsgd_preference_grad", QGRAD)):
            wide = dict(v=9000, ldz=9000) | (dict(lddz=9000) if "lddz" in args else {})
            assert _call(name, args, ws=ws, size=have, **wide) == WORKSPACE
    assert _call("dsgd_preference_loss", QLOSS, v=9000, ldz=9000, size=size - 1) == WORKSPACE
    assert _call("dsgd_preference_loss", QLOSS, ws=None) == WORKSPACE
    for bad in ((-1, 8, 0), (2, 0, 0), (2, 8, -1), (1 << 28, 8, 0), (1 << 27, 1 << 20, 0)):
        assert ceca.dsgd_token_workspace_bytes(*bad) == 0


def test_calls_without_work_succeed_without_a_device():
    assert _call("dsgd_keep8", KEEP, t=0, kept=None) == 0
    assert _call("dsgd_block_norm", NORM, t=0) == 0
    assert _call("dsgd_token_logprob", LOGP, r=0, z=None, tok=None, logp=None, ws=None, size=0) == 0
    assert _call("dsgd_policy_grad", PGRAD, r=0, z=None, dz=None, ws=None, size=0) == 0
    assert _call("dsgd_preference_loss", QLOSS, r=0, pairs=0, z=None, ws=None, size=0) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros((2, 3, 4)), torch.zeros((2, 4))
    z, tok, f = torch.zeros((2, 8)), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    st = torch.zeros((2, 3, 2))
    for call in (lambda: ceca.dsgd_keep8(x), lambda: ceca.dsgd_keep8(x[0]), lambda: ceca.dsgd_keep8(x.half()), lambda: ceca.dsgd_bring8(x, 4),
                 lambda: ceca.dsgd_block_norm(x, x, w, w), lambda: ceca.dsgd_block_norm(x, None, None, None), lambda: ceca.dsgd_block_norm(x, x, w, None),
                 lambda: ceca.dsgd_block_norm(x, None, w, None, gate=x), lambda: ceca.dsgd_block_norm(x[0], x, w, w),
                 lambda: ceca.dsgd_block_norm_grad(x, x, w, w, st, x), lambda: ceca.dsgd_block_norm_grad(x, x, w, w, st, None),
                 lambda: ceca.dsgd_token_logprob(z, tok), lambda: ceca.dsgd_token_logprob(z, tok.float()), lambda: ceca.dsgd_token_logprob(z, tok[:1]),
                 lambda: ceca.dsgd_policy_grad(z, tok, f, f), lambda: ceca.dsgd_policy_loss(z[0], tok, f, f),
                 lambda: ceca.dsgd_preference_grad(z, tok, tok), lambda: ceca.dsgd_preference_loss(z, tok, torch.zeros(3))):
        with pytest.raises(ValueError):
            call()
