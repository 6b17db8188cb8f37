"""The language-model operators on the GPU against their 64-bit statements, element by element, within the bounds
that oracle/lm.py derives for fp32 arithmetic (one more rounding for bf16 outputs)."""
import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import lm

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def _np(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _close(got, pair, name):
    want, tol = pair
    got = _np(got)
    assert got.shape == want.shape, name
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    assert not bad.any(), "%s: %d of %d off, first at %s: %r, want %r +- %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(shape, dtype, seed, mean=0.0, std=1.0):
    return (torch.randn(shape, generator=_gen(seed)) * std + mean).to(dtype).to(DEV)


def _inside(shape, strides, offset, dtype):
    """A view of the given strides in a NaN-filled buffer, and the buffer."""
    buf = torch.full((offset + sum((n - 1) * s for n, s in zip(shape, strides) if n) + 1 + 64,), NAN, dtype=dtype, device=DEV)
    return buf.as_strided(shape, strides, offset), buf


def _untouched(view, buf):
    """The buffer holds NaN everywhere but in the view."""
    mark = torch.zeros_like(buf)
    mark.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(1)
    return bool(torch.isnan(buf[mark == 0]).all())


# ------------------------------------------------------------------------------------------------ embedding

EMBED = [  # n, t, v, d
    (1, 1, 1, 1), (2, 5, 3, 7), (3, 64, 100, 32), (1, 300, 17, 129), (4, 129, 1025, 64), (2, 1000, 5000, 96),
    (5, 33, 513, 250), (1, 2000, 40, 260), (2, 77, 4099, 1031), (1, 40, 70000, 16), (1, 4097, 300, 512), (3, 9, 65, 2056),
    (2, 256, 30, 40), (1, 257, 30, 1048), (1, 9000, 20000, 24), (3, 70, 65, 100), (1, 700, 300, 1044),
]


def _tokens(n, t, v, seed, dtype):
    g = _gen(seed)
    tok = (torch.rand((n, t), generator=g) ** 3 * v).long().clamp(0, v - 1)
    tok[torch.rand((n, t), generator=g) < 0.05] = -1
    tok[torch.rand((n, t), generator=g) < 0.03] = v
    if dtype == torch.int64 and t > 2:
        tok[:, 2] = 2**32 + 1   # not token 1
    return tok.to(dtype).to(DEV)


@pytest.mark.parametrize("n,t,v,d", EMBED)
@pytest.mark.parametrize("te,to,ti", [(F32, F32, torch.int32), (BF16, BF16, torch.int64), (F32, BF16, torch.int64), (BF16, F32, torch.int32)])
def test_embedding_lookup_and_gradient(n, t, v, d, te, to, ti):
    tok = _tokens(n, t, v, 1, ti)
    E = _randn((n, v, d), te, 2)
    scale = 1.7
    out = ceca.dsgd_embed_lookup(E, tok, scale, out_dtype=to)
    assert out.dtype == to
    _close(out, lm.embed_lookup(_np(E), _np(tok), np.float32(scale), to == BF16), "out")
    dout = _randn((n, t, d), to, 3)
    dE = torch.full((n, v, d), NAN, dtype=te, device=DEV)
    got = ceca.dsgd_embed_grad(dout, tok, dE, scale)
    assert got is dE
    _close(dE, lm.embed_grad(_np(dout), _np(tok), v, np.float32(scale), None, te == BF16), "dE")
    again = ceca.dsgd_embed_grad(dout, tok, torch.empty_like(dE), scale)
    assert torch.equal(dE, again)
    more = _randn((n, v, d), te, 4)
    before = _np(more)
    ceca.dsgd_embed_grad(dout, tok, more, scale, accumulate=True)
    _close(more, lm.embed_grad(_np(dout), _np(tok), v, np.float32(scale), before, te == BF16), "dE accumulated")


@pytest.mark.parametrize("te,to", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 16), (3, 1), (5, 2)])
@pytest.mark.parametrize("t", [50, 300])
def test_embedding_in_a_block_of_parameter_columns(te, to, pad, offset, t):
    # the table of every agent is a block of columns of its row of X, and out a padded activation
    n, v, d = 3, 41, 64
    ld = v * d + 100 + pad
    E, _ = _inside((n, v, d), (ld, d, 1), offset, te)
    E.copy_(_randn((n, v, d), te, 5))
    tok = _tokens(n, t, v, 6, torch.int64)
    out, buf = _inside((n, t, d), (t * (d + pad) + 7, d + pad, 1), offset, to)
    ceca.dsgd_embed_lookup(E, tok, 0.5, out=out)
    _close(out, lm.embed_lookup(_np(E), _np(tok), 0.5, to == BF16), "out")
    assert _untouched(out, buf)
    dE, gbuf = _inside((n, v, d), (ld, d, 1), offset, te)
    size = ceca.dsgd_embed_workspace_bytes(n, t, v, d)
    ws = torch.full((size + 256,), 77, dtype=torch.uint8, device=DEV)
    ceca.dsgd_embed_grad(out, tok, dE, 0.5, workspace=ws[:size])
    _close(dE, lm.embed_grad(_np(out), _np(tok), v, 0.5, None, te == BF16), "dE")
    assert _untouched(dE, gbuf) and bool((ws[size:] == 77).all())


def test_embedding_of_no_positions():
    tok = torch.zeros((2, 0), dtype=torch.int32, device=DEV)
    E = _randn((2, 9, 8), F32, 0)
    assert ceca.dsgd_embed_lookup(E, tok).shape == (2, 0, 8)
    dE = torch.full((2, 9, 8), NAN, device=DEV)
    dout = torch.empty((2, 0, 8), device=DEV)
    ceca.dsgd_embed_grad(dout, tok, dE, accumulate=True)
    assert bool(torch.isnan(dE).all())
    ceca.dsgd_embed_grad(dout, tok, dE)
    assert bool((dE == 0).all())


def test_embedding_of_empty_positions_only():
    tok = torch.full((2, 70), -1, dtype=torch.int64, device=DEV)
    E = torch.full((2, 9, 40), NAN, device=DEV)
    assert bool((ceca.dsgd_embed_lookup(E, tok) == 0).all())
    dE = torch.full((2, 9, 40), NAN, device=DEV)
    ceca.dsgd_embed_grad(torch.full((2, 70, 40), NAN, device=DEV), tok, dE)
    assert bool((dE == 0).all())


@pytest.mark.parametrize("te,to", [(F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("hot", [1, 2, 5])
@pytest.mark.parametrize("t", [200, 9001])
def test_embedding_gradient_of_a_few_frequent_tokens(te, to, hot, t):
    # lists far longer than a warp takes, next to rows with none
    n, v, d = 2, 50, 72
    tok = (torch.arange(n * t).reshape(n, t) % hot * 7).to(torch.int32).to(DEV)
    dout = _randn((n, t, d), to, 8)
    dE = torch.empty((n, v, d), dtype=te, device=DEV)
    ceca.dsgd_embed_grad(dout, tok, dE, 0.25)
    _close(dE, lm.embed_grad(_np(dout), _np(tok), v, 0.25, None, te == BF16), "dE")
    assert torch.equal(dE, ceca.dsgd_embed_grad(dout, tok, torch.empty_like(dE), 0.25))


def test_embedding_of_one_table_for_all_agents():
    E = _randn((1, 30, 24), F32, 1).expand(4, 30, 24)
    tok = _tokens(4, 11, 30, 2, torch.int32)
    _close(ceca.dsgd_embed_lookup(E, tok, 2.0), lm.embed_lookup(_np(E), _np(tok), 2.0), "out")
    with pytest.raises(ceca.CecaError) as e:   # their gradients would fall on one another
        ceca.dsgd_embed_grad(torch.zeros((4, 11, 24), device=DEV), tok, E)
    assert e.value.status == 1
    # the gradient of a shared table: all agents' positions in one list
    dout = _randn((4, 11, 24), F32, 3)
    dE = torch.empty((1, 30, 24), device=DEV)
    ceca.dsgd_embed_grad(dout.reshape(1, 44, 24), tok.reshape(1, 44), dE, 2.0)
    _close(dE, lm.embed_grad(_np(dout).reshape(1, 44, 24), _np(tok).reshape(1, 44), 30, 2.0), "dE")


def test_embedding_gradient_of_a_broadcast_output_gradient():
    tok = _tokens(2, 37, 20, 4, torch.int32)
    row = _randn((16,), F32, 5)
    dE = torch.empty((2, 20, 16), device=DEV)
    ceca.dsgd_embed_grad(row.expand(2, 37, 16), tok, dE)
    _close(dE, lm.embed_grad(np.broadcast_to(_np(row), (2, 37, 16)), _np(tok), 20, 1.0), "dE")


def test_embedding_rows_beyond_32_bit_offsets():
    v, d, ld = 70000, 64, 65536
    buf = torch.empty(v * ld, dtype=BF16, device=DEV)
    E = buf.view(1, v, ld)[:, :, :d]
    tok = torch.tensor([[v - 1, 65536, 3, v - 1]], dtype=torch.int32, device=DEV)
    rows = _randn((3, d), BF16, 6)
    for j, w in enumerate((v - 1, 65536, 3)):
        E[0, w] = rows[j]
    out = ceca.dsgd_embed_lookup(E, tok, 1.0)
    assert torch.equal(out[0], rows[[0, 1, 2, 0]])
    ceca.dsgd_embed_grad(out, tok, E, 1.0, accumulate=True)
    assert torch.equal(E[0, 65536], 2 * rows[1]) and torch.equal(E[0, v - 1], (3 * rows[0].float()).to(BF16))
    assert torch.equal(E[0, 3], 2 * rows[2])


# ------------------------------------------------------------------------------------------------ recurrence

RECUR = [  # b, t, d
    (1, 1, 1), (2, 1, 64), (300, 1, 40), (3, 2, 33), (1, 5, 256), (2, 31, 8), (1, 127, 70), (2, 128, 64), (1, 129, 72), (4, 200, 520),
    (1, 1025, 24), (2, 513, 136), (1, 3000, 5), (1, 2500, 64), (7, 385, 16), (1, 17, 2048), (3, 16, 1000), (1, 6000, 32),
    (60, 100, 520), (30, 300, 520), (14, 300, 520), (8, 290, 520), (30, 150, 521), (16, 140, 521),   # channels enough for 4, 8 and 16 warps
]


def _recur_inputs(b, t, d, dtype, h0, starts, seed=0, mean=1.0):
    x, f = _randn((b, t, d), dtype, seed), _randn((b, t, d), dtype, seed + 1, mean, 2.0)
    s = (torch.rand((b, t), generator=_gen(seed + 2)) < 0.05).to(torch.uint8).to(DEV) if starts else None
    return x, f, _randn((b, d), F32, seed + 3) if h0 else None, s


@pytest.mark.parametrize("b,t,d", RECUR)
@pytest.mark.parametrize("dtype,h0,starts", [(F32, False, False), (F32, True, True), (BF16, True, False), (BF16, False, True)])
def test_recurrence_and_gradient(b, t, d, dtype, h0, starts):
    x, f, h0, st = _recur_inputs(b, t, d, dtype, h0, starts)
    bf = dtype == BF16
    h, last, marks = ceca.dsgd_recurrence(x, f, h0=h0, starts=st, save=True)
    want, _ = lm.recurrence(_np(x), _np(f), _np(h0), _np(st), bf)
    _close(h, want["h"], "h")
    _close(last, want["last"], "last")
    h2, last2, none = ceca.dsgd_recurrence(x, f, h0=h0, starts=st)
    assert none is None and torch.equal(h, h2) and torch.equal(last, last2)
    dh, dl = _randn((b, t, d), dtype, 7), _randn((b, d), F32, 8)
    for dlast in (dl, None):
        dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, dh, marks, h0=h0, starts=st, dh_last=dlast)
        want = lm.recurrence_grad(_np(x), _np(f), _np(dh), _np(h0), _np(st), _np(dlast), bf)
        _close(dx, want["dx"], "dx")
        _close(df, want["df"], "df")
        _close(dh0, want["dh0"], "dh0")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mean", [-6.0, 7.0])
def test_recurrence_with_gates_near_closed_and_open(dtype, mean):
    x, f, h0, _ = _recur_inputs(2, 700, 48, dtype, True, False, 20, mean)
    h, last, marks = ceca.dsgd_recurrence(x, f, h0=h0, save=True)
    want, _ = lm.recurrence(_np(x), _np(f), _np(h0), None, dtype == BF16)
    _close(h, want["h"], "h")
    dh = _randn((2, 700, 48), dtype, 27)
    dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, dh, marks, h0=h0)
    want = lm.recurrence_grad(_np(x), _np(f), _np(dh), _np(h0), None, None, dtype == BF16)
    for g, k in ((dx, "dx"), (df, "df"), (dh0, "dh0")):
        _close(g, want[k], k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [3, 200, 1500])
def test_recurrence_gates_that_are_shut_or_open_for_good(dtype, t):
    # f = +inf keeps the state exactly, -inf replaces it; the type's extremes behave the same
    d = 64
    x = _randn((1, t, d), dtype, 30)
    f = torch.zeros((1, t, d), dtype=dtype, device=DEV)
    f[..., 0], f[..., 1], f[..., 2], f[..., 3] = float("inf"), -float("inf"), torch.finfo(dtype).max, torch.finfo(dtype).min
    h0 = _randn((1, d), F32, 31)
    h, last, marks = ceca.dsgd_recurrence(x, f, h0=h0, save=True)
    for c in (0, 2):
        assert torch.equal(last[:, c], h0[:, c])
    for c in (1, 3):
        assert torch.equal(h[..., c], x[..., c])
    dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, torch.ones_like(x), marks, h0=h0)
    assert bool((dx[..., 0] == 0).all()) and bool((dx[..., 1] == 1).all()) and bool((df[..., :4] == 0).all())
    assert float(dh0[0, 0]) == t and float(dh0[0, 1]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,cut", [(40, 17), (600, 129), (600, 256), (2100, 1030)])
def test_recurrence_a_document_does_not_see_the_one_before(dtype, t, cut):
    # NaN and infinity before the document's first step stay there, in both directions
    d = 72
    x, f, _, _ = _recur_inputs(1, t, d, dtype, False, False, 40)
    dh = _randn((1, t, d), dtype, 45)
    st = torch.zeros((1, t), dtype=torch.uint8, device=DEV)
    st[0, cut] = 1
    alone, last, m = ceca.dsgd_recurrence(x[:, cut:].contiguous(), f[:, cut:].contiguous(), save=True)
    ref = lm.recurrence_grad(_np(x[:, cut:]), _np(f[:, cut:]), _np(dh[:, cut:]), None, None, None, dtype == BF16)
    want, _ = lm.recurrence(_np(x[:, cut:]), _np(f[:, cut:]), None, None, dtype == BF16)
    bad = x.clone()
    bad[0, cut - 1, ::2], bad[0, cut // 2, 1::2] = NAN, float("inf")
    h, last, marks = ceca.dsgd_recurrence(bad, f, h0=torch.full((1, d), NAN, device=DEV), starts=st, save=True)
    _close(h[:, cut:], want["h"], "h")
    _close(last, want["last"], "last")
    dx, df, dh0 = ceca.dsgd_recurrence_grad(bad, f, dh, marks, starts=st)
    _close(dx[:, cut:], ref["dx"], "dx")
    _close(df[:, cut:], ref["df"], "df")
    late = dh.clone()
    late[0, cut:] = NAN   # and gradients of the later document do not reach the earlier one
    h, last, marks = ceca.dsgd_recurrence(x, f, starts=st, save=True)
    dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, late, marks, starts=st)
    ref = lm.recurrence_grad(_np(x[:, :cut]), _np(f[:, :cut]), _np(dh[:, :cut]), None, None, None, dtype == BF16)
    _close(dx[:, :cut], ref["dx"], "dx")
    _close(df[:, :cut], ref["df"], "df")
    _close(dh0, ref["dh0"], "dh0")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,d,pad,offset", [(140, 64, 8, 8), (140, 64, 3, 1), (1, 64, 16, 0), (9, 50, 1, 3), (300, 128, 0, 4)])
def test_recurrence_strided_views(dtype, t, d, pad, offset):
    # x and f are halves of one projection; h, dx, df lie in padded buffers
    b = 2
    proj = _randn((b, t, 2 * d + pad), dtype, 50)
    x, f = proj[:, :, :d], proj[:, :, d:2 * d]
    h, hb = _inside((b, t, d), (t * (d + pad) + 5, d + pad, 1), offset, dtype)
    h0 = _randn((b, d), F32, 51)
    state = h0.clone()
    _, last, marks = ceca.dsgd_recurrence(x, f, h0=state, h=h, h_last=state, save=True)   # the state in place
    want, _ = lm.recurrence(_np(x), _np(f), _np(h0), None, dtype == BF16)
    _close(h, want["h"], "h")
    _close(state, want["last"], "last")
    assert _untouched(h, hb)
    dh = _randn((b, t, d), dtype, 52)
    gbuf = torch.full((b, t, 2 * d + pad), NAN, dtype=dtype, device=DEV)
    dx, df = gbuf[:, :, :d], gbuf[:, :, d:2 * d]
    _, _, dh0 = ceca.dsgd_recurrence_grad(x, f, dh, marks, h0=h0, dx=dx, df=df)
    want = lm.recurrence_grad(_np(x), _np(f), _np(dh), _np(h0), None, None, dtype == BF16)
    for g, k in ((dx, "dx"), (df, "df"), (dh0, "dh0")):
        _close(g, want[k], k)
    assert bool(torch.isnan(gbuf[:, :, 2 * d:]).all())


@pytest.mark.parametrize("dtype,t", [(F32, 300), (BF16, 300), (BF16, 1), (F32, 6)])
def test_recurrence_in_place(dtype, t):
    x, f, h0, st = _recur_inputs(2, t, 64, dtype, True, True, 60)
    h, last, marks = ceca.dsgd_recurrence(x, f, h0=h0, starts=st, save=True)
    for k in range(2):
        xs, fs = x.clone(), f.clone()
        got, _, _ = ceca.dsgd_recurrence(xs, fs, h0=h0, starts=st, h=(xs, fs)[k])
        assert torch.equal(got, h)
    dh = _randn((2, t, 64), dtype, 66)
    dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, dh, marks, h0=h0, starts=st)
    dhs, fs = dh.clone(), f.clone()
    gx, gf, _ = ceca.dsgd_recurrence_grad(x, fs, dhs, marks, h0=h0, starts=st, dx=dhs, df=fs)
    assert torch.equal(gx, dx) and torch.equal(gf, df)
    xs = x.clone()
    gx, gf, _ = ceca.dsgd_recurrence_grad(xs, f, dh, marks, h0=h0, starts=st, dx=xs)
    assert torch.equal(gx, dx) and torch.equal(gf, df)


def test_recurrence_of_no_steps():
    x = torch.empty((2, 0, 12), device=DEV)
    h0 = _randn((2, 12), F32, 70)
    h, last, marks = ceca.dsgd_recurrence(x, x, h0=h0, save=True)
    assert h.shape == (2, 0, 12) and torch.equal(last, h0) and marks.shape == (2, 0, 12)
    assert bool((ceca.dsgd_recurrence(x, x)[1] == 0).all())
    dl = _randn((2, 12), F32, 71)
    _, _, dh0 = ceca.dsgd_recurrence_grad(x, x, x, marks, h0=h0, dh_last=dl)
    assert torch.equal(dh0, dl)


def test_recurrence_token_by_token_is_the_whole_sequence():
    b, t, d = 3, 40, 72
    x, f, h0, st = _recur_inputs(b, t, d, F32, True, True, 80)
    want, _ = lm.recurrence(_np(x), _np(f), _np(h0), _np(st))
    state, steps = h0.clone(), []
    for s in range(t):
        h, _, _ = ceca.dsgd_recurrence(x[:, s:s + 1], f[:, s:s + 1], h0=state, starts=st[:, s:s + 1].contiguous(), h_last=state)
        steps.append(h)
    _close(torch.cat(steps, 1), want["h"], "h")
    _close(state, want["last"], "last")


def test_recurrence_steps_beyond_32_bit_offsets():
    t, ld, d = 70000, 65536, 16
    buf = torch.empty(t * ld, dtype=BF16, device=DEV).view(1, t, ld)
    x, f, h, dx, df = (buf[:, :, 16 * j:16 * j + 16] for j in range(5))
    x.copy_(_randn((1, t, d), BF16, 90))
    f.copy_(_randn((1, t, d), BF16, 91, -1.0))
    xs, fs = x.contiguous(), f.contiguous()
    _, last, marks = ceca.dsgd_recurrence(x, f, h=h, save=True)
    want, wlast, wmarks = ceca.dsgd_recurrence(xs, fs, save=True)
    assert torch.equal(h, want) and torch.equal(last, wlast) and torch.equal(marks, wmarks)
    ceca.dsgd_recurrence_grad(x, f, h, marks, dx=dx, df=df)
    wx, wf, _ = ceca.dsgd_recurrence_grad(xs, fs, want, wmarks)
    assert torch.equal(dx, wx) and torch.equal(df, wf)


# ------------------------------------------------------------------------------------------------ distillation

DISTILL = [  # r, v, k
    (1, 1, 1), (3, 2, 1), (5, 7, 7), (4, 33, 5), (3, 100, 64), (2, 129, 1), (6, 1000, 8), (2, 1023, 100), (2, 4096, 16), (3, 5001, 50),
    (2, 16385, 33), (2, 32000, 64), (2, 50001, 20), (1, 65536, 300), (1, 100003, 7), (1, 140000, 64), (1, 300001, 12),
]


def _distill_inputs(r, v, k, dtype, tail, seed=0, tt=F32, ti=torch.int32, temperature=1.0):
    g = _gen(seed)
    idx = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(r)])
    t = torch.randn((r, k), generator=g) * 2 + 3
    z = torch.randn((r, v), generator=g) * 2
    z.scatter_add_(1, idx, t * 0.7)
    t = t.to(tt)
    if k > 2:
        idx[:, 1] = -1
        idx[0, 2] = v
    lse = None
    if tail:
        here = (idx >= 0) & (idx < v)
        lse = torch.logsumexp((t.double() / temperature).masked_fill(~here, -float("inf")), 1).float() + 0.2
        lse = lse.to(DEV)
    w = torch.rand(r, generator=g) + 0.5
    if r > 2:
        w[1] = 0
    return z.to(dtype).to(DEV), idx.to(ti).to(DEV), t.to(DEV), lse, w.to(DEV)


def _distill_check(z, idx, t, lse, w, temperature, name=""):
    bf = z.dtype == BF16
    want = lm.distill(_np(z), _np(idx), _np(t), _np(lse), _np(w), temperature, bf)
    more = {"teacher_lse": lse, "weight": w, "temperature": temperature}
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, **more)
    _close(loss, want["loss"], name + "loss")
    _close(dz, want["dz"], name + "dz")
    only = ceca.dsgd_distill_loss(z, idx, t, **more)
    _close(only, want["loss"], name + "loss alone")
    loss2, dz2 = ceca.dsgd_distill_grad(z, idx, t, **more)
    assert torch.equal(loss, loss2, ) or bool(torch.isnan(loss).any())
    assert torch.equal(dz, dz2) or bool(torch.isnan(dz.float()).any())
    return loss, dz


@pytest.mark.parametrize("r,v,k", DISTILL)
@pytest.mark.parametrize("dtype,tail,temperature,tt,ti", [
    (F32, False, 1.0, F32, torch.int32), (F32, True, 2.0, BF16, torch.int64), (BF16, True, 1.0, F32, torch.int64), (BF16, False, 0.7, BF16, torch.int32)])
def test_distillation_loss_and_gradient(r, v, k, dtype, tail, temperature, tt, ti):
    z, idx, t, lse, w = _distill_inputs(r, v, k, dtype, tail, 1, tt, ti, temperature)
    _distill_check(z, idx, t, lse, w, temperature)
    _distill_check(z, idx, t, lse, None, temperature, "no weights: ")


@pytest.mark.parametrize("r,v", [(600, 9001), (2400, 130), (900, 1001), (700, 3000)])   # more rows than the GPU holds at a time
@pytest.mark.parametrize("dtype,tail", [(F32, True), (BF16, False), (BF16, True)])
def test_distillation_of_many_rows(r, v, dtype, tail):
    z, idx, t, lse, w = _distill_inputs(r, v, 5, dtype, tail, 21)
    w[::7] = 0
    idx[5, 3], idx[5, 4] = 9, 9
    _distill_check(z, idx, t, lse, w, 1.0)


def test_distillation_over_more_entries_than_the_bitmap_has_bits():
    # parts of more than 2^20 logits: entries 2^20 apart share a bit
    v = 9_000_001
    z, idx, t, _, _ = _distill_inputs(1, v, 40, F32, False, 25)
    idx[0, 5], idx[0, 6], idx[0, 7] = 5, 5 + (1 << 20), 11
    lse = torch.logsumexp(t.masked_fill((idx < 0) | (idx >= v), -float("inf")), 1) + 0.2
    _distill_check(z, idx, t, lse, None, 1.0)
    _distill_check(z, idx, t, None, None, 1.0)


@pytest.mark.parametrize("v", [70000, 250000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distillation_logits_further_apart_than_an_exponential_reaches(v, dtype):
    # what a thread sees first says nothing about what comes later: sums of 2^((z - m) c) from its first logits overflow
    z, idx, t, _, _ = _distill_inputs(2, v, 6, dtype, False, 23)
    z[0, -300:] += 400.0
    z[1, v // 2] = 1000.0
    _distill_check(z, idx, t, None, None, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("v", [300, 40001])
def test_distillation_rows_with_nothing_to_learn(dtype, tail, v):
    z, idx, t, lse, w = _distill_inputs(5, v, 6, dtype, tail, 3)
    w[0], w[1] = 1.0, 0.0
    z[1] = NAN                       # weight zero: not read
    idx[2] = -1                      # no teacher entry
    t[3] = -float("inf")             # entries without mass
    z[3, 5], z[2, 7] = NAN, float("inf")
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, w)
    for i in (1, 2, 3):
        assert float(loss[i]) == 0 and bool((dz[i] == 0).all())
    want = lm.distill(_np(z[4:]), _np(idx[4:]), _np(t[4:]), _np(lse[4:]) if tail else None, _np(w[4:]), 1.0, dtype == BF16)
    _close(dz[4:], want["dz"], "dz")
    assert bool((ceca.dsgd_distill_loss(z, idx, t, lse, w)[1:4] == 0).all())
    none = torch.empty((5, 0), dtype=torch.int32, device=DEV)
    loss, dz = ceca.dsgd_distill_grad(z, none, torch.empty((5, 0), device=DEV), lse, None)
    assert bool((loss == 0).all()) and bool((dz == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("v", [64, 1001, 33000, 150001])
def test_distillation_with_masked_logits(dtype, tail, v):
    # a grammar mask: most of the vocabulary at -infinity, or at the type's lowest value
    z, idx, t, lse, w = _distill_inputs(4, v, 4, dtype, tail, 5)
    keep = torch.zeros((4, v), dtype=torch.bool, device=DEV)
    keep.scatter_(1, idx.long().clamp(0, v - 1), True)
    keep[:, 3] = True
    z[:2] = z[:2].masked_fill(~keep[:2], -float("inf"))
    z[2:] = z[2:].masked_fill(~keep[2:], torch.finfo(dtype).min)
    bf = dtype == BF16
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, None)
    # as if the masked entries were not there at all
    ref = z.float().masked_fill(~keep, -float("inf"))
    want = lm.distill(_np(ref), _np(idx), _np(t), _np(lse), None, 1.0, bf)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [50, 70001])
def test_distillation_of_a_row_masked_throughout_and_of_a_masked_target(dtype, v):
    z = torch.full((2, v), -float("inf"), dtype=dtype, device=DEV)
    z[1] = _randn((v,), dtype, 6)
    z[1, 4] = -float("inf")
    idx = torch.tensor([[3, 4], [4, 9]], dtype=torch.int32, device=DEV)
    t = torch.zeros((2, 2), device=DEV)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t)
    assert bool((loss == float("inf")).all())
    want = torch.zeros(v)
    want[3] = want[4] = -0.5
    assert torch.equal(dz[0].float().cpu(), want)
    ref = lm.distill(_np(z[1:]), _np(idx[1:]), _np(t[1:]), None, None, 1.0, dtype == BF16)
    _close(dz[1:], ref["dz"], "dz")


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("v", [40, 2000, 60001])
def test_distillation_entries_listed_twice(tail, v):
    z, idx, t, lse, w = _distill_inputs(3, v, 12, F32, False, 7)
    idx[0, 5:9] = 3
    idx[2, 0] = idx[2, 11] = 17
    if tail:
        here = (idx >= 0) & (idx < v)
        lse = torch.logsumexp(t.masked_fill(~here, -float("inf")), 1) + 0.1
    _distill_check(z, idx, t, lse, None, 1.0)


@pytest.mark.parametrize("v", [9, 2000, 48000])
def test_distillation_when_the_top_is_everything_or_the_mass_is_spent(v):
    g = _gen(11)
    z = torch.randn((2, v), generator=g).to(DEV)
    k = min(v, 2000)
    idx = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(2)]).to(torch.int32).to(DEV)
    t = torch.randn((2, k), generator=g).to(DEV)
    for lse in (torch.logsumexp(t, 1) + 0.3, torch.logsumexp(t, 1) - 0.1):   # mass with nowhere to go; more than one
        loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, None)
        want = lm.distill(_np(z), _np(idx), _np(t), _np(lse), None)
        _close(loss, want["loss"], "loss")
        _close(dz, want["dz"], "dz")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v,pad,oz,og", [(1000, 24, 0, 0), (1000, 1, 0, 0), (999, 0, 1, 1), (999, 0, 3, 5), (40003, 0, 1, 1), (40000, 8, 8, 0), (150001, 3, 2, 2)])
def test_distillation_strided_and_in_place(dtype, v, pad, oz, og):
    r, k = 5, 9
    src, idx, t, lse, w = _distill_inputs(r, v, k, dtype, True, 9)
    z, _ = _inside((r, v), (v + pad, 1), oz, dtype)
    z.copy_(src)
    wide = torch.full((r, k + 3), 1, dtype=torch.int32, device=DEV)
    wide[:, :k] = idx
    tw = torch.full((r, k + 2), NAN, device=DEV)
    tw[:, :k] = t
    dz, buf = _inside((r, v), (v + pad, 1), og, dtype)
    more = {"teacher_lse": lse, "weight": w}
    loss, _ = ceca.dsgd_distill_grad(z, wide[:, :k], tw[:, :k], dz=dz, **more)
    want = lm.distill(_np(src), _np(idx), _np(t), _np(lse), _np(w), 1.0, dtype == BF16)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    assert _untouched(dz, buf)
    _close(ceca.dsgd_distill_loss(z, idx, t, **more), want["loss"], "loss")
    _, same = ceca.dsgd_distill_grad(z, idx, t, dz=z, **more)
    assert same is z
    _close(z, want["dz"], "dz in place")


def test_distillation_rows_beyond_32_bit_offsets():
    r, v, ld = 3, 1000, 1 << 31
    buf = torch.empty(2 * ld + v, dtype=BF16, device=DEV)
    z = buf.as_strided((r, v), (ld, 1))
    src, idx, t, lse, w = _distill_inputs(r, v, 5, BF16, True, 13)
    z.copy_(src)
    loss, _ = ceca.dsgd_distill_grad(z, idx, t, lse, w, dz=z)
    want, dz = ceca.dsgd_distill_grad(src, idx, t, lse, w)
    assert torch.equal(loss, want) and torch.equal(z, dz)


def test_distillation_of_no_rows():
    z = torch.empty((0, 10), device=DEV)
    loss, dz = ceca.dsgd_distill_grad(z, torch.empty((0, 2), dtype=torch.int64, device=DEV), torch.empty((0, 2), device=DEV))
    assert loss.shape == (0,) and dz.shape == (0, 10)


@pytest.mark.parametrize("tail", [False, True])
def test_distillation_gradient_against_differences(tail):
    # central differences of the library's own loss along random directions; the loss is good to LOSS and the
    # third derivative along a direction of norm 1 is below 1, so the quotient is off by LOSS / h + h^2
    r, v, k, h = 4, 500, 6, 2e-2
    z, idx, t, lse, _ = _distill_inputs(r, v, k, F32, tail, 15)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse)
    off = lm.distill(_np(z), _np(idx), _np(t), _np(lse))["loss"][1].max()
    for s in range(4):
        u = _randn((r, v), F32, 100 + s)
        u /= u.norm(dim=1, keepdim=True)
        up, dn = (ceca.dsgd_distill_loss(z + c * u, idx, t, lse) for c in (h, -h))
        quot = _np(up - dn) / (2 * h)
        # z +- h u is rounded too: |z| U in every logit, through a gradient of norm below 2
        slip = float(z.abs().max()) * lm.U * 2 * np.sqrt(v) / h
        assert np.abs(quot - _np((dz * u).sum(1))).max() <= off / h + h * h + slip + 1e-5


# ------------------------------------------------------------------------------------------------ all of them


def test_operators_run_on_a_given_stream():
    s = torch.cuda.Stream()
    tok = _tokens(2, 60, 500, 1, torch.int32)
    E = _randn((2, 500, 64), F32, 2)
    x, f, h0, _ = _recur_inputs(2, 260, 64, BF16, True, False, 3)
    z, idx, t, lse, w = _distill_inputs(40, 3001, 8, BF16, True, 4)
    want_out = ceca.dsgd_embed_lookup(E, tok)
    want_dE = ceca.dsgd_embed_grad(want_out, tok, torch.empty_like(E))
    want_h, _, m = ceca.dsgd_recurrence(x, f, h0=h0, save=True)
    want_g = ceca.dsgd_recurrence_grad(x, f, want_h, m, h0=h0)
    want_l, want_dz = ceca.dsgd_distill_grad(z, idx, t, lse, w)
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        out = ceca.dsgd_embed_lookup(E, tok, stream=stream)
        dE = ceca.dsgd_embed_grad(out, tok, torch.empty_like(E), stream=stream)
        h, _, marks = ceca.dsgd_recurrence(x, f, h0=h0, save=True, stream=stream)
        g = ceca.dsgd_recurrence_grad(x, f, h, marks, h0=h0, stream=stream)
        loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, w, stream=stream)
        s.synchronize()
        assert torch.equal(out, want_out) and torch.equal(dE, want_dE) and torch.equal(h, want_h)
        assert all(torch.equal(a, b) for a, b in zip(g, want_g))
        assert torch.equal(loss, want_l) and torch.equal(dz, want_dz)


def test_operators_in_a_captured_graph():
    tok = _tokens(2, 60, 500, 1, torch.int32)
    E = _randn((2, 500, 64), F32, 2)
    x, f, h0, _ = _recur_inputs(1, 1300, 64, BF16, True, False, 3)
    z, idx, t, lse, w = _distill_inputs(40, 50001, 8, BF16, True, 4)

    def step():
        out = ceca.dsgd_embed_lookup(E, tok)
        dE = ceca.dsgd_embed_grad(out, tok, torch.empty_like(E))
        h, last, m = ceca.dsgd_recurrence(x, f, h0=h0, save=True)
        return (out, dE, h, last) + tuple(ceca.dsgd_recurrence_grad(x, f, h, m, h0=h0)) + tuple(ceca.dsgd_distill_grad(z, idx, t, lse, w))

    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
