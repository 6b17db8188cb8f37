"""The operators around a model's blocks and behind its logits on the GPU against their 64-bit statements, element by element,
within the bounds that oracle/blocks.py derives for fp32 arithmetic (one more rounding for bf16 outputs)."""
import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import blocks

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


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


# ------------------------------------------------------------------------------------------------ 8 bits

KEEP = [(1, 1, 1), (2, 3, 31), (1, 5, 32), (3, 7, 33), (2, 129, 257), (1, 40, 1024), (4, 9, 100), (1, 3, 5001), (2, 17, 264), (1, 300, 2048), (1, 1, 40000)]


def _wide_range(shape, dtype, seed):
    """Values over many binades, with a tie to the even number, zeros and a block of nothing else."""
    x = torch.randn(shape, generator=_gen(seed)) * torch.exp(3 * torch.randn(shape, generator=_gen(seed + 1)))
    x[..., ::7] = torch.round(x[..., ::7] * 4) / 8
    x[0, 0] = 0
    return x.to(dtype).to(DEV)


@pytest.mark.parametrize("n,t,d", KEEP)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_keeping_in_8_bits_and_bringing_back(n, t, d, dtype):
    x = _wide_range((n, t, d), dtype, 3)
    kept = ceca.dsgd_keep8(x)
    assert np.array_equal(_np(kept), blocks.kept_bytes(_np(x)))
    want = blocks.kept(_np(x))[2]
    for back in (F32, BF16):
        assert np.array_equal(_np(ceca.dsgd_bring8(kept, d, back)), want)


def test_keeping_extreme_values():
    x = torch.zeros((1, 10, 64))
    x[0, 0, :4] = torch.tensor([3.4028e38, -3.4028e38, 1e38, 1.0])
    x[0, 1, :3] = torch.tensor([1e-45, 1.2e-38, -1.1754944e-38])
    x[0, 2, 3], x[0, 2, 40] = INF, 5.0
    x[0, 3, 3], x[0, 3, 40] = NAN, 5.0
    x[0, 4, 33], x[0, 4, 1] = -INF, -5.0
    x[0, 5, :5] = torch.tensor([127.5, -127.5, 126.5, 0.5, 1.5])
    x[0, 6, :2] = torch.tensor([2.0**-121, 2.0**-122])
    x[0, 7] = -0.0
    x[0, 8, 0] = 2.0**127
    kept = ceca.dsgd_keep8(x.to(DEV))
    assert np.array_equal(_np(kept), blocks.kept_bytes(_np(x)))
    got, want = _np(ceca.dsgd_bring8(kept, 64)), blocks.kept(_np(x))[2]
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(got[0, 2, :32]).all() and got[0, 2, 40] == 5


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,row", [(0, 80), (1, 80), (3, 77), (8, 72)])
def test_keeping_strided_tensors(dtype, offset, row):
    n, t, d = 3, 5, 70
    x, _ = _inside((n, t, d), (t * row + 9, row, 1), offset, dtype)
    x.copy_(_wide_range((n, t, d), dtype, 5))
    kept = ceca.dsgd_keep8(x)
    assert torch.equal(kept, ceca.dsgd_keep8(x.contiguous()))
    out, buf = _inside((n, t, d), (t * row + 9, row, 1), offset, dtype)
    assert ceca.dsgd_bring8(kept, d, x=out) is out
    assert torch.equal(out, ceca.dsgd_bring8(kept, d, dtype)) and _untouched(out, buf)
    across = x.transpose(0, 1)   # agents inside positions
    assert torch.equal(ceca.dsgd_keep8(across), kept.transpose(0, 1).contiguous())


def test_keeping_no_rows():
    assert ceca.dsgd_bring8(ceca.dsgd_keep8(torch.empty((2, 0, 9), device=DEV)), 9).shape == (2, 0, 9)


# ------------------------------------------------------------------------------------------------ block norms

TYPES = [(F32, F32, F32), (BF16, BF16, F32), (F32, BF16, BF16), (BF16, F32, F32)]   # stream, activations, weights
BLOCKS = [(1, 1, 1), (2, 3, 7), (1, 9, 64), (3, 5, 100), (2, 37, 256), (1, 130, 264), (4, 6, 771), (1, 33, 1024), (2, 11, 1032), (1, 300, 40), (2, 5, 2048), (1, 4, 2057),
          (1, 3, 4096), (1, 5, 4100), (2, 3, 8192), (1, 2, 8193), (1, 3, 10000)]


class Block:
    """Inputs of one call, of the given types, and the names that they go by in the statement."""

    def __init__(self, n, t, d, types, seed, gate=True, scale=True, parts="both"):
        s, a, w = types
        self.types, self.shape = types, (n, t, d)
        self.h, self.y = _randn((n, t, d), s, seed, 0.0, 2.0), _randn((n, t, d), a, seed + 1, 0.1, 0.7)
        self.gate = _randn((n, t, d), a, seed + 2, 0.3, 2.0) if gate else None
        self.w_pre, self.w_post = _randn((n, d), w, seed + 3, 1.0, 0.2), _randn((n, d), w, seed + 4, 1.0, 0.2)
        self.scale = _randn((n,), w, seed + 5, 0.5, 0.2) if scale else None
        self.du, self.dh_out = _randn((n, t, d), a, seed + 6), _randn((n, t, d), s, seed + 7)
        if parts == "no y":
            self.y = self.w_post = self.gate = self.scale = None
        if parts == "no w_pre":
            self.w_pre = self.du = None
        if t > 2:   # a row of nothing, and one of small values
            for x in (self.h, self.y):
                if x is not None:
                    x[0, 1] = 0
                    x[0, 2] *= 1e-4

    def run(self, act, **more):
        return ceca.dsgd_block_norm(self.h, self.y, self.w_pre, self.w_post, gate=self.gate, gate_act=act, scale=self.scale, **more)

    def want(self, act, eps):
        s, a, _ = self.types
        return blocks.block_norm(_np(self.h), _np(self.y), _np(self.w_pre), _np(self.w_post), _np(self.gate), act, _np(self.scale), np.float64(np.float32(eps)),
                                 s == BF16, a == BF16)

    def grad(self, act, src, stats, **more):
        h, y, gate = src
        more.setdefault("dh_out", self.dh_out)
        return ceca.dsgd_block_norm_grad(h, y, self.w_pre, self.w_post, stats, self.du, gate=gate, gate_act=act, scale=self.scale, **more)

    def want_grad(self, act, stats, kept=False, dh_out=True, before=None):
        s, a, w = self.types
        h, y, gate = (_np(x) for x in (self.h, self.y, self.gate))
        if kept:
            h, y, gate = (None if x is None else blocks.kept(x)[2] for x in (h, y, gate))
        return blocks.block_norm_grad(h, y, _np(self.w_pre), _np(self.w_post), _np(stats), _np(self.du), _np(self.dh_out) if dh_out else None, gate, act,
                                      _np(self.scale), s == BF16, a == BF16, w == BF16, before)


NAMES = ("dh", "dy", "dgate", "dw_pre", "dw_post", "dscale")


def _check_grad(got, want, types):
    s, a, w = types
    for k, g, ty in zip(NAMES, got, (s, a, a, w, w, w)):
        assert (g is None) == (k not in want), k
        if g is not None:
            assert g.dtype == ty, k
            _close(g, want[k], k)


@pytest.mark.parametrize("n,t,d", BLOCKS)
@pytest.mark.parametrize("types", TYPES)
def test_block_norm_and_gradient(n, t, d, types):
    act = (n + t + d) % 2
    b = Block(n, t, d, types, 11)
    eps = 1e-5
    h, u, stats, kept = b.run(act, eps=eps, save=True)
    assert kept is None and h.dtype == types[0] and u.dtype == types[1]
    want = b.want(act, eps)
    _close(h, want["h"], "h_out")
    _close(u, want["u"], "u")
    _close(stats, want["stats"], "stats")
    _check_grad(b.grad(act, (b.h, b.y, b.gate), stats), b.want_grad(act, stats), types)


@pytest.mark.parametrize("n,t,d", BLOCKS)
@pytest.mark.parametrize("types", TYPES[:3])
def test_block_norm_with_what_it_keeps_in_8_bits(n, t, d, types):
    act = (n + t) % 2
    b = Block(n, t, d, types, 23)
    plain = b.run(act, save=True)
    h, u, stats, kept = b.run(act, save=True, keep8=True)
    assert torch.equal(h, plain[0]) and torch.equal(u, plain[1]) and torch.equal(stats, plain[2])
    for k, x in zip(kept, (b.h, b.y, b.gate)):
        assert torch.equal(k, ceca.dsgd_keep8(x))
    _check_grad(b.grad(act, kept, stats), b.want_grad(act, stats, kept=True), types)


@pytest.mark.parametrize("d", [7, 256, 771, 2048, 9000])
@pytest.mark.parametrize("parts", ["no y", "no w_pre", "no gate", "no scale", "no dh_out"])
@pytest.mark.parametrize("keep", [False, True])
def test_block_norm_without_some_of_its_parts(d, parts, keep):
    n, t = 2, 19
    types = (F32, BF16, F32) if d % 2 else (BF16, BF16, F32)
    if parts == "no y":
        types = (types[0], types[0], F32)
    b = Block(n, t, d, types, 31, gate=parts != "no gate", scale=parts != "no scale", parts=parts)
    h, u, stats, kept = b.run(1, save=True, keep8=keep)
    want = b.want(1, 1e-6)
    if parts == "no y":
        assert h is b.h
    else:
        _close(h, want["h"], "h_out")
    assert (u is None) == (parts == "no w_pre")
    if u is not None:
        _close(u, want["u"], "u")
    _close(stats, want["stats"], "stats")
    src = kept if keep else (b.h, b.y, b.gate)
    more = {"dh_out": None, "dh": torch.empty(b.shape, dtype=types[0], device=DEV)} if parts == "no dh_out" else {}
    more |= {"dy": torch.empty(b.shape, dtype=types[1], device=DEV)} if parts == "no w_pre" and keep else {}
    if parts == "no w_pre" and keep:
        more |= {"dgate": torch.empty(b.shape, dtype=types[1], device=DEV)}
    _check_grad(b.grad(1, src, stats, **more), b.want_grad(1, stats, keep, parts != "no dh_out"), types)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("row,offset", [(80, 0), (83, 1), (72, 8), (77, 5)])
def test_block_norm_on_strided_tensors(types, row, offset):
    n, t, d = 3, 6, 72
    s, a, w = types
    b = Block(n, t, d, types, 41)
    c = Block(n, t, d, types, 41)
    outs = {}
    for k, ty in (("h", s), ("y", a), ("gate", a), ("du", a), ("dh_out", s)):
        x, _ = _inside((n, t, d), (t * row + 5, row, 1), offset, ty)
        x.copy_(getattr(b, k))
        setattr(b, k, x)
    X = torch.full((n, 500), NAN, dtype=w, device=DEV)   # weights as blocks of columns
    for k, at in (("w_pre", 3), ("w_post", 200)):
        X[:, at:at + d] = getattr(c, k)
        setattr(b, k, X[:, at:at + d])
    X[:, 0] = c.scale
    b.scale = X[:, 0]
    for k, ty in (("h_out", s), ("u", a), ("dh", s), ("dy", a), ("dgate", a)):
        outs[k] = _inside((n, t, d), (t * row + 5, row, 1), offset, ty)
    G = torch.full((n, 500), NAN, dtype=w, device=DEV)
    gw = {"dw_pre": G[:, 7:7 + d], "dw_post": G[:, 100:100 + d], "dscale": G[:, 499]}
    h, u, stats, kept = b.run(0, save=True, keep8=True, h_out=outs["h_out"][0], u=outs["u"][0])
    hc, uc, sc, kc = c.run(0, save=True, keep8=True)
    # (rows on other boundaries may be summed in another order: not the same bits)
    want = c.want(0, 1e-6)
    _close(h, want["h"], "h_out")
    _close(u, want["u"], "u")
    assert all(torch.equal(x, y) for x, y in zip(kept, kc))
    got = b.grad(0, (b.h, b.y, b.gate), stats, **{k: v[0] for k, v in outs.items() if k.startswith("d")}, **gw)
    _check_grad(got, c.want_grad(0, stats), types)
    for view, buf in outs.values():
        assert _untouched(view, buf)
    mark = torch.ones_like(G, dtype=torch.bool)
    for at in (slice(7, 7 + d), slice(100, 100 + d), slice(499, 500)):
        mark[:, at] = False
    assert torch.isnan(G[mark]).all() and not torch.isnan(G[~mark]).any()
    across = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.h, c.y, c.gate)]   # agents inside positions
    h2, u2, _, _ = ceca.dsgd_block_norm(across[0], across[1], c.w_pre, c.w_post, gate=across[2], scale=c.scale)
    assert torch.equal(h2, hc) and torch.equal(u2, uc)


@pytest.mark.parametrize("d", [96, 99, 9001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_block_norm_in_place(d, dtype):
    types = (dtype, dtype, F32)
    b = Block(2, 21, d, types, 51)
    src = [x.clone() for x in (b.h, b.y, b.gate)]
    h, u, stats, kept = b.run(1, save=True, keep8=True)
    want = b.grad(1, (b.h, b.y, b.gate), stats)
    h2, y2, g2 = (x.clone() for x in src)
    out = ceca.dsgd_block_norm(h2, y2, b.w_pre, b.w_post, gate=g2, gate_act=1, scale=b.scale, h_out=h2, u=y2, save=True, keep8=True)
    assert out[0] is h2 and torch.equal(h2, h) and torch.equal(y2, u) and torch.equal(out[2], stats) and all(torch.equal(x, y) for x, y in zip(out[3], kept))
    # over the inputs, and over the incoming gradients
    h3, y3, g3 = (x.clone() for x in src)
    got = ceca.dsgd_block_norm_grad(h3, y3, b.w_pre, b.w_post, stats, b.du, b.dh_out, gate=g3, gate_act=1, scale=b.scale, dh=h3, dy=y3, dgate=g3)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and got[0] is h3
    du, dh_out = b.du.clone(), b.dh_out.clone()
    got = ceca.dsgd_block_norm_grad(b.h, b.y, b.w_pre, b.w_post, stats, du, dh_out, gate=b.gate, gate_act=1, scale=b.scale, dh=dh_out, dy=du)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and got[0] is dh_out and got[1] is du


def test_block_norm_gradients_are_added_and_repeat_to_the_bit():
    b = Block(3, 700, 136, (F32, BF16, F32), 61)
    _, _, stats, _ = b.run(0, save=True)
    first = b.grad(0, (b.h, b.y, b.gate), stats)
    again = b.grad(0, (b.h, b.y, b.gate), stats)
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    before = {k: _randn(v.shape, F32, 70 + i) for i, (k, v) in enumerate(zip(NAMES[3:], first[3:]))}
    got = b.grad(0, (b.h, b.y, b.gate), stats, accumulate=True, **{k: v.clone() for k, v in before.items()})
    _check_grad(got, b.want_grad(0, stats, before={k: _np(v) for k, v in before.items()}), b.types)


def test_block_norm_of_no_rows():
    b = Block(2, 0, 40, (F32, F32, F32), 1)
    h, u, stats, kept = b.run(0, save=True, keep8=True)
    assert h.shape == (2, 0, 40) and stats.shape == (2, 0, 2) and kept[0].shape[1] == 0
    got = b.grad(0, (b.h, b.y, b.gate), stats)
    assert all((g == 0).all() for g in got[3:])


def test_block_norm_with_a_gradient_of_one_row_for_all():
    b = Block(2, 30, 200, (F32, BF16, F32), 71)
    _, _, stats, _ = b.run(0, save=True)
    b.du = b.du[:1, :1].expand(2, 30, 200)
    b.dh_out = b.dh_out[:1, :1].expand(2, 30, 200)
    got = b.grad(0, (b.h, b.y, b.gate), stats)
    _check_grad(got, b.want_grad(0, stats), b.types)


@pytest.mark.parametrize("d", [64, 101, 9000])
def test_block_norm_of_very_large_and_of_broken_rows(d):
    b = Block(1, 12, d, (F32, F32, F32), 81)
    b.y[0, 3] *= 1e25      # whose squares are beyond fp32
    b.h[0, 4] *= 1e30
    b.gate[0, 5, 0], b.gate[0, 5, 1] = 1e30, -1e30
    b.y[0, 6, 2] = NAN
    b.y[0, 7, 3] = INF
    b.gate[0, 8, 1] = NAN
    h, u, stats, _ = b.run(0, save=True)
    rows = [0, 1, 2, 3, 4, 5, 9, 10, 11]
    want = b.want(0, 1e-6)
    for got, k in ((h, "h"), (u, "u"), (stats, "stats")):
        _close(got[:, rows], tuple(x[:, rows] for x in want[k]), k)
    assert torch.isnan(h[0, 6]).all() and torch.isnan(u[0, 6]).all()
    assert torch.isnan(h[0, 7, 3]) and torch.isnan(u[0, 7]).all() and (stats[0, 7, 0] == 0)
    assert torch.isnan(h[0, 8, 1]) and torch.isnan(h[0, 8]).sum() == 1 and torch.isnan(u[0, 8]).all()
    got = b.grad(0, (b.h, b.y, b.gate), stats)
    wg = b.want_grad(0, stats)
    for g, k in zip(got[:3], NAMES):
        _close(g[:, rows], tuple(x[:, rows] for x in wg[k]), k)
        assert torch.isnan(g[0, 6]).all() and torch.isnan(g[0, 8, 1])


def test_block_norm_gradient_against_differences_of_the_library():
    # along a direction of norm 1 the third derivative is below 10 here; the loss is good to its bound over h
    n, t, d, h = 1, 4, 50, 2e-2
    b = Block(n, t, d, (F32, F32, F32), 91)
    b.y[0, 1], b.h[0, 1] = _randn((d,), F32, 1), _randn((d,), F32, 2)
    b.y[0, 2], b.h[0, 2] = _randn((d,), F32, 3), _randn((d,), F32, 4)
    _, _, stats, _ = b.run(1, save=True)
    got = dict(zip(NAMES, b.grad(1, (b.h, b.y, b.gate), stats)))

    def loss():
        ho, u, _, _ = b.run(1)
        want = b.want(1, 1e-6)
        off = (want["h"][1] * np.abs(_np(b.dh_out))).sum() + (want["u"][1] * np.abs(_np(b.du))).sum()
        return float((ho.double() * b.dh_out.double()).sum() + (u.double() * b.du.double()).sum()), off

    for i, (k, dk) in enumerate((("h", "dh"), ("y", "dy"), ("gate", "dgate"), ("w_pre", "dw_pre"), ("w_post", "dw_post"), ("scale", "dscale"))):
        keep = getattr(b, k)
        dirn = _randn(keep.shape, F32, 200 + i)
        dirn /= dirn.norm()
        setattr(b, k, keep + h * dirn)
        up, off = loss()
        setattr(b, k, keep - h * dirn)
        down, _ = loss()
        setattr(b, k, keep)
        slip = float(keep.abs().max()) * 2.0**-24 * float(got[dk].abs().sum()) / h   # keep +- h dirn is rounded too
        assert abs((up - down) / (2 * h) - float((got[dk].double() * dirn.double()).sum())) <= off / h + 10 * h * h + slip


# ------------------------------------------------------------------------------------------------ tokens and losses

LOGITS = [(1, 1), (2, 2), (3, 7), (70, 33), (5, 1000), (200, 501), (40, 4099), (33, 6001), (3, 50001), (600, 2050), (7, 32000), (2, 200000)]


def _logits(r, v, dtype, seed, it=torch.int64):
    z = _randn((r, v), dtype, seed, 0.0, 2.0)
    tok = torch.randint(0, v, (r,), generator=_gen(seed + 1))
    z[torch.arange(r, device=DEV), tok.to(DEV)] += 3.0
    if r > 4:
        tok[2], tok[4] = -1, v
    if r > 6 and it == torch.int64:
        tok[6] = 2**32 + 1   # not token 1
    return z, tok.to(it).to(DEV)


def _policy_inputs(r, v, dtype, temperature, seed, it=torch.int64):
    z, tok = _logits(r, v, dtype, seed, it)
    lp = torch.from_numpy(blocks.token_logprob(_np(z), _np(tok), temperature)[0])
    g = _gen(seed + 2)
    moved = 0.3 * torch.randn(r, generator=g)
    for corner in (np.log(0.8), np.log(1.3)):   # off the corners of the clipping, where either side is right
        moved = torch.where((moved - corner).abs() < 1e-3, moved + 4e-3, moved)
    old, ref = (lp - moved).float(), (lp + 0.4 * torch.randn(r, generator=g)).float()
    adv, w = torch.randn(r, generator=g), torch.rand(r, generator=g) + 0.1
    if r > 3:
        w[1] = 0
        old[1] = ref[1] = NAN   # not looked at
        z[1] = NAN
    return (z, tok) + tuple(x.to(DEV) for x in (old, adv, ref, w))


@pytest.mark.parametrize("r,v", LOGITS)
@pytest.mark.parametrize("dtype,it,temperature", [(F32, torch.int64, 1.0), (BF16, torch.int32, 0.7)])
def test_log_probabilities(r, v, dtype, it, temperature):
    z, tok = _logits(r, v, dtype, 5, it)
    _close(ceca.dsgd_token_logprob(z, tok, temperature), blocks.token_logprob(_np(z), _np(tok), np.float64(np.float32(temperature))), "logp")


@pytest.mark.parametrize("r,v", LOGITS)
@pytest.mark.parametrize("dtype,it,temperature,kl", [(F32, torch.int64, 1.0, 0.1), (BF16, torch.int32, 0.7, 0.0), (F32, torch.int32, 2.0, 0.0), (BF16, torch.int64, 1.0, 0.5)])
def test_policy_loss_and_gradient(r, v, dtype, it, temperature, kl):
    temp = np.float64(np.float32(temperature))
    z, tok, old, adv, ref, w = _policy_inputs(r, v, dtype, temp, 7, it)
    kw = dict(ref_logp=ref if kl else None, weight=w, temperature=temperature, clip_low=0.2, clip_high=0.3, kl=kl)
    logp = torch.full((r,), NAN, device=DEV)
    loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, logp=logp, **kw)
    want = blocks.policy(_np(z), _np(tok), _np(old), _np(adv), _np(ref) if kl else None, _np(w), temp, 0.2, 0.3, np.float64(np.float32(kl)), dtype == BF16)
    assert dz.dtype == dtype
    _close(loss, want["loss"], "loss")
    _close(logp, want["logp"], "logp")
    _close(dz, want["dz"], "dz")
    _close(ceca.dsgd_policy_loss(z, tok, old, adv, **kw), want["loss"], "loss alone")


@pytest.mark.parametrize("r,v,ld", [(4800, 60, 60), (4801, 203, 203), (4739, 500, 504), (4736, 2040, 2040), (4740, 900, 901), (5001, 13, 13)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_losses_of_many_short_rows(r, v, ld, dtype):
    src, tok, old, adv, ref, w = _policy_inputs(r, v, dtype, 1.0, 41)
    for row, x in ((9, NAN), (10, INF), (11, -INF), (3000, 2.0**100)):   # rows that take the slow way, beside others
        src[row, ::2] = x
    z, _ = _inside((r, v), (ld, 1), 0, dtype)
    z.copy_(src)
    out, buf = _inside((r, v), (ld, 1), 0, dtype)
    kw = dict(ref_logp=ref, weight=w, kl=0.1, clip_high=0.3)
    loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, dz=out, **kw)
    want = blocks.policy(_np(src), _np(tok), _np(old), _np(adv), _np(ref), _np(w), high=0.3, kl=np.float64(np.float32(0.1)), bf16=dtype == BF16)
    fine = np.isfinite(want["loss"][0])
    for i in (9, 10, 11, 3000):   # (the ratio was made for other logits)
        fine[i] = False
    ok = torch.from_numpy(fine).to(DEV)
    _close(loss[ok], tuple(x[fine] for x in want["loss"]), "loss")
    _close(dz[ok], tuple(x[fine] for x in want["dz"]), "dz")
    assert _untouched(out, buf)
    _close(ceca.dsgd_token_logprob(z, tok), blocks.token_logprob(_np(src), _np(tok)), "logp")
    bounds = [0, r // 3, r // 2, r // 2 + 1, r - 5]
    tok2 = tok.clone()
    tok2[[9, 10, 11, 1]] = -1
    got = ceca.dsgd_preference_grad(z, tok2, torch.tensor(bounds, device=DEV), average=True)
    want = blocks.preference(_np(src), _np(tok2), bounds, average=True, bf16=dtype == BF16, beta=np.float64(np.float32(0.1)))
    for g, k in zip(got, ("loss", "logp", "dz")):
        _close(g, want[k], k)
    same = z.clone() if ld == v else None
    if same is not None:
        l2, d2 = ceca.dsgd_policy_grad(same, tok, old, adv, dz=same, **kw)
        assert torch.equal(l2.nan_to_num(), loss.nan_to_num()) and torch.equal(d2.nan_to_num(), dz.nan_to_num())


PAIRS = [  # r, v, bounds
    (2, 5, [0, 1, 2]), (40, 33, [0, 7, 7, 20, 38]), (300, 501, [3, 100, 180, 180, 290]), (64, 4099, [0, 30, 64]), (12, 50001, [0, 5, 12]),
    (700, 2050, [0, 100, 230, 300, 460, 600, 690]), (9, 7, [0, 0, 0, 4, 9]), (30, 32000, [0, 10, 29]),
]


def _pair_inputs(r, v, bounds, dtype, seed, average=False, it=torch.int64):
    z, tok = _logits(r, v, dtype, seed, it)
    tok[: max(1, r // 9)] = -1
    b = torch.tensor(bounds, dtype=torch.int32 if it == torch.int64 else torch.int64, device=DEV)
    out = blocks.preference(_np(z), _np(tok), bounds, average=average)
    ref = (torch.from_numpy(out["logp"][0]) + torch.randn(len(bounds) - 1, generator=_gen(seed + 9))).float().to(DEV)
    w = (torch.rand(len(bounds) // 2, generator=_gen(seed + 3)) + 0.5).to(DEV)
    return z, tok, b, ref, w


@pytest.mark.parametrize("r,v,bounds", PAIRS)
@pytest.mark.parametrize("dtype,it,average,smoothing", [(F32, torch.int64, False, 0.0), (BF16, torch.int32, True, 0.1), (F32, torch.int32, True, 0.0), (BF16, torch.int64, False, 0.3)])
def test_preference_loss_and_gradient(r, v, bounds, dtype, it, average, smoothing):
    temp = 1.0 if average else 1.25
    z, tok, b, ref, w = _pair_inputs(r, v, bounds, dtype, 13, average, it)
    kw = dict(ref_logp=ref, weight=w, temperature=temp, beta=0.5, smoothing=smoothing, average=average)
    loss, logp, dz = ceca.dsgd_preference_grad(z, tok, b, **kw)
    want = blocks.preference(_np(z), _np(tok), bounds, _np(ref), _np(w), temp, 0.5, np.float64(np.float32(smoothing)), average, dtype == BF16)
    for got, k in ((loss, "loss"), (logp, "logp"), (dz, "dz")):
        _close(got, want[k], k)
    again = ceca.dsgd_preference_loss(z, tok, b, **kw)
    _close(again[0], want["loss"], "loss alone")
    _close(again[1], want["logp"], "logp alone")
    bare = ceca.dsgd_preference_grad(z, tok, b)
    want = blocks.preference(_np(z), _np(tok), bounds, bf16=dtype == BF16, beta=np.float64(np.float32(0.1)))
    for got, k in zip(bare, ("loss", "logp", "dz")):
        _close(got, want[k], k)


def test_preference_bounds_beyond_the_rows_and_pairs_of_weight_zero():
    r, v = 20, 300
    z, tok, _, _, _ = _pair_inputs(r, v, [0, 5, 12], F32, 17)
    b = torch.tensor([-7, 5, 9, 15, 99], device=DEV)
    w = torch.tensor([1.0, 0.0], device=DEV)
    loss, logp, dz = ceca.dsgd_preference_grad(z, tok, b, weight=w)
    want = blocks.preference(_np(z), _np(tok), [0, 5, 9, 15, 20], weight=_np(w), beta=np.float64(np.float32(0.1)))
    for got, k in ((loss, "loss"), (logp, "logp"), (dz, "dz")):
        _close(got, want[k], k)
    assert (dz[9:] == 0).all() and loss[1] == 0
    none = ceca.dsgd_preference_grad(z, tok, b[:1])
    assert none[0].shape == (0,) and none[1].shape == (0,) and (none[2] == 0).all()


def test_preference_of_sequences_far_apart():
    # margins of hundreds: the loss is the margin on one side and e^-margin on the other, where the slope may underflow
    r, v = 40, 64
    z, tok = _logits(r, v, F32, 19)
    b = torch.tensor([0, 20, 40], device=DEV)
    for ref in ([0.0, 900.0], [900.0, 0.0], [0.0, 60.0], [1e6, 0.0]):
        ref = torch.tensor(ref, device=DEV)
        got = ceca.dsgd_preference_grad(z, tok, b, ref_logp=ref, beta=1.0)
        want = blocks.preference(_np(z), _np(tok), [0, 20, 40], _np(ref), beta=1.0)
        for g, k in zip(got, ("loss", "logp", "dz")):
            _close(g, want[k], k)


ROWS = ["offset", "far offset", "masked", "all masked", "only the token", "the token masked", "sure", "unsure", "nan", "inf", "own inf", "large", "low mask", "far apart"]


def _odd_row(kind, v, tok, seed, dtype):
    z = _randn((v,), F32, seed).cpu()
    z[tok] += 1
    if kind == "offset":
        z += 1000
    elif kind == "far offset":
        z = torch.round(z * 4) * 2.0**28
    elif kind == "masked":
        z[torch.arange(v) % 3 != 0] = -INF
        z[tok] = 0.5
    elif kind == "all masked":
        z[:] = -INF
    elif kind == "only the token":
        z[torch.arange(v) != tok] = -INF
    elif kind == "the token masked":
        z[tok] = -INF
    elif kind == "sure":
        z[tok] = 40
    elif kind == "unsure":
        z[tok] = -60
    elif kind == "nan":
        z[(tok + 1) % v] = NAN
    elif kind == "inf":
        z[(tok + 1) % v] = INF
    elif kind == "own inf":
        z[tok] = INF
    elif kind == "large":
        z = torch.where(torch.arange(v) == tok, 3e38, -3e38)
    elif kind == "low mask":
        z[torch.arange(v) % 5 != 0] = torch.finfo(dtype).min
        z[tok] = 0.25
    elif kind == "far apart":
        z[torch.arange(v) % 2 == 0] -= 1e4
    return z.to(dtype)


@pytest.mark.parametrize("v", [9, 1003, 40000, 131072])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_odd_logits(v, dtype):
    tok = torch.tensor([(37 * i) % v for i in range(len(ROWS))])
    z = torch.stack([_odd_row(k, v, int(t), 100 + i, dtype) for i, (k, t) in enumerate(zip(ROWS, tok))]).to(DEV)
    tok = tok.to(DEV)
    r = len(ROWS)
    lp = ceca.dsgd_token_logprob(z, tok)
    want = blocks.token_logprob(_np(z), _np(tok))
    _close(lp, want, "logp")
    old = torch.where(torch.isfinite(lp), lp, -1.0).contiguous()
    adv = -torch.ones(r, device=DEV)
    loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, clip_low=1.0)
    want = blocks.policy(_np(z), _np(tok), _np(old), _np(adv), low=1.0, bf16=dtype == BF16)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    # the same rows as sequences of one
    odd = torch.arange(r + 1, device=DEV)
    got = ceca.dsgd_preference_grad(z, tok, odd, smoothing=0.5)
    want = blocks.preference(_np(z), _np(tok), list(range(r + 1)), smoothing=0.5, bf16=dtype == BF16, beta=np.float64(np.float32(0.1)))
    good = np.isfinite(want["loss"][0])
    _close(got[0][torch.from_numpy(good).to(DEV)], tuple(x[good] for x in want["loss"]), "loss")
    good = np.repeat(good, 2)
    _close(got[2][torch.from_numpy(good).to(DEV)], tuple(x[good] for x in want["dz"]), "dz")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,ld", [(0, 1008), (1, 1003), (3, 1001), (5, 1007)])
def test_losses_on_strided_logits_and_in_place(dtype, offset, ld):
    r, v = 50, 1001
    src, tok, old, adv, ref, w = _policy_inputs(r, v, dtype, 1.0, 23)
    z, buf = _inside((r, v), (ld, 1), offset, dtype)
    z.copy_(src)
    bounds = [0, 20, 45]
    b = torch.tensor(bounds, device=DEV)
    out, obuf = _inside((r, v), (ld, 1), offset, dtype)
    kw = dict(ref_logp=ref, weight=w, kl=0.2, clip_high=0.3)
    loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, dz=out, **kw)
    want = blocks.policy(_np(src), _np(tok), _np(old), _np(adv), _np(ref), _np(w), high=0.3, kl=np.float64(np.float32(0.2)), bf16=dtype == BF16)
    assert dz is out and _untouched(out, obuf)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    z[1] = 0
    src[1] = 0
    pl, _, pz = ceca.dsgd_preference_grad(z, tok, b, dz=out)
    pw = blocks.preference(_np(src), _np(tok), bounds, bf16=dtype == BF16, beta=np.float64(np.float32(0.1)))
    _close(pl, pw["loss"], "preference loss")
    _close(pz, pw["dz"], "preference dz")
    assert _untouched(out, obuf)
    if ld % 8 == 0:
        _, dense = ceca.dsgd_preference_grad(src, tok, b)[1:]
        _close(dense, pw["dz"], "dense")
    _, _, same = ceca.dsgd_preference_grad(z, tok, b, dz=z)
    assert same is z and torch.equal(z, out) and _untouched(z, buf)
    z.copy_(src)
    _, first = ceca.dsgd_policy_grad(z, tok, old, adv, **kw)
    _, second = ceca.dsgd_policy_grad(z, tok, old, adv, dz=z, **kw)
    assert torch.equal(first, second) and _untouched(z, buf)


def test_losses_repeat_to_the_bit():
    z, tok, old, adv, ref, w = _policy_inputs(90, 70001, BF16, 1.0, 29)
    z[1] = 0
    b = torch.tensor([0, 20, 45, 60, 90], device=DEV)
    first = ceca.dsgd_policy_grad(z, tok, old, adv, ref_logp=ref, kl=0.1) + ceca.dsgd_preference_grad(z, tok, b) + (ceca.dsgd_token_logprob(z, tok),)
    for _ in range(3):
        again = ceca.dsgd_policy_grad(z, tok, old, adv, ref_logp=ref, kl=0.1) + ceca.dsgd_preference_grad(z, tok, b) + (ceca.dsgd_token_logprob(z, tok),)
        assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(first, again))


def test_losses_of_no_rows():
    z, tok, f = torch.empty((0, 10), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    assert ceca.dsgd_token_logprob(z, tok).shape == (0,)
    assert ceca.dsgd_policy_grad(z, tok, f, f)[1].shape == (0, 10)
    loss, logp, dz = ceca.dsgd_preference_grad(z, tok, torch.zeros(3, dtype=torch.int64, device=DEV))
    assert abs(float(loss) - np.log(2)) < 1e-6 and (logp == 0).all() and dz.shape == (0, 10)


# ------------------------------------------------------------------------------------------------ all of them


def _step(b, z, tok, old, adv, bounds):
    h, u, stats, kept = b.run(1, save=True, keep8=True)
    x8 = ceca.dsgd_keep8(u)
    grads = b.grad(1, kept, stats)
    return (h, u, stats, ceca.dsgd_bring8(x8, u.shape[2], u.dtype)) + tuple(grads) + (ceca.dsgd_token_logprob(z, tok),) + tuple(
        ceca.dsgd_policy_grad(z, tok, old, adv)) + tuple(ceca.dsgd_preference_grad(z, tok, bounds))


@pytest.fixture(scope="module")
def whole():
    b = Block(2, 70, 264, (F32, BF16, F32), 101)
    z, tok, old, adv, _, _ = _policy_inputs(60, 9001, BF16, 1.0, 37)
    z[1] = 0
    old[1] = -9
    return b, z, tok, old, adv, torch.tensor([0, 20, 60], device=DEV)


def test_operators_run_on_a_given_stream(whole):
    b, z, tok, old, adv, bounds = whole
    want = _step(*whole)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        h, u, stats, kept = b.run(1, save=True, keep8=True, stream=stream)
        back = ceca.dsgd_bring8(ceca.dsgd_keep8(u, stream=stream), 264, u.dtype, stream=stream)
        got = (h, u, stats, back) + tuple(b.grad(1, kept, stats, stream=stream)) + (ceca.dsgd_token_logprob(z, tok, stream=stream),) + tuple(
            ceca.dsgd_policy_grad(z, tok, old, adv, stream=stream)) + tuple(ceca.dsgd_preference_grad(z, tok, bounds, stream=stream))
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_operators_in_a_captured_graph(whole):
    want = _step(*whole)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(*whole)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_calls_on_two_streams_at_once(whole):
    want = _step(*whole)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(_step(*whole))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))


# ------------------------------------------------------------------------------------------------ edges


def test_offsets_past_32_bits_in_rows():
    # 2.2e9 channels: the last rows are those of a small call on the same rows
    t, d, last = 530001, 4104, 5
    g = torch.Generator(DEV).manual_seed(1)

    def big(seed):
        x = torch.empty((1, t, d), dtype=BF16, device=DEV)
        x[:, :1000].normal_(generator=g)
        x[:, 1000:530000].view(529, 1000, d).copy_(x[:, :1000].expand(529, 1000, d))
        x[:, -last:].normal_(generator=g)
        return x

    h, y, a = (big(i) for i in range(3))
    w, s = _randn((1, d), F32, 5, 1.0, 0.1), _randn((1,), F32, 6)
    ho, u, stats, kept = ceca.dsgd_block_norm(h, y, w, w, gate=a, scale=s, save=True, keep8=True)
    end = [x[:, -last:].contiguous() for x in (h, y, a)]
    small = ceca.dsgd_block_norm(end[0], end[1], w, w, gate=end[2], scale=s, save=True, keep8=True)
    assert torch.equal(ho[:, -last:], small[0]) and torch.equal(u[:, -last:], small[1]) and torch.equal(stats[:, -last:], small[2])
    assert all(torch.equal(x[:, -last:], z) for x, z in zip(kept, small[3]))
    du, dho = a, y
    for src, few in (((h, y, a), end), (kept, small[3])):
        got = ceca.dsgd_block_norm_grad(src[0], src[1], w, w, stats, du, dho, gate=src[2], scale=s)
        want = ceca.dsgd_block_norm_grad(few[0], few[1], w, w, small[2], end[2], end[1], gate=few[2], scale=s)
        assert all(torch.equal(x[:, -last:], z) for x, z in zip(got[:3], want[:3]))
        del got
    k = ceca.dsgd_keep8(u)
    assert torch.equal(k[:, -last:], ceca.dsgd_keep8(small[1]))
    assert torch.equal(ceca.dsgd_bring8(k, d, BF16)[:, -last:], ceca.dsgd_bring8(k[:, -last:].contiguous(), d, BF16))


def test_offsets_past_32_bits_in_logits():
    r, v, last = 16700, 131073, 6
    z = torch.empty((r, v), dtype=BF16, device=DEV)
    z[:200].normal_(generator=torch.Generator(DEV).manual_seed(2))
    for i in range(200, r, 200):
        z[i:i + 200].copy_(z[:min(200, r - i)])
    z[-last:].normal_(generator=torch.Generator(DEV).manual_seed(3))
    tok = torch.randint(0, v, (r,), generator=_gen(4)).to(DEV)
    adv, old = _randn((r,), F32, 5), torch.full((r,), -11.0, device=DEV)
    end, few = z[-last:].clone(), tok[-last:].clone()
    assert torch.equal(ceca.dsgd_policy_grad(z, tok, old, adv)[1][-last:], ceca.dsgd_policy_grad(end, few, old[-last:].clone(), adv[-last:].clone())[1])
    want = blocks.token_logprob(_np(end), _np(few))
    _close(ceca.dsgd_token_logprob(z, tok)[-last:], want, "logp")
    b = torch.tensor([0, r - last, r - last + 2, r - 3, r], device=DEV)
    dz = ceca.dsgd_preference_grad(z, tok, b, average=True)[2]
    small = blocks.preference(_np(end), _np(few), [0, 0, 2, 3, 6], average=True, bf16=True, beta=np.float64(np.float32(0.1)))
    _close(dz[-4:], tuple(x[-4:] for x in small["dz"]), "dz")   # the second pair


@pytest.mark.parametrize("temperature", [1e-3, 0.05, 30.0, 1e4])
@pytest.mark.parametrize("v", [300, 20000])
def test_losses_at_other_temperatures(temperature, v):
    r, temp = 30, np.float64(np.float32(temperature))
    z, tok = _logits(r, v, F32, 51)
    z *= min(1.0, temperature * 10)   # (what a policy at that temperature has learnt)
    lp = torch.from_numpy(blocks.token_logprob(_np(z), _np(tok), temp)[0])
    old, adv = (lp - 0.1).float().to(DEV), _randn((r,), F32, 52)
    loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, temperature=temperature)
    want = blocks.policy(_np(z), _np(tok), _np(old), _np(adv), temperature=temp)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    got = ceca.dsgd_preference_grad(z, tok, torch.tensor([0, 11, 30], device=DEV), temperature=temperature)
    want = blocks.preference(_np(z), _np(tok), [0, 11, 30], temperature=temp, beta=np.float64(np.float32(0.1)))
    for g, k in zip(got, ("loss", "logp", "dz")):
        _close(g, want[k], k)


def test_many_agents_of_few_rows():
    n, t, d = 3000, 2, 40
    b = Block(n, t, d, (F32, F32, F32), 61)
    h, u, stats, kept = b.run(1, save=True, keep8=True)
    want = b.want(1, 1e-6)
    _close(h, want["h"], "h_out")
    _close(u, want["u"], "u")
    _check_grad(b.grad(1, kept, stats), b.want_grad(1, stats, kept=True), b.types)


@pytest.mark.parametrize("d", [1, 8, 31, 33, 56, 64, 65, 72, 104, 127, 128])
@pytest.mark.parametrize("types", TYPES)
def test_block_norm_of_narrow_rows(d, types):
    # several rows a warp, of which some have a row less than others; one that overflows beside others that do not
    n, t = 2, 1000 if d % 3 else 37
    b = Block(n, t, d, types, 111)
    if types[1] == F32:
        b.y[0, 5] *= 1e25
        b.y[1, t - 1] *= 1e25
    for keep in (False, True):
        h, u, stats, kept = b.run(1, save=True, keep8=keep)
        want = b.want(1, 1e-6)
        for got, k in ((h, "h"), (u, "u"), (stats, "stats")):
            _close(got, want[k], k)
        if keep:
            assert all(torch.equal(k, ceca.dsgd_keep8(x)) for k, x in zip(kept, (b.h, b.y, b.gate)))
        _check_grad(b.grad(1, kept if keep else (b.h, b.y, b.gate), stats), b.want_grad(1, stats, kept=keep), types)


def test_block_norm_outputs_over_other_inputs():
    # u over the gate, dy over the gate, dgate over y: each element is read before it is written
    for d in (96, 99, 9000):
        b = Block(2, 13, d, (BF16, BF16, F32), 71)
        h, u, stats, _ = b.run(0, save=True)
        g = b.gate.clone()
        ho, uo, _, _ = ceca.dsgd_block_norm(b.h, b.y, b.w_pre, b.w_post, gate=g, scale=b.scale, u=g)
        assert uo is g and torch.equal(ho, h) and torch.equal(g, u)
        want = b.grad(0, (b.h, b.y, b.gate), stats)
        y, g = b.y.clone(), b.gate.clone()
        got = ceca.dsgd_block_norm_grad(b.h, y, b.w_pre, b.w_post, stats, b.du, b.dh_out, gate=g, scale=b.scale, dy=g, dgate=y)
        assert all(torch.equal(x, z) for x, z in zip(got, want))


def test_one_tensor_in_several_places():
    # h, y and the gate may be one tensor, as inputs
    x = _randn((2, 9, 128), F32, 81)
    w = _randn((2, 128), F32, 82)
    got = ceca.dsgd_block_norm(x, x, w, w, gate=x, save=True)
    want = ceca.dsgd_block_norm(x.clone(), x.clone(), w, w, gate=x.clone(), save=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_given_workspace_is_kept_to():
    b = Block(2, 50, 200, (F32, F32, F32), 91)
    _, _, stats, _ = b.run(0, save=True)
    size = ceca.dsgd_block_norm_workspace_bytes(2, 50, 200)
    ws = torch.full((size + 256,), 7, dtype=torch.uint8, device=DEV)
    want = b.grad(0, (b.h, b.y, b.gate), stats)
    got = b.grad(0, (b.h, b.y, b.gate), stats, workspace=ws[:size])
    assert all(torch.equal(x, z) for x, z in zip(got, want)) and (ws[size:] == 7).all()
    z, tok = _logits(900, 33000, BF16, 92)
    size = ceca.dsgd_token_workspace_bytes(900, 33000, 2)
    ws = torch.full((size + 256,), 7, dtype=torch.uint8, device=DEV)
    bounds = torch.tensor([0, 100, 300, 301, 880], device=DEV)
    want = ceca.dsgd_preference_grad(z, tok, bounds)
    got = ceca.dsgd_preference_grad(z, tok, bounds, workspace=ws[:size])
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and (ws[size:] == 7).all()
    size = ceca.dsgd_token_workspace_bytes(900, 33000)
    assert torch.equal(ceca.dsgd_token_logprob(z, tok, workspace=ws[:size]), ceca.dsgd_token_logprob(z, tok))
