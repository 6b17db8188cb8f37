"""The language-model operators at the edges of their range: NaN where it has to be seen, logits far apart or far from
zero, teachers whose mass is spent, arguments that have to be refused.  Bounds as in oracle/lm.py."""
import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import lm
from test_gpu_lm_operators import BF16, DEV, F32, NAN, _close, _distill_inputs, _gen, _np, _randn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ recurrence


@pytest.mark.parametrize("dtype,d", [(F32, 40), (BF16, 40), (BF16, 41)])   # every layout of the lanes
@pytest.mark.parametrize("t,at,cut", [(1, 0, None), (9, 4, 7), (40, 13, None), (40, 13, 14), (40, 13, 13), (300, 200, 260), (1500, 700, None), (1500, 700, 1200)])
@pytest.mark.parametrize("b", [1, 70])
def test_recurrence_a_gate_that_is_not_a_number_is_seen(dtype, d, t, at, cut, b):
    # sigmoid(NaN) is NaN: so are the states from there to the next document, and the gradients before
    if b > 1 and t > 300:
        pytest.skip("long sequences run as segments with few of them only")
    x, f, h0 = _randn((b, t, d), dtype, 1), _randn((b, t, d), dtype, 2, 1.0), _randn((b, d), F32, 3)
    dh, dl = _randn((b, t, d), dtype, 4), _randn((b, d), F32, 5)
    f[b - 1, at, 3], f[b - 1, at, d - 1] = NAN, NAN
    st = None
    if cut is not None:
        st = torch.zeros((b, t), dtype=torch.uint8, device=DEV)
        st[b - 1, cut] = 1
    h, last, marks = ceca.dsgd_recurrence(x, f, h0=h0, starts=st, save=True)
    want, _ = lm.recurrence(_np(x), _np(f), _np(h0), _np(st), dtype == BF16)
    assert np.isnan(want["h"][0][b - 1, at:cut if cut is None or cut > at else at + 1, 3]).all()
    _close(h, want["h"], "h")
    _close(last, want["last"], "last")
    dx, df, dh0 = ceca.dsgd_recurrence_grad(x, f, dh, marks, h0=h0, starts=st, dh_last=dl)
    want = lm.recurrence_grad(_np(x), _np(f), _np(dh), _np(h0), _np(st), _np(dl), dtype == BF16)
    for g, k in ((dx, "dx"), (df, "df"), (dh0, "dh0")):
        _close(g, want[k], k)


@pytest.mark.parametrize("lo,hi", [(-88.5, -86.5), (-104.0, -101.0), (14.0, 20.0), (86.5, 89.0)])
def test_recurrence_gates_of_every_number_where_they_are_next_to_zero_or_one(lo, hi):
    # every fp32 number of the range: neither gate leaves [0, 1], each is within its bound of the sigmoid
    ends = np.array(sorted((lo, hi), key=abs), np.float32).view(np.int32)
    f = torch.from_numpy(np.arange(ends[0], ends[1] + 1, dtype=np.int32).view(np.float32)).to(DEV).view(1, 1, -1)
    one = torch.ones_like(f)
    h, _, marks = ceca.dsgd_recurrence(one, f, save=True)   # 1 - a
    _, _, a = ceca.dsgd_recurrence_grad(one, f, one, marks)
    h, a, f64 = _np(h)[0, 0], _np(a)[0], _np(f)[0, 0]
    assert a.min() >= 0 and a.max() <= 1 and h.min() >= 0 and h.max() <= 1 + 4 * lm.U
    bound = lm.U * (12 + 2.4 * np.minimum(np.abs(f64), 90.0))
    want, rest = 1 / (1 + np.exp(-f64)), 1 / (1 + np.exp(f64))
    assert (np.abs(a - want) <= bound * want + 2.0 ** -124).all() and (np.abs(h - rest) <= bound * rest + 2.0 ** -124).all()
    if hi < 0:
        assert a.min() == 0 and h.min() >= 1 - 4 * lm.U   # shut for good, and open


# ------------------------------------------------------------------------------------------------ distillation

# a period and how much of its beginning is low: what the threads of one warp, of one CTA, of a cluster see first
APART = [(F32, 1000, 1000, 520), (F32, 3000, 3000, 1030), (BF16, 50000, 50000, 8200), (F32, 50000, 6252, 2100), (BF16, 400000, 50000, 8200)]


def _rows_apart(v, period, low, gaps, top, seed):
    """Rows of N(0, 1) whose first logits in every period lie `gap` below one logit of `top` in the middle of a period."""
    z = torch.randn((len(gaps), v), generator=_gen(seed))
    peak = (v // period // 2) * period + (low + period) // 2
    where = torch.arange(v) % period < low
    for i, gap in enumerate(gaps):
        z[i, where] += top - gap
        z[i, peak] = top
    return z, peak


@pytest.mark.parametrize("dtype,v,period,low", APART)
@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("top,alone", [(10.0, False), (10.0, True), (60.0, False)])
def test_distillation_whatever_the_threads_see_first(dtype, v, period, low, listed, top, alone):
    gaps = [40.0, 55.0, 62.0, 70.0] + [80.0 + 0.25 * i for i in range(61)] + [120.0, 300.0, 10000.0]
    if v > 100000:
        gaps = gaps[::4] + [87.5, 88.0, 88.25, 88.5]
    z, peak = _rows_apart(v, period, low, gaps, top, 31)
    r = len(gaps)
    idx = torch.stack([torch.randperm(v, generator=_gen(32 + i))[:5] for i in range(r)])
    idx[idx == peak] = 0
    if listed:
        idx[:, 2] = peak
    t = torch.randn((r, 5), generator=_gen(33)) + 2.0
    w = torch.full((r,), 1e-4)
    z, idx, t, w = z.to(dtype).to(DEV), idx.to(DEV), t.to(DEV), w.to(DEV)
    want = lm.distill(_np(z), _np(idx), _np(t), None, _np(w), 1.0, dtype == BF16)
    if alone:   # as many rows as the GPU needs to stream them, for the loss alone
        many = 700 // r + 1
        loss = ceca.dsgd_distill_loss(z.repeat(many, 1), idx.repeat(many, 1), t.repeat(many, 1), None, w.repeat(many))
        _close(loss, tuple(np.tile(a, many) for a in want["loss"]), "loss alone")
        return
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, None, w)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")


def _time_of(call, n=10):
    for _ in range(3):
        call()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    times = []
    for _ in range(n):
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return sorted(times)[n // 2]


@pytest.mark.parametrize("dtype,v", [(BF16, 32000), (F32, 128000), (F32, 8001)])
def test_distillation_a_finite_mask_costs_what_an_infinite_one_does(dtype, v):
    # an additive mask of -1e4 over most of the vocabulary, its first part included: a factor 2 leaves room for noise
    r, k = 2048, 8
    z = torch.randn((r, v), generator=_gen(41)).to(dtype).to(DEV)
    gone = torch.arange(v, device=DEV) % 4096 < 3800
    idx = (torch.arange(k, device=DEV) * 4096 % (v // 4096 * 4096) + 3900 + torch.arange(k, device=DEV)).expand(r, k).contiguous()
    t = torch.randn((r, k), generator=_gen(42)).to(DEV)
    out = torch.empty_like(z)
    hard, soft = z.masked_fill(gone, -float("inf")), torch.where(gone, z.float() - 1e4, z.float()).to(dtype)
    for a, b in zip(ceca.dsgd_distill_grad(hard[:9], idx[:9], t[:9]), ceca.dsgd_distill_grad(soft[:9], idx[:9], t[:9])):
        assert torch.equal(a, b)
    cost = [_time_of(lambda: ceca.dsgd_distill_grad(m, idx, t, dz=out)) for m in (hard, soft)]
    assert cost[1] <= 2 * cost[0], cost


@pytest.mark.parametrize("dtype,v", [(F32, 700), (F32, 33000), (BF16, 5000), (F32, 50001)])
@pytest.mark.parametrize("temperature", [0.2, 0.05, 0.01, 0.002])
def test_distillation_small_shares_at_low_temperatures(dtype, v, temperature):
    # q below the smallest normal number, over the temperature, is a gradient that is not
    z, idx, t, _, _ = _distill_inputs(4, v, 6, dtype, False, 45)
    T = float(np.float32(temperature))
    want = lm.distill(_np(z), _np(idx), _np(t * T), None, None, T, dtype == BF16)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t * T, None, None, T)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")


def _check_offset(dtype, v, tail, temperature, offset):
    z, idx, t, lse, w = _distill_inputs(4, v, 6, F32, tail, 51, F32, torch.int32, temperature)
    z = (z + offset).to(dtype)
    t = t * temperature   # (what the teacher sends for this temperature)
    if tail:
        here = (idx >= 0) & (idx < v)
        lse = torch.logsumexp((t.double() / float(np.float32(temperature))).masked_fill(~here, -float("inf")), 1).float() + 0.2
    T = float(np.float32(temperature))
    want = lm.distill(_np(z), _np(idx), _np(t), _np(lse), None, T, dtype == BF16)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, None, T)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    _close(ceca.dsgd_distill_loss(z, idx, t, lse, None, T), want["loss"], "loss alone")


OFFSET_SIZES = [(F32, 700), (F32, 3000), (F32, 33000), (F32, 50001), (BF16, 33000)]


@pytest.mark.parametrize("dtype,v", OFFSET_SIZES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("offset", [100.0, -100.0, 1e3, -1e3, 1e4, -1e4, 1e5, 1e7, -1e7, 9e7])
def test_distillation_of_logits_that_share_an_offset(dtype, v, tail, offset):
    _check_offset(dtype, v, tail, 1.0, offset)   # softmax does not know it


LOW = [(0.05, 1e3), (0.01, 3e5), (0.01, 1e6), (0.01, -1e6), (1e-5, 30.0), (1e-7, 30.0), (100.0, 1e9)]


@pytest.mark.parametrize("dtype,v", OFFSET_SIZES)
@pytest.mark.parametrize("temperature,offset", LOW)
def test_distillation_of_an_offset_at_a_low_temperature(dtype, v, temperature, offset):
    _check_offset(dtype, v, False, temperature, offset)   # which makes a large one of any


@pytest.mark.parametrize("dtype,v", [(F32, 900), (BF16, 50000), (F32, 50000), (F32, 300001), (F32, 2500001)])
@pytest.mark.parametrize("temperature", [1.0, 0.25, 0.1])
def test_distillation_outside_of_a_top_that_towers_over_it(dtype, v, temperature):
    # q0, the student's mass outside the top, is below what fp32 holds: its logarithm and its shares are not
    gaps = [20.0, 60.0, 80.0, 86.0, 87.0, 88.0, 90.0, 100.0, 104.0, 150.0, 300.0, 1000.0, -30.0, -95.0, -400.0]
    if v > 100000:
        gaps = gaps[::3]
    r = len(gaps)
    z = torch.randn((r, v), generator=_gen(61))
    idx = torch.stack([torch.randperm(v, generator=_gen(62 + i))[:4] for i in range(r)])
    z[torch.arange(r), idx[:, 1]] = torch.tensor(gaps)
    t = torch.randn((r, 4), generator=_gen(63)) * temperature
    idx[:, 3] = -1
    lse = torch.logsumexp(t[:, :3] / temperature, 1) + 0.3
    z, idx, t, lse = z.to(dtype).to(DEV), idx.to(DEV), t.to(DEV), lse.to(DEV)
    T = float(np.float32(temperature))
    want = lm.distill(_np(z), _np(idx), _np(t), _np(lse), None, T, dtype == BF16)
    assert np.isfinite(want["loss"][0]).all()
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, None, T)
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")
    _close(ceca.dsgd_distill_loss(z, idx, t, lse, None, T), want["loss"], "loss alone")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [600, 40000])
def test_distillation_outside_of_a_top_among_logits_far_from_zero(dtype, v):
    # the same where every logit is too far from zero for one multiplication by 1 / T
    r, base = 4, 3e8 if dtype == F32 else 2.0 ** 28
    step, temperatures = (32.0, (2.0, 0.5)) if dtype == F32 else (2.0 ** 21, (1.0, 0.25))   # the type's spacing there
    z = base + step * torch.randint(-3, 4, (r, v), generator=_gen(65)).float()
    idx = torch.stack([torch.randperm(v, generator=_gen(66 + i))[:4] for i in range(r)])
    z[torch.arange(r), idx[:, 0]] = base + 40 * step
    t = torch.randn((r, 4), generator=_gen(67))
    lse = (torch.logsumexp(t, 1) + 0.3).to(DEV)
    z, idx, t = z.to(dtype).to(DEV), idx.to(DEV), t.to(DEV)
    for e in (lse, None):
        for T in temperatures:
            want = lm.distill(_np(z), _np(idx), _np(t * T), _np(e), None, T, dtype == BF16)
            loss, dz = ceca.dsgd_distill_grad(z, idx, t * T, e, None, T)
            _close(loss, want["loss"], "loss")
            _close(dz, want["dz"], "dz")


@pytest.mark.parametrize("dtype,v", OFFSET_SIZES)
@pytest.mark.parametrize("temperature,offset", LOW)
def test_distillation_outside_of_a_top_at_a_low_temperature(dtype, v, temperature, offset):
    _check_offset(dtype, v, True, temperature, offset)


def _mass_inputs(v, teacher, more, r=5, k=6, seed=71):
    z, idx, t, _, _ = _distill_inputs(r, v, k, F32, False, seed)
    lse = torch.logsumexp(t.masked_fill((idx < 0) | (idx >= v), -float("inf")), 1)
    return z, idx, t.to(teacher), lse + more


@pytest.mark.parametrize("v", [300, 20001, 60001])
@pytest.mark.parametrize("teacher,more", [(F32, -0.05), (F32, -0.3), (F32, -2.0), (BF16, 0.0), (BF16, 0.002), (F32, 0.0), (F32, 1e-6)])
def test_distillation_gradient_where_the_top_holds_more_than_all_mass(v, teacher, more):
    # the listed mass exceeds 1 by the caller's teacher_lse, or by the rounding of logits that were sent in bf16
    z, idx, t, lse = _mass_inputs(v, teacher, more)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse)
    want = lm.distill(_np(z), _np(idx), _np(t), _np(lse))
    _close(loss, want["loss"], "loss")
    _close(dz, want["dz"], "dz")


@pytest.mark.parametrize("teacher,more", [(F32, -0.05), (F32, -0.3), (BF16, -0.01)])
def test_distillation_gradient_of_spent_mass_against_differences(teacher, more):
    # central differences of the library's own loss; off by its error over h and by a third derivative below the mass
    v, h = 500, 2e-2
    z, idx, t, lse = _mass_inputs(v, teacher, more)
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse)
    off = lm.distill(_np(z), _np(idx), _np(t), _np(lse))["loss"][1].max()
    for s in range(4):
        u = _randn(tuple(z.shape), F32, 100 + s)
        u[:, :3] += 8.0   # (a direction along which the gradient's sum would show)
        u /= u.norm(dim=1, keepdim=True)
        up, dn = (ceca.dsgd_distill_loss(z + c * u, idx, t, lse) for c in (h, -h))
        slip = float(z.abs().max()) * lm.U * 2 * np.sqrt(v) / h
        assert np.abs(_np(up - dn) / (2 * h) - _np((dz * u).sum(1))).max() <= off / h + 2 * h * h + slip + 1e-5
    # without a shift of all logits: the loss does not know it, so the gradient sums to nothing
    assert float(dz.double().sum(1).abs().max()) <= 1e-5


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [90, 20001, 60001])
def test_distillation_a_teacher_that_is_not_a_number_is_seen(dtype, v):
    z, idx, t, lse, _ = _distill_inputs(4, v, 5, dtype, True, 81)
    idx[:, 1:3] = torch.arange(2, device=DEV, dtype=idx.dtype)
    t[1, 0] = NAN
    lse[2] = NAN
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse)
    want = lm.distill(_np(z[::3]), _np(idx[::3]), _np(t[::3]), _np(lse[::3]), None, 1.0, dtype == BF16)
    _close(loss[::3], want["loss"], "loss")
    _close(dz[::3], want["dz"], "dz")
    assert bool(torch.isnan(loss[1:3]).all()) and bool(torch.isnan(dz[1:3].float()).all())
    # renormalised, a NaN spoils the entries; q, which is all there is elsewhere, has nothing to do with it
    loss, dz = ceca.dsgd_distill_grad(z, idx, t)
    inside = torch.zeros((v,), dtype=torch.bool, device=DEV)
    inside[idx[1][(idx[1] >= 0) & (idx[1] < v)].long()] = True
    assert bool(torch.isnan(loss[1])) and bool(torch.isnan(dz[1, inside].float()).all()) and bool(torch.isfinite(dz[1, ~inside].float()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("r,v", [(9, 700), (700, 5001), (40, 130001)])
def test_distillation_repeats_to_the_bit_beside_rows_that_are_not_numbers(dtype, tail, r, v):
    z, idx, t, lse, w = _distill_inputs(r, v, 6, dtype, tail, 91)
    z[3, 5], z[4, v - 1] = NAN, float("inf")
    bits = (lambda a: a.view(torch.int32)) if dtype == F32 else (lambda a: a.view(torch.int16))
    loss, dz = ceca.dsgd_distill_grad(z, idx, t, lse, w)
    assert bool(torch.isnan(loss[3:5]).all()) and bool(torch.isfinite(loss[5:]).all()) and bool(torch.isfinite(dz[5:].float()).all())
    only = ceca.dsgd_distill_loss(z, idx, t, lse, w)
    for _ in range(3):
        again, gz = ceca.dsgd_distill_grad(z, idx, t, lse, w)
        assert torch.equal(again.view(torch.int32), loss.view(torch.int32)) and torch.equal(bits(gz), bits(dz))
        assert torch.equal(ceca.dsgd_distill_loss(z, idx, t, lse, w).view(torch.int32), only.view(torch.int32))


@pytest.mark.parametrize("v", [500, 1000, 4000, 20000])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_distillation_gradient_is_good_to_fp32(v, tail, seed):
    # What makes the norm of dz are shares within a few binades of the largest: exponents below 8, off by 2^-22 ln 2 at most and by
    # half of that mostly, an exponential of 2 ulp, the sum's own error and two products: 4 U in the norm leaves room
    z, idx, t, lse, w = _distill_inputs(64, v, 8, F32, tail, 300 + seed)
    _, dz = ceca.dsgd_distill_grad(z, idx, t, lse, w)
    want = lm.distill(_np(z), _np(idx), _np(t), _np(lse), _np(w))["dz"][0]
    assert np.linalg.norm(_np(dz) - want) <= 4 * lm.U * np.linalg.norm(want)


# ------------------------------------------------------------------------------------------------ arguments


def test_a_workspace_with_gaps_is_refused():
    # its memory between the elements is not the call's
    tok = torch.zeros((1, 2000), dtype=torch.int32, device=DEV)
    dout, dE = torch.zeros((1, 2000, 16), device=DEV), torch.zeros((1, 50, 16), device=DEV)
    size = ceca.dsgd_embed_workspace_bytes(1, 2000, 50, 16)
    ws = torch.full((2 * size,), 77, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        ceca.dsgd_embed_grad(dout, tok, dE, workspace=ws[::2])
    x = torch.zeros((1, 5000, 16), device=DEV)
    size = ceca.dsgd_recurrence_workspace_bytes(1, 5000, 16)
    more = torch.full((2 * size,), 77, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        ceca.dsgd_recurrence(x, x, workspace=more[::2])
    marks = ceca.dsgd_recurrence(x, x, save=True)[2]
    with pytest.raises(ValueError):
        ceca.dsgd_recurrence_grad(x, x, x, marks, workspace=more[::2])
    torch.cuda.synchronize()
    assert bool((ws == 77).all()) and bool((more == 77).all())
