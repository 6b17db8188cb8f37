"""The operators around a model's blocks and behind its logits at the edges of their range: workspaces to the byte, gates and logits far out, rows
without a token beside rows of NaN.  Bounds as in oracle/blocks.py."""
import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import blocks
from test_gpu_block_operators import BF16, DEV, F32, INF, NAMES, NAN, TYPES, Block, _check_grad, _close, _logits, _np, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1, 8, 40, 64, 65, 100, 128, 129, 200, 256, 264])
@pytest.mark.parametrize("types", TYPES[:3])
@pytest.mark.parametrize("n,t", [(2, 3), (3, 1000)])
def test_block_norm_gradient_keeps_to_its_workspace(n, t, d, types):
    b = Block(n, t, d, types, 121)
    _, _, stats, kept = b.run(1, save=True, keep8=True)
    size = ceca.dsgd_block_norm_workspace_bytes(n, t, d)
    guard = 1 << 20   # more than every group of every CTA could write behind
    for src, held in (((b.h, b.y, b.gate), False), (kept, True)):
        ws = torch.full((size + guard,), 7, dtype=torch.uint8, device=DEV)
        got = b.grad(1, src, stats, workspace=ws[:size])
        assert (ws[size:] == 7).all()
        _check_grad(got, b.want_grad(1, stats, held), types)
        ws.fill_(255)   # NaNs: nothing is read that was not written
        again = b.grad(1, src, stats, workspace=ws[:size])
        assert (ws[size:] == 255).all() and all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("d", [40, 256, 771, 2048, 9000])   # every form of the kernels
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("act", [blocks.SIGMOID, blocks.SILU])
def test_gates_far_below_zero_are_shut(d, types, act):
    far = [-86.0, -88.0, -100.0, -1e4, -1e30, -1e38, float(torch.finfo(types[1]).min)]
    b = Block(1, 4 + len(far), d, types, 131)
    for i, a in enumerate(far):
        b.gate[0, 3 + i, i % 2::2] = a
    # below -87.3 the sigmoid is held at 2^-126: it is off by that at most and silu and its slope by 87.4 times that, below 2^-119;
    # what they are multiplied with (scale, weight, the normalised y, dh) stays below 2^9 here
    floor = 2.0 ** -110

    def near(got, pair, name):
        _close(got, (pair[0], pair[1] + floor), name)

    h, u, stats, kept = b.run(act, save=True, keep8=True)
    want = b.want(act, 1e-6)
    near(h, want["h"], "h_out")
    near(u, want["u"], "u")
    for src, held in (((b.h, b.y, b.gate), False), (kept, True)):
        wg = b.want_grad(act, stats, held)
        for k, g in zip(NAMES, b.grad(act, src, stats)):
            near(g, wg[k], k)
    # -infinity is as shut as the lowest value
    low = b.run(act), b.grad(act, (b.h, b.y, b.gate), stats)
    b.gate[b.gate < -1e20] = -INF
    shut = b.run(act), b.grad(act, (b.h, b.y, b.gate), stats)
    assert all(torch.equal(x, y) for x, y in zip(low[0][:2] + low[1], shut[0][:2] + shut[1]))
    b.gate[0, 3, 1] = NAN
    assert torch.isnan(b.run(act)[0][0, 3, 1])


@pytest.mark.parametrize("d", [40, 300, 9000])
@pytest.mark.parametrize("scale", [NAN, INF, 0.5])
def test_block_norm_gradient_of_no_rows_is_zero_whatever_the_scale(d, scale):
    b = Block(2, 0, d, (F32, F32, F32), 1)
    stats = torch.empty((2, 0, 2), device=DEV)
    b.scale.fill_(scale)   # right before, on the same stream
    got = b.grad(0, (b.h, b.y, b.gate), stats)
    assert all((g == 0).all() for g in got[3:])
    before = {k: _randn(v.shape, F32, 70 + i) for i, (k, v) in enumerate(zip(NAMES[3:], got[3:]))}
    got = b.grad(0, (b.h, b.y, b.gate), stats, accumulate=True, **{k: v.clone() for k, v in before.items()})
    assert all(torch.equal(g, before[k]) for k, g in zip(NAMES[3:], got[3:]))


@pytest.mark.parametrize("v", [7, 1001, 6001, 40000])   # rows held by a warp and by a CTA, rows in parts
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("broken", ["nan", "both masked"])
def test_preference_rows_without_a_token_stay_still_beside_broken_ones(v, dtype, broken):
    r, bounds = 900, [0, 6, 12, 400, 900]
    z, tok = _logits(r, v, dtype, 61)
    tok[:] = torch.arange(r, device=DEV) % v
    tok[[0, 1, 7, 450]] = torch.tensor([-1, v, -5, -1], device=DEV)
    z[1] = NAN
    z[7, ::2] = INF
    at = [3] if broken == "nan" else [3, 9]
    for i in at:
        z[i, tok[i]] = NAN if broken == "nan" else -INF
    b = torch.tensor(bounds, device=DEV)
    for out in (torch.full_like(z, 5), None):
        loss, logp, dz = ceca.dsgd_preference_grad(z, tok, b, average=out is None, dz=out)
        assert torch.isnan(loss[0]) and (dz[[0, 1, 7, 450]] == 0).all()
        assert torch.isnan(dz[2]).all() and torch.isnan(dz[8]).all()
        rest = blocks.preference(_np(z[12:]), _np(tok[12:]), [0, 388, 888], average=out is None, bf16=dtype == BF16, beta=np.float64(np.float32(0.1)))
        _close(loss[1:], rest["loss"], "loss")
        _close(dz[12:], rest["dz"], "dz")


@pytest.mark.parametrize("smoothing", [0.0, 1.0])
@pytest.mark.parametrize("v", [9, 20000])
def test_preference_of_an_impossible_answer_that_the_smoothing_wants(smoothing, v):
    z, tok = _logits(8, v, F32, 71)
    tok[:] = torch.arange(8, device=DEV)
    z[5 if smoothing == 0 else 1, 5 if smoothing == 0 else 1] = -INF
    loss, logp, dz = ceca.dsgd_preference_grad(z, tok, torch.tensor([0, 4, 8], device=DEV), smoothing=smoothing)
    assert loss[0] == 0 and (dz == 0).all()


@pytest.mark.parametrize("v", [9, 3000, 20000, 140000])
def test_policy_rows_without_an_advantage_whose_ratio_leaves_fp32(v):
    z, tok = _logits(7, v, F32, 73, torch.int32)
    old = torch.full((7,), -300.0, device=DEV)
    adv = torch.tensor([0.0, -0.0, 0.0, 0.0, 0.0, -1.0, 1.0], device=DEV)
    for kl in (0.0, 0.1):
        ref = torch.full((7,), -3.0, device=DEV)
        loss, dz = ceca.dsgd_policy_grad(z, tok, old, adv, ref_logp=ref, kl=kl)
        want = blocks.policy(_np(z), _np(tok), _np(old), _np(adv), _np(ref), kl=np.float64(np.float32(kl)))
        rest = [0, 1, 2, 3, 4, 6]   # of row 5 the loss leaves fp32 too
        _close(loss[rest], tuple(x[rest] for x in want["loss"]), "loss")
        _close(dz[rest], tuple(x[rest] for x in want["dz"]), "dz")
        assert loss[5] == INF


@pytest.mark.parametrize("v", [9, 3000, 20000, 140000])
@pytest.mark.parametrize("own", [NAN, INF])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_of_nothing_but_a_broken_token(v, own, dtype):
    z, tok = _logits(6, v, dtype, 75, torch.int32)
    tok[:] = 5
    z[3] = -INF
    z[3, 5] = own
    f = torch.full((6,), -1.0, device=DEV)
    loss, dz = ceca.dsgd_policy_grad(z, tok, f, f)
    assert torch.isnan(loss[3]) and torch.isnan(dz[3]).all()
    assert torch.isfinite(dz[[0, 1, 2, 4, 5]]).all()
    loss, _, dz = ceca.dsgd_preference_grad(z, tok, torch.tensor([0, 2, 4], device=DEV))
    assert torch.isnan(loss[0]) and torch.isnan(dz[:4]).all() and (dz[4:] == 0).all()
