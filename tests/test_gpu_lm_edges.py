"""The language-model operators at the edges of their range: NaN where it has to be seen, logits far apart or far from
zero, teachers whose mass is spent, arguments that have to be refused.  Bounds as in oracle/lm.py."""
import numpy as np
import pytest
import torch

import paper_2306_00256_b200 as ceca
from oracle import lm
from test_gpu_lm_operators import BF16, DEV, F32, NAN, _close, _np, _randn

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
