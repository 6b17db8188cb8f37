"""The 64-bit statements of the language-model operators at the edges of their range, without a GPU."""
import numpy as np
import pytest
import torch

from oracle import lm


@pytest.mark.parametrize("temperature", [0.7, 1.0, 3.0])
@pytest.mark.parametrize("more", [0.3, 0.0, -0.05, -0.3, -2.0, "bf16"])
def test_distillation_statement_against_differences_whatever_mass_the_top_holds(temperature, more):
    # the teacher's own log-sum-exp may lie below that of its top, by the caller's choice or by the top's rounding to bf16
    r = np.random.default_rng(14)
    z, t = r.standard_normal((3, 20)) * 2, r.standard_normal((3, 6)) * 3
    idx = np.stack([r.permutation(20)[:6] for _ in range(3)])
    idx[0, 2], idx[1, 0] = -1, idx[1, 5]
    lse = np.log(np.where(idx >= 0, np.exp(t / temperature), 0).sum(1))
    if more == "bf16":
        sent = torch.from_numpy(t).to(torch.bfloat16).double().numpy()
        t = np.where(sent < t, sent + 2.0 ** -7 * np.abs(sent), sent)   # rounded up throughout: more than all mass
    else:
        lse = lse + more
    p = np.where(idx >= 0, np.exp(t / temperature - lse[:, None]), 0).sum(1)
    assert (p > 1 + 1e-4).all() if more == "bf16" or more < 0 else (p < 1 + 1e-12).all()
    w = np.array([0.5, 2.0, 1.0])
    g = lm.distill(z, idx, t, lse, w, temperature)["dz"][0]
    assert np.abs(g.sum(1)).max() <= 1e-12   # the loss does not know an offset of all logits
    if more == 0.0:
        return   # a kink: p0 is rounding
    for seed in range(3):
        u, h = np.random.default_rng(seed).standard_normal(z.shape), 1e-5
        up, dn = (lm.distill(z + c * u, idx, t, lse, w, temperature)["loss"][0].sum() for c in (h, -h))
        assert abs((up - dn) / (2 * h) - (g * u).sum()) <= 1e-8 * max(1.0, abs((g * u).sum()))


def test_the_module_is_built_for_one_python_and_one_torch(monkeypatch):
    from paper_2306_00256_b200 import build
    here = build.module_path()
    assert torch.__version__ in here and not build.module_is_stale()
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "0.0.1")
    assert build.module_path() != here and build.module_is_stale()
    assert not build.is_stale()   # the library has nothing to do with it


def test_rows_wider_than_the_embedding_supports_are_refused():
    from test_lm_operators_host import GRAD, INVALID, LOOKUP, UNSUPPORTED, _call
    import paper_2306_00256_b200 as ceca
    wide, huge = 65535 * 256 + 1, 1 << 31
    for t in (4, 4000):
        more = {"t": t, "agent": 1 << 45, "tok": t, "o_agent": 1 << 50}
        assert _call("dsgd_embed_grad", GRAD, d=wide, row=wide, o_row=wide, **more) == UNSUPPORTED
        assert _call("dsgd_embed_grad", GRAD, d=huge, row=huge, o_row=huge, **more) == INVALID
        assert _call("dsgd_embed_lookup", LOOKUP, d=huge, row=huge, o_row=huge, **more) == INVALID
    assert ceca.dsgd_embed_workspace_bytes(2, 4000, 8, wide) == 0 and ceca.dsgd_embed_workspace_bytes(2, 4000, 8, wide - 1) > 0
