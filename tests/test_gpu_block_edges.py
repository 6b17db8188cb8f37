"""The operators around a model's blocks and behind its logits at the edges of their range: workspaces to the byte, gates and logits far out, rows
without a token beside rows of NaN.  Bounds as in oracle/blocks.py."""
import pytest
import torch

import paper_2306_00256_b200 as ceca
from test_gpu_block_operators import DEV, TYPES, Block, _check_grad

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
