"""The operators around a model's blocks and behind its logits at the edges of their range, without a GPU."""
import pytest

import paper_2306_00256_b200 as ceca


def _written(n, t, d):
    """Bytes of its workspace that the block norms' gradient writes for rows of up to 256 channels: CTAs of 128 threads, four on each of 148 SMs, of
    as many groups of threads as one row of d channels needs.  Each CTA is a part of an agent's rows, and leaves the sums of the two
    weights' gradients for every channel and of the scale's for every group, in fp32."""
    groups = 16 if d <= 64 else 8 if d <= 128 else 4
    parts = max(1, min(148 * 4 // n, max(min(-(-t // groups), 32), -(-t // (4 * groups)))))
    return 4 * n * parts * (2 * d + groups)


@pytest.mark.parametrize("d", [1, 8, 40, 64, 65, 100, 128, 129, 200, 256])
@pytest.mark.parametrize("n,t", [(1, 1), (1, 256), (2, 1000), (8, 4096), (4, 32768), (3000, 2), (65535, 1)])
def test_block_norm_workspace_holds_what_the_gradient_writes(n, t, d):
    assert _written(n, t, d) <= ceca.dsgd_block_norm_workspace_bytes(n, t, d) < _written(n, t, d) + 16 * n
