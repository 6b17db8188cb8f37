"""The operators around a model's blocks and behind its logits at the edges of their range, without a GPU."""
import ctypes

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


def _at(i):   # stands for device memory: every call here is refused before anything is launched
    return ctypes.c_void_p(4096 * (i + 1))


@pytest.mark.parametrize("over", [dict(loss="old"), dict(loss="adv"), dict(loss="ref"), dict(logp="old"), dict(logp="adv"), dict(logp="ref"), dict(logp="loss")])
def test_policy_loss_refuses_outputs_over_what_is_read(over):
    args = {k: _at(i) for i, k in enumerate(("z", "tok", "old", "adv", "ref", "w", "loss", "logp"))}
    args |= {k: args[v] for k, v in over.items()}
    lib, ws = ceca.library(), _at(20)
    assert lib.dsgd_policy_loss(*args.values(), 2, 8, 8, 0, 0, 1.0, 0.2, 0.2, 0.1, ws, 1 << 20, None) == 4
    assert lib.dsgd_policy_grad(*args.values(), _at(30), 2, 8, 8, 8, 0, 0, 1.0, 0.2, 0.2, 0.1, ws, 1 << 20, None) == 4


@pytest.mark.parametrize("over", [dict(loss="ref"), dict(logp="ref"), dict(logp="loss")])
def test_preference_loss_refuses_outputs_over_what_is_read(over):
    args = {k: _at(i) for i, k in enumerate(("z", "tok", "bounds", "ref", "w", "loss", "logp"))}
    args |= {k: args[v] for k, v in over.items()}
    lib, ws = ceca.library(), _at(20)
    assert lib.dsgd_preference_loss(*args.values(), 1, 2, 8, 8, 0, 0, 0, 1.0, 0.1, 0.0, 0, ws, 1 << 20, None) == 4
    assert lib.dsgd_preference_grad(*args.values(), _at(30), 1, 2, 8, 8, 8, 0, 0, 0, 1.0, 0.1, 0.0, 0, ws, 1 << 20, None) == 4


@pytest.mark.parametrize("temperature,status", [(1e-39, 1), (1e-45, 1), (4.2e-39, 1), (4.3e-39, 5)])   # (5: of the workspace, which is looked at later)
def test_losses_refuse_temperatures_whose_reciprocal_leaves_fp32(temperature, status):
    lib, p, f = ceca.library(), _at(0), [_at(i) for i in range(1, 12)]
    v = 100000
    assert lib.dsgd_token_logprob(p, f[0], f[1], 2, v, v, 0, 0, temperature, None, 0, None) == status
    assert lib.dsgd_policy_loss(p, *f[:7], 2, v, v, 0, 0, temperature, 0.2, 0.2, 0.1, None, 0, None) == status
    assert lib.dsgd_policy_grad(p, *f[:8], 2, v, v, v, 0, 0, temperature, 0.2, 0.2, 0.1, None, 0, None) == status
    assert lib.dsgd_preference_loss(p, *f[:6], 1, 2, v, v, 0, 0, 0, temperature, 0.1, 0.0, 0, None, 0, None) == status
    assert lib.dsgd_preference_grad(p, *f[:7], 1, 2, v, v, v, 0, 0, 0, temperature, 0.1, 0.0, 0, None, 0, None) == status
