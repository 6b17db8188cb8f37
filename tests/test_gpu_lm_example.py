"""The language-model operators together, as examples/distill_lm.py uses them: the gradient of a whole model against
automatic differentiation of the same model in 64 bits, and a training run."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("distill_lm", os.path.join(ROOT, "examples", "distill_lm.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _loss64(model, Z, batch):
    """The mean loss of every agent from the definitions, differentiable, on the CPU."""
    tok, starts, idx, top, lse = (b.cpu() for b in batch)
    n, t = tok.shape
    w = model.views(Z)
    e = model.scale * torch.stack([w["E"][i][tok[i]] for i in range(n)])
    x, f = e @ w["Wx"], e @ w["Wf"] + 1.0
    a, h, hs = torch.sigmoid(f), torch.zeros(n, model.d, dtype=torch.float64), []
    for s in range(t):
        h = torch.where(starts[:, s:s + 1] != 0, 0.0, a[:, s]) * h + (1 - a[:, s]) * x[:, s]
        hs.append(h)
    z = torch.stack(hs, 1) @ w["U"].transpose(1, 2)
    logq = torch.log_softmax(z.reshape(n * t, -1), 1)
    logp = top.double() - lse.double()[:, None]
    inside = torch.zeros_like(logq, dtype=torch.bool).scatter_(1, idx, True)
    rest = 1 - logp.exp().sum(1)
    kl = (logp.exp() * (logp - logq.gather(1, idx))).sum(1) + rest * (rest.log() - torch.logsumexp(logq.masked_fill(inside, -np.inf), 1))
    return kl.view(n, t).mean(1)


@pytest.mark.parametrize("n,v,d,t", [(3, 61, 24, 37), (2, 130, 40, 300)])
def test_model_gradient_against_automatic_differentiation(n, v, d, t):
    ex = _example()
    gen = torch.Generator().manual_seed(1)
    model, teacher = ex.SequenceModel(v, d), ex.BigramTeacher(v, 9, gen, "cuda:0")
    X, G = torch.zeros(n, model.size, device="cuda:0"), torch.full((n, model.size), float("nan"), device="cuda:0")
    model.init(X, gen)
    X += 0.1 * torch.randn(X.shape, generator=gen).to(X.device)   # the agents differ
    batch = teacher.batch(n, t, gen)
    loss = model.loss_and_gradient(X, G, batch)
    Z = X.double().cpu().requires_grad_()
    want = _loss64(model, Z, batch)
    want.sum().backward()
    # fp32 products of up to v + d terms in a chain of five: relative 2-norm errors stay below 1e-4 by a wide margin
    assert float((loss.double().cpu() - want.detach()).abs().max()) <= 1e-4 * float(want.detach().abs().max())
    for name, g in model.views(G).items():
        ref = model.views(Z.grad)[name]
        assert float((g.double().cpu() - ref).norm()) <= 1e-4 * float(ref.norm()), name


@pytest.mark.parametrize("agents", [5, 6])
def test_training_brings_the_loss_down_and_the_agents_together(agents):
    first, last, off = _example().train(agents=agents, steps=40, log=lambda *_: None)
    assert last < 0.8 * first and off <= 1e-5
