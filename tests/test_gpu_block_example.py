"""The example that trains residual models from preferences: its whole gradient against automatic differentiation in 64 bits, and a short run."""
import importlib.util
import os

import pytest
import torch

import paper_2306_00256_b200 as ceca

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("preference_lm", os.path.join(ROOT, "examples", "preference_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _logits64(model, Z, tok, starts):
    """The same models in elementary operations, for automatic differentiation."""
    w = model.views(Z)
    norm = lambda x: x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    h = torch.stack([e[t] for e, t in zip(w["E"], tok)]) * model.scale
    u = norm(h) * w["w0"][:, None]
    for k in range(model.blocks):
        x, f, a = u @ w["Wx%d" % k], u @ w["Wf%d" % k] + 1, u @ w["Wg%d" % k]
        keep, state, ys = torch.sigmoid(f), torch.zeros_like(x[:, 0]), []
        for s in range(x.shape[1]):
            state = keep[:, s] * torch.where(starts[:, s, None] != 0, 0.0, 1.0) * state + (1 - keep[:, s]) * x[:, s]
            ys.append(state)
        h = h + w["r%d" % k][:, None, None] * a * torch.sigmoid(a) * norm(torch.stack(ys, 1)) * w["wq%d" % k][:, None]
        u = norm(h) * w["wp%d" % k][:, None]
    return u @ w["U"].transpose(1, 2)


def _preference64(z, target, bounds, ref, weight, beta):
    lp = torch.where(target >= 0, torch.log_softmax(z, 1).gather(1, target.clamp_min(0)[:, None])[:, 0], 0.0)
    L = torch.stack([lp[a:b].sum() for a, b in zip(bounds[:-1], bounds[1:])])
    m = beta * ((L[0::2] - ref[0::2]) - (L[1::2] - ref[1::2]))
    return (-weight * torch.nn.functional.logsigmoid(m)).sum()


@pytest.mark.parametrize("width", [32, 45])
@pytest.mark.parametrize("keep8", [False, True])
def test_whole_gradient_against_automatic_differentiation(width, keep8):
    ex = _example()
    torch.backends.cuda.matmul.allow_tf32 = False
    gen = torch.Generator().manual_seed(3)
    n, v, pairs = 3, 61, 2
    model, data = ex.ResidualModel(v, width, 2, keep8), ex.Preferences(v, gen, DEV)
    Z, G = (torch.zeros(n, model.size, device=DEV) for _ in range(2))
    model.init(Z, gen)
    Z += 0.05 * torch.randn(Z.shape, generator=gen).to(DEV)
    tok, starts, target, bounds = data.batch(n, pairs, 3, 9, gen)
    ref = torch.randn(2 * n * pairs, generator=gen).to(DEV) - 30
    weight = torch.rand(n * pairs, generator=gen).to(DEV)
    z, saved = model.forward(Z, tok, starts)
    loss, _, dz = ceca.dsgd_preference_grad(z.view(-1, v), target, bounds, ref_logp=ref, weight=weight, beta=0.5)
    model.backward(Z, G, tok, starts, saved, dz.view(n, -1, v))
    Z64 = Z.double().requires_grad_()
    want = _preference64(_logits64(model, Z64, tok, starts).view(-1, v), target, bounds.tolist(), ref.double(), weight.double(), 0.5)
    want.backward()
    # 32 bits: some 10^3 roundings along the longest path.  8 bits: every activation is off by at most 2^-8 of its block's largest, which
    # is some 4 times its own size; a gradient passes a handful of them, with signs that are as good as random.
    assert abs(float(loss.sum()) - float(want.detach())) <= 1e-4 * abs(float(want.detach()))
    bound = 0.05 if keep8 else 1e-4
    for name, g in model.views(G).items():
        w = model.views(Z64.grad)[name]
        assert float((g.double() - w).norm()) <= bound * float(w.norm()), name


@pytest.mark.parametrize("loss", ["preference", "policy"])
@pytest.mark.parametrize("keep8", [False, True])
def test_example_runs(loss, keep8):
    lines = []
    first, last, off = _example().train(agents=5, vocabulary=50, width=32, blocks=1, pairs=2, prompt=4, length=8, steps=9, loss=loss, keep8=keep8, log=lines.append)
    assert first == first and last == last and off < 1e-5 and len(lines) == 3


def test_a_training_step_in_a_captured_graph():
    ex = _example()
    gen = torch.Generator().manual_seed(5)
    n, v = 3, 100
    model, data = ex.ResidualModel(v, 48, 2), ex.Preferences(v, gen, DEV)
    Z, G = (torch.zeros(n, model.size, device=DEV) for _ in range(2))
    model.init(Z, gen)
    tok, starts, target, bounds = data.batch(n, 2, 4, 12, gen)

    def step():
        z, saved = model.forward(Z, tok, starts)
        loss, logp, dz = ceca.dsgd_preference_grad(z.view(-1, v), target, bounds)
        model.backward(Z, G, tok, starts, saved, dz.view(n, -1, v))
        return loss, logp

    want = [x.clone() for x in step()] + [G.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    G.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(list(got) + [G], want):
        assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max()) + 1e-12   # (torch may choose another product in a graph)
