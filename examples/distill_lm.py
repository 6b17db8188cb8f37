"""Decentralised training of small language models from a teacher's top logits.

n agents hold one sequence model each, all parameters of agent i in row i of X:

    e = scale * E[token]                     E: vocabulary x width             dsgd_embed_lookup
    h_s = a_s h_{s-1} + (1 - a_s) x_s        x = e Wx, a = sigmoid(e Wf + 1)   dsgd_recurrence
    z = h U^T                                U: vocabulary x width

and is trained on sequences of its own against the top logits that a teacher sends for every position
(dsgd_distill_grad).  The gradients go straight into the agent's row of G (dsgd_embed_grad writes the embedding's
block of columns), and ceca_gossip_sgd_step applies them together with one CECA gossip round.  The dense
products are torch's.  The teacher here is a random bigram model, so that nothing has to be downloaded.

    python examples/distill_lm.py --agents 6 --steps 60
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_00256_b200 as ceca  # noqa: E402


class SequenceModel:
    """Where the parameters lie in a row, and the model's loss and gradient for all agents at once."""

    def __init__(self, vocabulary, width):
        self.v, self.d = vocabulary, width
        self.shapes = {"E": (vocabulary, width), "Wx": (width, width), "Wf": (width, width), "U": (vocabulary, width)}
        self.at, end = {}, 0
        for name, (rows, cols) in self.shapes.items():
            self.at[name] = (end, end + rows * cols)
            end += rows * cols
        self.size = end
        self.scale = math.sqrt(width)

    def views(self, X):
        """name -> [n, rows, cols] view of that block of columns of X [n, size]."""
        return {k: X[:, a:b].unflatten(1, self.shapes[k]) for k, (a, b) in self.at.items()}

    def init(self, X, generator):
        for name, w in self.views(X).items():
            w.copy_(torch.randn(w.shape[1:], generator=generator).to(X.device) * (0.02 if name == "E" else w.shape[2] ** -0.5))

    def loss_and_gradient(self, Z, G, batch):
        """Mean loss per agent at the models Z [n, size]; writes their gradient to G."""
        tok, starts, idx, top, lse = batch
        n, t = tok.shape
        w, g = self.views(Z), self.views(G)
        e = ceca.dsgd_embed_lookup(w["E"], tok, self.scale)
        x = torch.bmm(e, w["Wx"])
        f = torch.bmm(e, w["Wf"]).add_(1.0)
        h, _, marks = ceca.dsgd_recurrence(x, f, starts=starts, save=True)
        z = torch.bmm(h, w["U"].transpose(1, 2))
        weight = torch.full((n * t,), 1.0 / t, device=Z.device)
        loss, dz = ceca.dsgd_distill_grad(z.view(n * t, self.v), idx, top, teacher_lse=lse, weight=weight, dz=z.view(n * t, self.v))
        dz = dz.view(n, t, self.v)
        g["U"].copy_(torch.bmm(dz.transpose(1, 2), h))
        dx, df, _ = ceca.dsgd_recurrence_grad(x, f, torch.bmm(dz, w["U"]), marks, starts=starts)
        g["Wx"].copy_(torch.bmm(e.transpose(1, 2), dx))
        g["Wf"].copy_(torch.bmm(e.transpose(1, 2), df))
        de = torch.bmm(dx, w["Wx"].transpose(1, 2)).baddbmm_(df, w["Wf"].transpose(1, 2))
        ceca.dsgd_embed_grad(de, tok, g["E"], self.scale)
        return loss.view(n, t).sum(1)


class BigramTeacher:
    """Knows the next token's logits from the last token alone; sends the top k and their log-sum-exp over all."""

    def __init__(self, vocabulary, k, generator, device):
        self.logits = (3.0 * torch.randn(vocabulary, vocabulary, generator=generator)).to(device)
        self.k = k

    def batch(self, n, t, generator):
        v, device = self.logits.shape[0], self.logits.device
        tok = torch.randint(0, v, (n, t), generator=generator).to(device)
        starts = (torch.rand(n, t, generator=generator) < 0.02).to(torch.uint8).to(device)
        rows = self.logits[tok.reshape(-1)]
        top, idx = rows.topk(self.k, dim=1)
        return tok, starts, idx, top, torch.logsumexp(rows, 1)


def train(agents=6, vocabulary=500, width=64, length=128, k=16, steps=60, gamma=6.0, variant=None, seed=0, log=print):
    """Returns (first and last mean loss, deviation of the models from their mean after a final consensus)."""
    device = "cuda:%d" % torch.cuda.current_device()
    variant = variant or (ceca.CECA_2P if agents % 2 else ceca.CECA_1P)
    gen = torch.Generator().manual_seed(seed)
    model, teacher = SequenceModel(vocabulary, width), BigramTeacher(vocabulary, k, gen, device)
    X, G = (torch.zeros(agents, model.size, device=device) for _ in range(2))
    model.init(X, gen)
    Y = X.clone()
    first = last = None
    for step in range(steps):
        at = ceca.ceca_schedule(agents, variant, step, peers=False)[0]
        losses = model.loss_and_gradient(Y if at.payload else X, G, teacher.batch(agents, length, gen))
        ceca.ceca_gossip_sgd_step(X, Y, G, gamma, variant, step)
        if step % 10 == 0 or step == steps - 1:
            last = float(losses.mean())
            first = last if first is None else first
            log("step %4d  mean loss %.4f" % (step, last))
    rounds = ceca.ceca_schedule(agents, variant, 0, peers=False)[0].tau
    ceca.ceca_consensus_rounds(X, Y, variant, 0, rounds, ceca.UNFUSED)
    off = float((X - X.mean(0)).norm() / X.norm())
    log("after %d rounds of consensus the models differ by %.1e of their norm" % (rounds, off))
    return first, last, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--agents", type=int, default=6)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--vocabulary", type=int, default=500)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--length", type=int, default=128)
    a = ap.parse_args()
    train(agents=a.agents, steps=a.steps, vocabulary=a.vocabulary, width=a.width, length=a.length)
