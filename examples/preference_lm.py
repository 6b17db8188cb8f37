"""Decentralised training of small residual sequence models from preferences, and from rewards.

n agents hold one model each, all parameters of agent i in row i of X:

    h = scale * E[token],  u = w0 * h / rms(h)                                       dsgd_embed_lookup, dsgd_block_norm
    for every block:   x = u Wx,  a = sigmoid(u Wf + 1),  y_s = a_s y_{s-1} + (1 - a_s) x_s         dsgd_recurrence
                       h = h + r silu(u Wg) * wq * y / rms(y),  u = wp * h / rms(h)   dsgd_block_norm
    z = u U^T

Activations wait for the backward pass in 8 bits (dsgd_keep8, and dsgd_block_norm's keep8), or as they are.  A batch holds pairs of answers to
a prompt, packed into each agent's sequence; dsgd_preference_grad compares their log-probabilities with those under the models that training
began with.  With --loss policy the answers are the models' own samples, rewarded, and dsgd_policy_grad takes a few clipped steps on them.
Gradients go straight into the agent's row of G, and ceca_gossip_sgd_step applies them together with one CECA gossip round.  The dense products
are torch's.  What is preferred (and rewarded) here is a fixed random half of the vocabulary, so that nothing has to be downloaded.

    python examples/preference_lm.py --agents 6 --steps 40
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_00256_b200 as ceca  # noqa: E402


class ResidualModel:
    """Where the parameters lie in a row, and the models' logits and gradients for all agents at once."""

    def __init__(self, vocabulary, width, blocks=2, keep8=True):
        self.v, self.d, self.blocks, self.keep8 = vocabulary, width, blocks, keep8
        self.shapes = {"E": (vocabulary, width), "U": (vocabulary, width), "w0": (width,)}
        for k in range(blocks):
            self.shapes |= {"Wx%d" % k: (width, width), "Wf%d" % k: (width, width), "Wg%d" % k: (width, width), "wq%d" % k: (width,), "wp%d" % k: (width,), "r%d" % k: ()}
        self.at, end = {}, 0
        for name, shape in self.shapes.items():
            self.at[name] = (end, end + math.prod(shape))
            end += math.prod(shape)
        self.size = end
        self.scale = math.sqrt(width)

    def views(self, X):
        """name -> [n, ...] view of that block of columns of X [n, size]."""
        return {k: X[:, a:b].unflatten(1, self.shapes[k]) if self.shapes[k] else X[:, a] for k, (a, b) in self.at.items()}

    def init(self, X, generator):
        for name, w in self.views(X).items():
            if name[0] == "w" or name[0] == "r":
                w.fill_(1.0 if name[0] == "w" else 0.5)
            else:
                w.copy_(torch.randn(w.shape[1:], generator=generator).to(X.device) * (0.05 if name == "E" else self.d ** -0.5))

    def forward(self, Z, tok, starts, save=True):
        """Logits [n, t, v] of the models Z [n, size], and what `backward` needs."""
        w, kept = self.views(Z), []
        h = ceca.dsgd_embed_lookup(w["E"], tok, self.scale)
        _, u, first, h8 = ceca.dsgd_block_norm(h, None, w["w0"], None, save=save, keep8=save and self.keep8)
        kept.append((h if h8 is None else h8[0], first, u))
        for k in range(self.blocks):
            x, f, a = (torch.bmm(u, w[m + str(k)]) for m in ("Wx", "Wf", "Wg"))
            y, _, marks = ceca.dsgd_recurrence(x, f.add_(1.0), starts=starts, save=save)
            ho, uo, stats, packed = ceca.dsgd_block_norm(h, y, w["wp%d" % k], w["wq%d" % k], gate=a, gate_act=ceca.GATE_SILU, scale=w["r%d" % k], save=save,
                                                         keep8=save and self.keep8)
            if save:
                xf = [ceca.dsgd_keep8(m) for m in (x, f)] if self.keep8 else [x, f]
                kept.append((xf, marks, packed or (h, y, a), stats, u))
            h, u = ho, uo
        return torch.bmm(u, w["U"].transpose(1, 2)), (kept, u)

    def backward(self, Z, G, tok, starts, saved, dz):
        """Writes the gradient with respect to Z to G, dz being that with respect to the logits."""
        w, g = self.views(Z), self.views(G)
        kept, u = saved
        g["U"].copy_(torch.bmm(dz.transpose(1, 2), u))
        du, dh = torch.bmm(dz, w["U"]), None
        for k in reversed(range(self.blocks)):
            (x, f), marks, (h, y, a), stats, u = kept[k + 1]
            if self.keep8:
                x, f = (ceca.dsgd_bring8(m, self.d) for m in (x, f))
            dh, dy, da, _, _, _ = ceca.dsgd_block_norm_grad(h, y, w["wp%d" % k], w["wq%d" % k], stats, du, dh, gate=a, gate_act=ceca.GATE_SILU, scale=w["r%d" % k],
                                                            dw_pre=g["wp%d" % k], dw_post=g["wq%d" % k], dscale=g["r%d" % k])
            dx, df, _ = ceca.dsgd_recurrence_grad(x, f, dy, marks, starts=starts)
            du = torch.zeros_like(dx)
            for m, d in (("Wx", dx), ("Wf", df), ("Wg", da)):
                g[m + str(k)].copy_(torch.bmm(u.transpose(1, 2), d))
                du.baddbmm_(d, w[m + str(k)].transpose(1, 2))
        h, first, _ = kept[0]
        dh = ceca.dsgd_block_norm_grad(h, None, w["w0"], None, first, du, dh, dw_pre=g["w0"])[0]
        ceca.dsgd_embed_grad(dh, tok, g["E"], self.scale)


class Preferences:
    """Pairs of answers to random prompts: of the preferred one more tokens come from a fixed half of the vocabulary."""

    def __init__(self, vocabulary, generator, device):
        self.good = torch.randperm(vocabulary, generator=generator)[: vocabulary // 2].to(device)
        self.liked = torch.zeros(vocabulary, dtype=torch.bool, device=device)
        self.liked[self.good] = True
        self.v, self.device = vocabulary, device

    def batch(self, n, pairs, prompt, length, generator):
        """Tokens and document starts [n, t], the token that each position is to predict (-1 in prompts and at the ends) and the sequences' bounds."""
        each = prompt + length
        draw = lambda *shape: torch.randint(0, self.v, shape, generator=generator).to(self.device)  # noqa: E731
        tok = draw(n, pairs, 2, each)
        tok[:, :, 1, :prompt] = tok[:, :, 0, :prompt]
        better = torch.rand((n, pairs, length), generator=generator).to(self.device) < 0.8
        tok[:, :, 0, prompt:] = torch.where(better, self.good[draw(n, pairs, length) % len(self.good)], tok[:, :, 0, prompt:])
        target = torch.full_like(tok, -1)
        target[..., prompt - 1:-1] = tok[..., prompt:]
        starts = torch.zeros(tok.shape, dtype=torch.uint8, device=self.device)
        starts[..., 0] = 1
        bounds = torch.arange(n * pairs * 2 + 1, device=self.device) * each
        return tok.reshape(n, -1), starts.reshape(n, -1), target.reshape(-1), bounds


def train(agents=6, vocabulary=200, width=64, blocks=2, pairs=4, prompt=8, length=24, steps=40, gamma=0.5, beta=0.5, loss="preference", keep8=True, variant=None,
          seed=0, log=print):
    """Returns (first and last mean loss, deviation of the models from their mean after a final consensus)."""
    device = "cuda:%d" % torch.cuda.current_device()
    variant = variant or (ceca.CECA_2P if agents % 2 else ceca.CECA_1P)
    gen = torch.Generator().manual_seed(seed)
    model, data = ResidualModel(vocabulary, width, blocks, keep8), Preferences(vocabulary, gen, device)
    X, G = (torch.zeros(agents, model.size, device=device) for _ in range(2))
    model.init(X, gen)
    Y, reference = X.clone(), X.clone()
    first = last = held = None
    for step in range(steps):
        at = ceca.ceca_schedule(agents, variant, step, peers=False)[0]
        Z = Y if at.payload else X
        if loss == "preference":
            tok, starts, target, bounds = data.batch(agents, pairs, prompt, length, gen)
            rows = lambda z: z.view(-1, vocabulary)  # noqa: E731
            ref = ceca.dsgd_preference_loss(rows(model.forward(reference, tok, starts, save=False)[0]), target, bounds)[1]
            z, saved = model.forward(Z, tok, starts)
            losses, _, dz = ceca.dsgd_preference_grad(rows(z), target, bounds, ref_logp=ref, weight=torch.full((agents * pairs,), 1.0 / pairs, device=device), beta=beta,
                                                      dz=rows(z))
            losses = losses.view(agents, pairs).sum(1)
        else:
            if step % 4 == 0:   # new samples, of which four steps are taken
                tok, starts, target, _ = data.batch(agents, 2 * pairs, prompt, length, gen)
                z, _ = model.forward(Z, tok, starts, save=False)
                live = target >= 0
                sample = torch.distributions.Categorical(logits=z.view(-1, vocabulary)).sample()
                target = torch.where(live, sample, -1)
                reward = data.liked[sample].float()
                advantage = (reward - reward[live].mean()) / (reward[live].std() + 1e-6)
                flat = z.view(-1, vocabulary)
                old = ceca.dsgd_token_logprob(flat, target)
                ref = ceca.dsgd_token_logprob(model.forward(reference, tok, starts, save=False)[0].view(-1, vocabulary), target)
                held = (tok, starts, target, old, advantage, ref, live.float() / live.view(agents, -1).sum(1).repeat_interleave(tok.shape[1]))
            tok, starts, target, old, advantage, ref, weight = held
            z, saved = model.forward(Z, tok, starts)
            flat = z.view(-1, vocabulary)
            losses, dz = ceca.dsgd_policy_grad(flat, target, old, advantage, ref_logp=ref, weight=weight, kl=0.02, dz=flat)
            losses = losses.view(agents, -1).sum(1)
        model.backward(Z, G, tok, starts, saved, dz.view(agents, -1, vocabulary))
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
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--vocabulary", type=int, default=200)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--loss", choices=["preference", "policy"], default="preference")
    ap.add_argument("--whole", action="store_true", help="keep activations as they are")
    a = ap.parse_args()
    train(agents=a.agents, steps=a.steps, vocabulary=a.vocabulary, width=a.width, loss=a.loss, keep8=not a.whole)
