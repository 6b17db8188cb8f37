"""What the operators around a model's blocks and behind its logits are measured on, and their plain forms.

Four operators that stand next to the embedding, the recurrence and the distillation loss.  `n` agents train side
by side, so activations are n x t x d and weights n x d, one row for each agent.

  block, block_train      the end of a block and the start of the next: the block's output is normalised, gated, scaled
                          and added to the residual stream, which is normalised again; with the gradient, from
                          activations kept whole or in 8 bits
  keep8                   activations kept in 8 bits, and brought back
  logprob, policy         log-probabilities of tokens, and the clipped policy loss with a KL term and its gradient
  prefer                  the preference loss of pairs of answers (paired log ratios) and its gradient

  listed(), draw(rng)    the cases
  prepare(case, seed)    a case's inputs on the GPU
  run(state)             one pass: elementary torch operations in 32 bits, or (own = True) the library's calls
  work(case)             the bytes and operations that a pass cannot do without
  exact(case, seed)      the outputs from the definitions, in 64 bits
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TOKENS = {"i32": torch.int32, "i64": torch.int64}
DEV = "cuda"

EPS = 1e-6        # of the norms
BLOCK = 32        # channels that share an exponent in 8 bits
CLIP = (0.2, 0.3)  # of the policy's ratio, below and above 1
BETA = 0.1        # of the preference loss


def listed():
    return [
        # One new token for each of 256 sequences that are being answered; latency counts.
        {"name": "block_token", "op": "block", "n": 1, "t": 256, "d": 2048, "stream": "bf16", "act": "bf16", "gate": "silu"},
        # A long document read by one agent, its residual stream in 32 bits.
        {"name": "block_prompt", "op": "block", "n": 1, "t": 32768, "d": 1024, "stream": "f32", "act": "bf16", "gate": "sigmoid"},
        # A training step of eight agents, forward and backward, what the backward pass needs kept in 8 bits.
        {"name": "block_train_8bit", "op": "block_train", "n": 8, "t": 4096, "d": 2048, "stream": "bf16", "act": "bf16", "gate": "silu", "kept": "8bit"},
        # Odd length and width in 32 bits: rows that are not 16-byte aligned, activations kept as they are.
        {"name": "block_train_odd", "op": "block_train", "n": 3, "t": 1537, "d": 771, "stream": "f32", "act": "f32", "gate": "sigmoid", "kept": "whole"},
        # Activations of a short batch of odd width; latency counts.
        {"name": "keep8_small", "op": "keep8", "n": 4, "t": 129, "d": 257, "act": "f32"},
        # The recurrence's inputs of a training batch, kept between its forward and backward pass.
        {"name": "keep8_large", "op": "keep8", "n": 8, "t": 8192, "d": 2048, "act": "bf16"},
        # The log-probability of the token that each of 256 sequences just got.
        {"name": "logprob_token", "op": "logprob", "r": 256, "v": 32000, "dtype": "bf16", "tokens": "i64", "temperature": 1.0},
        # Log-probabilities under a reference model: a vocabulary of odd size in 32 bits.
        {"name": "logprob_odd", "op": "logprob", "r": 2047, "v": 50001, "dtype": "f32", "tokens": "i32", "temperature": 0.7},
        # The step of a small vocabulary and few positions; latency counts.
        {"name": "policy_small", "op": "policy", "r": 64, "v": 1000, "dtype": "f32", "tokens": "i32", "ref": True, "grad": True, "temperature": 1.0},
        # A training step over a large vocabulary: eight agents with 1024 positions each.
        {"name": "policy_large", "op": "policy", "r": 8192, "v": 128000, "dtype": "bf16", "tokens": "i64", "ref": True, "grad": True, "temperature": 1.0},
        # Three pairs of answers of uneven length, means instead of sums, an odd vocabulary in 32 bits.
        {"name": "prefer_odd", "op": "prefer", "pairs": 3, "r": 1023, "v": 50001, "dtype": "f32", "tokens": "i64", "ref": False, "average": True, "grad": True},
        # A training batch of sixteen pairs of some 512 positions with their prompts.
        {"name": "prefer_large", "op": "prefer", "pairs": 16, "r": 16384, "v": 32000, "dtype": "bf16", "tokens": "i32", "ref": True, "average": False, "grad": True},
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; odd ones and multiples of eight both come often."""
    x = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    x = x // 8 * 8 if rng.random() < 0.5 else x | 1
    return min(hi, max(lo, x))


def draw(rng):
    op = rng.choice(["block", "block_train", "keep8", "logprob", "policy", "prefer"])
    if op in ("block", "block_train", "keep8"):
        case = {"op": op, "n": rng.randint(1, 8), "d": _log_int(rng, 64, 4096), "act": rng.choice(["f32", "bf16"])}
        case["t"] = _log_int(rng, 1, min(32768, 8 * 4096 * 2048 // (case["n"] * case["d"])))
        if op != "keep8":
            case["stream"] = "f32" if case["act"] == "f32" else rng.choice(["f32", "bf16"])
            case["gate"] = rng.choice(["none", "sigmoid", "silu"])
        if op == "block_train":
            case["kept"] = rng.choice(["whole", "8bit"])
        return case
    case = {"op": op, "v": _log_int(rng, 500, 131072), "dtype": rng.choice(["f32", "bf16"]), "tokens": rng.choice(["i32", "i64"])}
    case["r"] = _log_int(rng, 16, min(16384, (512 << 20) // case["v"]))
    if op == "prefer":
        case["pairs"] = _log_int(rng, 1, max(1, min(64, case["r"] // 8)))
        case["average"] = rng.random() < 0.3
    else:
        case["temperature"] = rng.choice([0.7, 1.0, 1.5])
    if op != "logprob":
        case["ref"] = rng.random() < 0.7
        case["grad"] = rng.random() < 0.75
    return case


# ------------------------------------------------------------------------------------------------- inputs


def _normal(g, shape, dtype=torch.float32, mean=0.0, std=1.0):
    x = torch.empty(shape, device=DEV, dtype=dtype)
    return x.normal_(mean, std, generator=g)


def _logprob_of(z, tok, temperature):
    """log softmax(z / temperature) at the tokens (any number where there is none), some rows at a time."""
    out = []
    for r0 in range(0, z.shape[0], 1024):
        y = z[r0:r0 + 1024].double() / temperature if z.shape[1] < 4096 else z[r0:r0 + 1024].float() / temperature
        out.append(y.gather(1, tok[r0:r0 + 1024, None].long().clamp_min(0))[:, 0] - torch.logsumexp(y, 1))
    return torch.cat(out).double()


def _logits(case, g, s):
    r, v, dt = case["r"], case["v"], DTYPES[case["dtype"]]
    tok = torch.randint(0, v, (r,), device=DEV, generator=g)
    z = _normal(g, (r, v), dt, 0.0, 1.5)
    z.scatter_add_(1, tok[:, None], (4.0 + 3.0 * torch.rand((r, 1), device=DEV, generator=g)).to(dt))  # the model has learnt some of it
    s["z"], s["token"] = z, tok
    return z, tok


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    s = dict(case)
    if case["op"] == "keep8":
        # channels of unlike size, as activations have them
        x = _normal(g, (case["n"], case["t"], case["d"]))
        x *= torch.exp(_normal(g, (case["d"],)))
        s["x"] = x.to(DTYPES[case["act"]])
    elif case["op"] in ("block", "block_train"):
        n, t, d, dh, da = case["n"], case["t"], case["d"], DTYPES[case["stream"]], DTYPES[case["act"]]
        s["h"] = _normal(g, (n, t, d), dh, 0.0, 2.0)
        s["y"] = _normal(g, (n, t, d), da, 0.1, 0.7)
        s["gate_"] = _normal(g, (n, t, d), da, 0.5, 1.5) if case["gate"] != "none" else None
        s["w_pre"] = _normal(g, (n, d), torch.float32, 1.0, 0.1)
        s["w_post"] = _normal(g, (n, d), torch.float32, 1.0, 0.1)
        s["scale"] = _normal(g, (n,), torch.float32, 0.5, 0.1)
        if case["op"] == "block_train":
            s["du"] = _normal(g, (n, t, d), da, 0.0, 1e-2)
            s["dh_out"] = _normal(g, (n, t, d), dh, 0.0, 1e-2)
    elif case["op"] == "logprob":
        _, tok = _logits(case, g, s)
        tok[torch.rand(case["r"], device=DEV, generator=g) < 0.02] = -1  # a sequence that has ended
        s["token"] = tok.to(TOKENS[case["tokens"]])
    elif case["op"] == "policy":
        r = case["r"]
        z, tok = _logits(case, g, s)
        lp = _logprob_of(z, tok, case["temperature"])
        # some steps after the samples were drawn; the ratio is kept off the corners of its clipping
        moved = _normal(g, (r,), torch.float64, 0.0, 0.15)
        for corner in (math.log1p(-CLIP[0]), math.log1p(CLIP[1])):
            moved = torch.where((moved - corner).abs() < 2e-3, corner + 4e-3, moved)
        s["old"] = (lp - moved).float()
        s["ref_"] = (lp + _normal(g, (r,), torch.float64, 0.0, 0.3)).float() if case["ref"] else None
        s["advantage"] = _normal(g, (r,))
        s["weight"] = torch.rand(r, device=DEV, generator=g) / r
        s["kl"] = 0.05 if case["ref"] else 0.0
        tok[_prompt_rows(r)] = -1
        s["token"] = tok.to(TOKENS[case["tokens"]])
    else:
        r, pairs = case["r"], case["pairs"]
        z, tok = _logits(case, g, s)
        # answers of uneven length, packed one behind the other, and a few positions of padding at the end
        part = 0.5 + torch.rand(2 * pairs, device=DEV, generator=g)
        ends = (torch.cumsum(part, 0) / part.sum() * (r - r // 32)).long()
        s["bounds"] = torch.cat([ends.new_zeros(1), ends]).to(TOKENS[case["tokens"]])
        at = torch.arange(r, device=DEV)
        of = torch.bucketize(at, ends, right=True)
        begin = s["bounds"].long()[of.clamp_max(2 * pairs - 1)]
        length = ends[of.clamp_max(2 * pairs - 1)] - begin
        tok[(at - begin) * 4 < length - 3] = -1  # the first quarter of each sequence is its prompt
        s["token"] = tok.to(TOKENS[case["tokens"]])
        s["ref_"] = None
        if case["ref"]:
            lp = torch.where(tok >= 0, _logprob_of(z, tok, 1.0), 0.0)
            total = torch.zeros(2 * pairs + 1, device=DEV, dtype=torch.float64).index_add_(0, of, lp)[:-1]
            count = torch.zeros(2 * pairs + 1, device=DEV, dtype=torch.float64).index_add_(0, of, (tok >= 0).double())[:-1]
            total = total / count.clamp_min(1) if case["average"] else total
            s["ref_"] = (total + _normal(g, (2 * pairs,), torch.float64, 0.0, 4.0)).float()
    return s


def _prompt_rows(r):
    """Which of a policy step's rows are prompt: one run of 64 of every 512."""
    return torch.arange(r, device=DEV) // 64 % 8 == 7


# ------------------------------------------------------------------------------------------------- plain forms


def _keep8(x):
    """The values that 8 bits hold: whole multiples, up to 127, of 2^(E - 6), where 2^E is the largest power of two
    that the largest magnitude of the 32 channels reaches."""
    d = x.shape[-1]
    y = torch.nn.functional.pad(x.float(), (0, -d % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = y.abs().amax(-1, keepdim=True)
    step = torch.ldexp(torch.ones_like(top), torch.frexp(top).exponent - 7)
    q = torch.round(y / step).clamp(-127, 127)
    return (q * step).flatten(-2)[..., :d]


def _block(s):
    h, y = s["h"].float(), s["y"].float()
    w_pre, w_post = s["w_pre"][:, None], s["w_post"][:, None]
    rho = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    add = y * rho * w_post * s["scale"][:, None, None]
    if s["gate"] != "none":
        a = s["gate_"].float()
        add = add * (torch.sigmoid(a) if s["gate"] == "sigmoid" else a * torch.sigmoid(a))
    ho = h + add
    r = torch.rsqrt(ho.square().mean(-1, keepdim=True) + EPS)
    return {"h": ho.to(s["h"].dtype), "u": (ho * r * w_pre).to(s["y"].dtype)}, rho, r


def _block_train(s):
    out, rho, r = _block(s)
    h, y, a = s["h"], s["y"], s["gate_"]
    if s["kept"] == "8bit":
        h, y, a = _keep8(h), _keep8(y), None if a is None else _keep8(a)
    w_pre, w_post, scale = s["w_pre"][:, None], s["w_post"][:, None], s["scale"][:, None, None]
    yn = y.float() * rho
    if a is None:
        gate, slope = torch.ones_like(yn), None
    else:
        a = a.float()
        gate = torch.sigmoid(a)
        slope = gate * (1 - gate)
        if s["gate"] == "silu":
            slope = gate + a * slope
            gate = a * gate
    hn = (h.float() + scale * gate * yn * w_post) * r
    du = s["du"].float()
    flow = du * w_pre
    dh = s["dh_out"].float() + r * (flow - hn * (hn * flow).mean(-1, keepdim=True))
    dyn = dh * scale * gate * w_post
    dy = rho * (dyn - yn * (yn * dyn).mean(-1, keepdim=True))
    part = (dh * gate * yn).sum(1)
    ta = s["y"].dtype
    out |= {"dh": dh.to(s["h"].dtype), "dy": dy.to(ta), "dw_pre": (du * hn).sum(1), "dw_post": part * s["scale"][:, None],
            "dscale": (part * s["w_post"]).sum(1)}
    if slope is not None:
        out["dgate"] = (dh * scale * slope * yn * w_post).to(ta)
    return out


def _logprob(s):
    """(log-probability of each row's token, or 0 without one; exponentials of the row and their sum; the rows that have one)."""
    z = s["z"].float() / s.get("temperature", 1.0)
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    live = (s["token"] >= 0) & (s["token"] < s["v"])
    tok = torch.where(live, s["token"], 0).long()[:, None]
    lp = torch.where(live, (z.gather(1, tok) - top - total.log())[:, 0], 0)
    return lp, e, total, live, tok


def _through(e, total, tok, by):
    """by (one-hot - softmax), row by row."""
    dz = e * (-by[:, None] / total)
    return dz.scatter_add_(1, tok, by[:, None])


def _policy(s):
    lp, e, total, live, tok = _logprob(s)
    adv = s["advantage"]
    ratio = (lp - s["old"]).exp()
    plain, clipped = ratio * adv, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv
    loss = -torch.minimum(plain, clipped)
    slope = torch.where(plain <= clipped, -plain, 0)
    if s["ref"]:
        x = s["ref_"] - lp
        loss = loss + s["kl"] * (torch.expm1(x) - x)
        slope = slope - s["kl"] * torch.expm1(x)
    out = {"loss": torch.where(live, s["weight"] * loss, 0)}
    if s["grad"]:
        by = torch.where(live, s["weight"] * slope, 0) / s["temperature"]
        out["dz"] = _through(e, total, tok, by).to(s["z"].dtype)
    return out


def _prefer(s):
    lp, e, total, live, tok = _logprob(s)
    bounds, pairs = s["bounds"].long(), s["pairs"]
    of = torch.bucketize(torch.arange(s["r"], device=DEV), bounds[1:], right=True)
    sums = torch.zeros(2 * pairs + 1, device=DEV, dtype=torch.float64).index_add_(0, of, lp.double())[:-1]
    by = torch.ones(2 * pairs, device=DEV, dtype=torch.float64)
    if s["average"]:
        count = torch.zeros(2 * pairs + 1, device=DEV, dtype=torch.float64).index_add_(0, of, live.double())[:-1]
        by = 1 / count.clamp_min(1)
        sums = sums * by
    ratio = sums if s["ref_"] is None else sums - s["ref_"].double()
    m = BETA * (ratio[0::2] - ratio[1::2])
    # log sigma(m), by the side on which the exponential stays small
    loss = (torch.log1p((-m.abs()).exp()) + (-m).clamp_min(0)).float()
    out = {"loss": loss, "logp": sums.float()}
    if s["grad"]:
        slope = -BETA / (1 + m.exp())
        share = torch.stack([slope, -slope], 1).flatten() * by
        row = torch.where(live, torch.cat([share, share.new_zeros(1)])[of], 0)
        out["dz"] = _through(e, total, tok, row.float()).to(s["z"].dtype)
    return out


def run(s):
    op = s["op"]
    if own:
        import paper_2306_00256_b200 as ceca
        if op == "keep8":
            return ceca.dsgd_bring8(ceca.dsgd_keep8(s["x"]), s["d"], s["x"].dtype)
        if op in ("block", "block_train"):
            act = {"none": None, "sigmoid": ceca.GATE_SIGMOID, "silu": ceca.GATE_SILU}[s["gate"]]
            more = {"gate_act": act or ceca.GATE_SIGMOID, "scale": s["scale"]}
            train, kept = op == "block_train", (s["h"], s["y"], s["gate_"])
            h, u, stats, packed = ceca.dsgd_block_norm(s["h"], s["y"], s["w_pre"], s["w_post"], gate=s["gate_"], eps=EPS,
                                                       save=train, keep8=train and s["kept"] == "8bit", **more)
            out = {"h": h, "u": u}
            if train:
                hk, yk, ak = kept if packed is None else packed
                dh, dy, dgate, dw_pre, dw_post, dscale = ceca.dsgd_block_norm_grad(hk, yk, s["w_pre"], s["w_post"], stats, s["du"],
                                                                                   s["dh_out"], gate=ak, **more)
                out |= {"dh": dh, "dy": dy, "dw_pre": dw_pre, "dw_post": dw_post, "dscale": dscale}
                if dgate is not None:
                    out["dgate"] = dgate
            return out
        if op == "logprob":
            return {"logp": ceca.dsgd_token_logprob(s["z"], s["token"], s["temperature"])}
        if op == "policy":
            more = {"ref_logp": s["ref_"], "weight": s["weight"], "temperature": s["temperature"], "clip_low": CLIP[0], "clip_high": CLIP[1],
                    "kl": s["kl"]}
            if not s["grad"]:
                return {"loss": ceca.dsgd_policy_loss(s["z"], s["token"], s["old"], s["advantage"], **more)}
            loss, dz = ceca.dsgd_policy_grad(s["z"], s["token"], s["old"], s["advantage"], **more)
            return {"loss": loss, "dz": dz}
        more = {"ref_logp": s["ref_"], "beta": BETA, "average": s["average"]}
        if not s["grad"]:
            loss, logp = ceca.dsgd_preference_loss(s["z"], s["token"], s["bounds"], **more)
            return {"loss": loss, "logp": logp}
        loss, logp, dz = ceca.dsgd_preference_grad(s["z"], s["token"], s["bounds"], **more)
        return {"loss": loss, "logp": logp, "dz": dz}
    if op == "keep8":
        return _keep8(s["x"]).to(s["x"].dtype)
    if op == "block":
        return _block(s)[0]
    if op == "block_train":
        return _block_train(s)
    if op == "logprob":
        return {"logp": _logprob(s)[0]}
    return _policy(s) if op == "policy" else _prefer(s)


# ------------------------------------------------------------------------------------------------- work


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    op = case["op"]
    if op in ("block", "block_train", "keep8"):
        n, t, d, a = case["n"], case["t"], case["d"], size[case["act"]]
        rows, held = n * t * d, n * t * (d + -(-d // BLOCK))
        if op == "keep8":
            return {"bytes": 2 * rows * a + 2 * held, "flops": 4 * rows}
        e, gate = size[case["stream"]], case["gate"] != "none"
        more = 2 * n * d * 4 + n * 4
        forward = rows * (2 * e + (2 + gate) * a) + more
        if op == "block":
            return {"bytes": forward, "flops": 16 * rows}
        # backward: what was kept, du and dh_out read; dh, dy, dgate and the weights' gradients written
        kept = held * (2 + gate) if case["kept"] == "8bit" else rows * (e + (1 + gate) * a)
        forward += n * t * 8 + (kept if case["kept"] == "8bit" else 0)
        return {"bytes": forward + kept + n * t * 8 + rows * (2 * e + (2 + gate) * a) + 2 * more, "flops": 50 * rows}
    r, v, e = case["r"], case["v"], size[case["dtype"]]
    small = r * size[case["tokens"]]
    if op == "logprob":
        live = r * 0.98
        small += 4 * r
    elif op == "policy":
        live = r - sum(i // 64 % 8 == 7 for i in range(r))
        small += 4 * r * (4 + case["ref"])
    else:
        live = (r - r // 32) * 0.75
        small += (2 * case["pairs"] + 1) * size[case["tokens"]] + case["pairs"] * 4 * (3 + 2 * case["ref"])
    if not case.get("grad"):
        return {"bytes": int(live * v * e + small), "flops": int(4 * live * v)}
    return {"bytes": int((live + r) * v * e + small), "flops": int(8 * live * v)}


# ------------------------------------------------------------------------------------------------- 64 bits


def _held_values(x):
    """As _keep8, by logarithms and halves in 64 bits."""
    d = x.shape[-1]
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    for c0 in range(0, d, BLOCK):
        part = x[..., c0:c0 + BLOCK].double()
        top = part.abs().max(-1, keepdim=True).values
        power = torch.floor(torch.log2(top))
        power = power + (torch.exp2(power + 1) <= top).double() - (torch.exp2(power) > top).double()
        unit = torch.where(top > 0, torch.exp2(power - 6), 1.0)
        out[..., c0:c0 + BLOCK] = torch.clamp(torch.round(part / unit), min=-127, max=127) * unit
    return out


def _exact_block(s, i, train):
    """One agent's outputs."""
    h, y = s["h"][i].double(), s["y"][i].double()
    w_pre, w_post, scale = s["w_pre"][i].double(), s["w_post"][i].double(), s["scale"][i].double()
    d = h.shape[1]

    def gates(a):
        if a is None:
            return 1.0, 0.0
        sig = 1 / (1 + torch.exp(-a))
        if s["gate"] == "sigmoid":
            return sig, sig / (1 + torch.exp(a))
        return a * sig, sig * (1 + a / (1 + torch.exp(a)))

    a = None if s["gate_"] is None else s["gate_"][i].double()
    rho = 1 / torch.sqrt((y * y).sum(1, keepdim=True) / d + EPS)
    ho = h + scale * gates(a)[0] * (y * rho) * w_post
    r = 1 / torch.sqrt((ho * ho).sum(1, keepdim=True) / d + EPS)
    out = {"h": ho, "u": ho * r * w_pre}
    if not train:
        return out
    if s["kept"] == "8bit":
        h, y, a = _held_values(s["h"][i]), _held_values(s["y"][i]), None if a is None else _held_values(s["gate_"][i])
    g, slope = gates(a)
    yn = y * rho
    ho = h + scale * g * yn * w_post
    du = s["du"][i].double()
    back = du * w_pre * r
    dh = s["dh_out"][i].double() + back - ho * r * r * ((ho * back).sum(1, keepdim=True) / d)
    back = dh * scale * g * w_post * rho
    out["dh"] = dh
    out["dy"] = back - yn * rho * ((y * back).sum(1, keepdim=True) / d)
    out["dw_pre"] = (du * ho * r).sum(0)
    out["dw_post"] = scale * (dh * g * yn).sum(0)
    out["dscale"] = (dh * g * yn * w_post).sum()
    if a is not None:
        out["dgate"] = dh * scale * slope * yn * w_post
    return out


def _exact_logprob(s):
    tau = s.get("temperature", 1.0)
    lp = torch.zeros(s["r"], dtype=torch.float64, device=DEV)
    for r0 in range(0, s["r"], 1024):
        at = slice(r0, r0 + 1024)
        z = s["z"][at].double() / tau
        tok = s["token"][at].long()
        lp[at] = torch.where(tok >= 0, z.gather(1, tok.clamp_min(0)[:, None])[:, 0] - torch.logsumexp(z, 1), 0.0)
    return lp


def _exact_dz(s, slope):
    """slope / T (one-hot - softmax), some rows at a time; the slope of a row without a token is 0."""
    tau = s.get("temperature", 1.0)
    dz = torch.empty((s["r"], s["v"]), dtype=torch.float64, device=DEV)
    for r0 in range(0, s["r"], 1024):
        at = slice(r0, r0 + 1024)
        by = slope[at, None] / tau
        z = s["z"][at].double() / tau
        dz[at] = -by * torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
        dz[at].scatter_add_(1, s["token"][at].long().clamp_min(0)[:, None], by)
    return dz


def _exact_policy(s):
    lp, live = _exact_logprob(s), s["token"] >= 0
    adv, ratio = s["advantage"].double(), torch.exp(lp - s["old"].double())
    low, high = 1 - CLIP[0], 1 + CLIP[1]
    free = torch.where(adv >= 0, ratio <= high, ratio >= low)
    inside = torch.where(free, ratio, torch.where(adv >= 0, high, low))
    loss, slope = -inside * adv, torch.where(free, -ratio * adv, 0.0)
    if s["ref"]:
        x = s["ref_"].double() - lp
        loss, slope = loss + s["kl"] * (torch.exp(x) - 1 - x), slope + s["kl"] * (1 - torch.exp(x))
    w = torch.where(live, s["weight"].double(), 0.0)
    out = {"loss": w * loss}
    if s["grad"]:
        out["dz"] = _exact_dz(s, w * slope)
    return out


def _exact_prefer(s):
    lp, live = _exact_logprob(s), s["token"] >= 0
    cut = s["bounds"].tolist()
    slope = torch.zeros_like(lp)
    loss, logp = [], []
    for p in range(s["pairs"]):
        spans = [slice(cut[2 * p + k], cut[2 * p + k + 1]) for k in (0, 1)]
        counts = [max(1, int(live[a].sum())) if s["average"] else 1 for a in spans]
        sums = [float(lp[a].sum()) / c for a, c in zip(spans, counts)]
        m = BETA * (sums[0] - sums[1])
        if s["ref_"] is not None:
            m -= BETA * (float(s["ref_"][2 * p]) - float(s["ref_"][2 * p + 1]))
        loss.append(math.log1p(math.exp(-m)) if m > 0 else -m + math.log1p(math.exp(m)))
        logp += sums
        down = BETA / (1 + math.exp(m)) if m < 700 else 0.0
        slope[spans[0]] = -down / counts[0]
        slope[spans[1]] = down / counts[1]
    out = {"loss": torch.tensor(loss, dtype=torch.float64, device=DEV), "logp": torch.tensor(logp, dtype=torch.float64, device=DEV)}
    if s["grad"]:
        out["dz"] = _exact_dz(s, torch.where(live, slope, 0.0))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "keep8":
        return _held_values(s["x"])
    if case["op"] in ("block", "block_train"):
        parts = [_exact_block(s, i, case["op"] == "block_train") for i in range(case["n"])]
        return {k: torch.stack([p[k] for p in parts]) for k in parts[0]}
    if case["op"] == "logprob":
        return {"logp": _exact_logprob(s)}
    return _exact_policy(s) if case["op"] == "policy" else _exact_prefer(s)
