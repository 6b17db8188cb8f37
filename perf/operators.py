"""What the language-model training operators are measured on, and their plain forms.

Three operators, each with its gradient: the embedding lookup of every agent, the gated linear recurrence over
a sequence, and the distillation loss against a teacher's top logits.  `n` agents train side by side, so a table
is n x V x D, a batch of sequences n * batch, and the rows of the logits are all agents' positions.

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

# Every EMPTY-th row of the logits carries weight zero: a position of the prompt or of the padding.
EMPTY = 16


def listed():
    return [
        # The lookup of a few short sequences: what an agent does per decoded chunk or in a smoke run; latency counts.
        {"name": "lookup_small", "op": "lookup", "n": 4, "t": 64, "v": 4096, "d": 256, "table": "f32", "out": "f32", "tokens": "i32"},
        # A training batch's lookup: eight agents with tables in 16 bits, one packed sequence of 8192 tokens each.
        {"name": "lookup_large", "op": "lookup", "n": 8, "t": 8192, "v": 32000, "d": 2048, "table": "bf16", "out": "bf16", "tokens": "i64"},
        # The gradient of a short batch on a small vocabulary of odd size: a dense gradient row for every table row.
        {"name": "embed_grad_small", "op": "embed_grad", "n": 4, "t": 129, "v": 4097, "d": 256, "table": "f32", "out": "f32", "tokens": "i64"},
        # The gradient of a training batch: activations' gradients in 16 bits, the agents' gradient matrix in 32.
        {"name": "embed_grad_large", "op": "embed_grad", "n": 8, "t": 8192, "v": 32000, "d": 1024, "table": "f32", "out": "bf16", "tokens": "i32"},
        # One new token for each of 256 sequences that are being answered, from their kept states.
        {"name": "recur_token", "op": "recur", "b": 256, "t": 1, "d": 2048, "dtype": "bf16", "h0": True, "starts": False},
        # One long document read by one agent: few channels, a long axis.
        {"name": "recur_long", "op": "recur", "b": 1, "t": 32768, "d": 1024, "dtype": "bf16", "h0": False, "starts": False},
        # A training step of eight agents on packed documents, forward and backward.
        {"name": "recur_train", "op": "recur_train", "b": 8, "t": 4096, "d": 2048, "dtype": "bf16", "h0": False, "starts": True},
        # Odd length and width in 32 bits, from a carried state: the tail of a document, rows that are not 16-byte aligned.
        {"name": "recur_train_odd", "op": "recur_train", "b": 3, "t": 1537, "d": 771, "dtype": "f32", "h0": True, "starts": False},
        # Evaluation: the loss alone, a vocabulary of odd size in 32 bits, the teacher renormalised over what it sent.
        {"name": "distill_loss_odd", "op": "distill_loss", "r": 2047, "v": 50001, "k": 16, "dtype": "f32", "tail": False, "temperature": 2.0},
        # The step of a small vocabulary and few positions; latency counts.
        {"name": "distill_grad_small", "op": "distill_grad", "r": 64, "v": 1000, "k": 8, "dtype": "f32", "tail": True, "temperature": 1.0},
        # An odd vocabulary in 16 bits, in rows without padding.
        {"name": "distill_grad_odd", "op": "distill_grad", "r": 2047, "v": 50001, "k": 50, "dtype": "bf16", "tail": False, "temperature": 1.5},
        # A training step over a large vocabulary: eight agents with 1024 positions each, and the teacher's remaining mass.
        {"name": "distill_grad_large", "op": "distill_grad", "r": 8192, "v": 128000, "k": 64, "dtype": "bf16", "tail": True, "temperature": 1.0},
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; odd ones and multiples of eight both come often."""
    x = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    x = x // 8 * 8 if rng.random() < 0.5 else x | 1
    return min(hi, max(lo, x))


def draw(rng):
    op = rng.choice(["lookup", "embed_grad", "recur", "recur_train", "distill_loss", "distill_grad"])
    if op in ("lookup", "embed_grad"):
        case = {"op": op, "n": rng.randint(1, 8), "v": _log_int(rng, 1000, 131072), "d": _log_int(rng, 64, 4096),
                "table": rng.choice(["f32", "bf16"]), "out": rng.choice(["f32", "bf16"]), "tokens": rng.choice(["i32", "i64"])}
        while case["n"] * case["v"] * case["d"] > 8 * 32000 * 1024:
            case["v"] = max(1000, case["v"] // 2 + 1)
            case["n"] = max(1, case["n"] // 2)
        most = min(65536, 8 * 8192 * 2048 // (case["n"] * case["d"]))
        case["t"] = _log_int(rng, 1, most)
        return case
    if op in ("recur", "recur_train"):
        case = {"op": op, "b": _log_int(rng, 1, 64), "d": _log_int(rng, 64, 4096), "dtype": rng.choice(["f32", "bf16"]),
                "h0": rng.random() < 0.5, "starts": rng.random() < 0.5}
        most = min(32768, 8 * 4096 * 2048 // (case["b"] * case["d"]))
        case["t"] = _log_int(rng, 1, most)
        if op == "recur" and rng.random() < 0.25:  # one new token for each of many sequences
            case["t"], case["b"] = 1, _log_int(rng, 1, 1024)
        return case
    case = {"op": op, "v": _log_int(rng, 500, 131072), "k": _log_int(rng, 1, 128), "dtype": rng.choice(["f32", "bf16"]),
            "tail": rng.random() < 0.5, "temperature": rng.choice([0.7, 1.0, 2.0, 4.0])}
    case["r"] = _log_int(rng, 16, min(16384, (512 << 20) // case["v"]))
    return case


# ------------------------------------------------------------------------------------------------- inputs


def _normal(g, shape, dtype=torch.float32, mean=0.0, std=1.0):
    x = torch.empty(shape, device=DEV, dtype=dtype)
    return x.normal_(mean, std, generator=g)


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    s = dict(case)
    if case["op"] in ("lookup", "embed_grad"):
        n, t, v, d = case["n"], case["t"], case["v"], case["d"]
        # token frequencies fall as 1 / rank; about one position in 50 is empty (-1)
        u = torch.rand((n, t), device=DEV, generator=g)
        tok = ((u * math.log(v + 1)).exp() - 1).long().clamp_(0, v - 1)
        tok[torch.rand((n, t), device=DEV, generator=g) < 0.02] = -1
        s["tok"] = tok.to(TOKENS[case["tokens"]])
        s["scale"] = math.sqrt(d)
        if case["op"] == "lookup":
            s["table_"] = _normal(g, (n, v, d), DTYPES[case["table"]], 0.0, 0.02)
        else:
            s["dout"] = _normal(g, (n, t, d), DTYPES[case["out"]], 0.0, 1e-2)
    elif case["op"] in ("recur", "recur_train"):
        b, t, d, dt = case["b"], case["t"], case["d"], DTYPES[case["dtype"]]
        s["x"] = _normal(g, (b, t, d), dt)
        s["f"] = _normal(g, (b, t, d), dt, 2.0, 1.5)  # gates that keep most of the state, as trained ones do
        s["h0_"] = _normal(g, (b, d)) if case["h0"] else None
        s["starts_"] = None
        if case["starts"]:  # documents of some 500 tokens, packed
            s["starts_"] = (torch.rand((b, t), device=DEV, generator=g) < 0.002).to(torch.uint8)
        if case["op"] == "recur_train":
            s["dh"] = _normal(g, (b, t, d), dt, 0.0, 1e-2)
            s["dlast"] = _normal(g, (b, d), torch.float32, 0.0, 1e-2)
    else:
        r, v, k, dt = case["r"], case["v"], case["k"], DTYPES[case["dtype"]]
        first = torch.randint(0, v, (r, 1), device=DEV, generator=g)
        idx = (first + torch.arange(k, device=DEV) * max(1, v // k - 1)) % v
        t = _normal(g, (r, k), torch.float32, 0.0, 0.5) + 8.0 - 4.0 * torch.arange(k, device=DEV) / k
        z = _normal(g, (r, v), dt, 0.0, 1.5)
        z.scatter_add_(1, idx, (0.7 * t).to(dt))  # the student has learnt some of it
        gone = torch.rand((r, k), device=DEV, generator=g) < 0.05
        gone[:, 0] = False
        idx[gone] = -1  # the teacher sent fewer
        s["z"], s["idx"], s["t_"] = z, idx.to(torch.int32), t
        s["lse"] = None
        if case["tail"]:
            # the teacher's own normaliser over its whole vocabulary, at this temperature: some 5 to 10 % lie outside its top
            s["lse"] = (t / case["temperature"]).masked_fill(gone, -math.inf).exp().sum(1).log() + 0.05 + 0.05 * torch.rand(r, device=DEV, generator=g)
        w = torch.rand(r, device=DEV, generator=g) / r
        w[EMPTY - 1::EMPTY] = 0.0
        s["weight"] = w
    return s


# ------------------------------------------------------------------------------------------------- plain forms


def _lookup(s):
    ok = (s["tok"] >= 0) & (s["tok"] < s["v"])
    agent = torch.arange(s["n"], device=DEV)[:, None]
    rows = s["table_"][agent, torch.where(ok, s["tok"], 0).long()]
    return (rows.float() * s["scale"] * ok[:, :, None]).to(DTYPES[s["out"]])


def _embed_grad(s):
    n, v, d = s["n"], s["v"], s["d"]
    ok = (s["tok"] >= 0) & (s["tok"] < v)
    row = torch.where(ok, s["tok"], 0).long() + torch.arange(n, device=DEV)[:, None] * v
    part = s["dout"].float() * s["scale"] * ok[:, :, None]
    grad = torch.zeros((n * v, d), device=DEV).index_add_(0, row.reshape(-1), part.reshape(-1, d))
    return grad.reshape(n, v, d).to(DTYPES[s["table"]])


def _scan(c, b):
    """h_t = c_t h_{t-1} + b_t along dimension 1 from h_{-1} = 0: log2(t) doublings, in place on its arguments."""
    span = 1
    while span < c.shape[1]:
        b[:, span:] += c[:, span:] * b[:, :-span]
        c[:, span:] = c[:, span:] * c[:, :-span]
        span *= 2
    return b


def _gates(s):
    a = torch.sigmoid(s["f"].float())
    keep = a if s["starts_"] is None else a * (s["starts_"] == 0)[:, :, None]
    b = torch.sigmoid(-s["f"].float()) * s["x"].float()
    if s["h0_"] is not None:
        b[:, 0] += keep[:, 0] * s["h0_"]
    return a, keep, b


def _recur(s):
    _, keep, b = _gates(s)
    h = _scan(keep.clone(), b)
    return {"h": h.to(s["x"].dtype), "last": h[:, -1].clone()}


def _recur_train(s):
    a, keep, b = _gates(s)
    h = _scan(keep.clone(), b)
    lam = s["dh"].float().clone()  # (a tensor of 32 bits is its own float(), and the inputs stay as they are)
    lam[:, -1] += s["dlast"]
    after = torch.zeros_like(keep)
    after[:, :-1] = keep[:, 1:]
    lam = _scan(after.flip(1), lam.flip(1)).flip(1)
    before = torch.zeros_like(h)
    before[:, 1:] = h[:, :-1]
    if s["h0_"] is not None:
        before[:, 0] = s["h0_"]
    if s["starts_"] is not None:
        before = before * (s["starts_"] == 0)[:, :, None]
    one = torch.sigmoid(-s["f"].float())
    dt = s["x"].dtype
    return {"h": h.to(dt), "last": h[:, -1].clone(), "dx": (one * lam).to(dt), "df": (lam * (before - s["x"].float()) * a * one).to(dt),
            "dh0": keep[:, 0] * lam[:, 0]}


def _distill(s, grad):
    tau = s["temperature"]
    z = s["z"].float() / tau
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    there = (s["idx"] >= 0) & (s["idx"] < s["v"])
    idx = torch.where(there, s["idx"], 0).long()
    t = torch.where(there, s["t_"] / tau, -math.inf)
    if s["tail"]:
        p = (t - s["lse"][:, None]).exp()
        rest = (1 - p.sum(1, keepdim=True)).clamp_min(0)
    else:
        p = (t - t.amax(1, keepdim=True)).exp()
        p = p / p.sum(1, keepdim=True)
    w = s["weight"][:, None]
    live = w != 0
    logq = z.gather(1, idx) - top - total.log()
    loss = torch.where(there, p * (torch.where(p > 0, p, 1).log() - logq), 0).sum(1, keepdim=True)
    if s["tail"]:
        mark = torch.zeros_like(z).scatter_add_(1, idx, there.float())
        e_rest = e * (mark == 0)
        outside = e_rest.sum(1, keepdim=True)
        loss = loss + torch.where(rest > 0, rest * (rest / (outside / total)).log(), 0)
    loss = torch.where(live, w * loss, 0)[:, 0]
    if not grad:
        return {"loss": loss}
    dz = e / total
    if s["tail"]:
        dz -= e_rest * (rest / outside)
    dz.scatter_add_(1, idx, torch.where(there, -p, 0))
    return {"loss": loss, "dz": torch.where(live, dz * (w / tau), 0).to(s["z"].dtype)}


def run(s):
    op = s["op"]
    if own:
        import paper_2306_00256_b200 as ceca
        if op == "lookup":
            return ceca.dsgd_embed_lookup(s["table_"], s["tok"], s["scale"], out_dtype=DTYPES[s["out"]])
        if op == "embed_grad":
            grad = torch.empty((s["n"], s["v"], s["d"]), dtype=DTYPES[s["table"]], device=DEV)
            return ceca.dsgd_embed_grad(s["dout"], s["tok"], grad, s["scale"])
        if op == "recur":
            h, last, _ = ceca.dsgd_recurrence(s["x"], s["f"], h0=s["h0_"], starts=s["starts_"])
            return {"h": h, "last": last}
        if op == "recur_train":
            h, last, marks = ceca.dsgd_recurrence(s["x"], s["f"], h0=s["h0_"], starts=s["starts_"], save=True)
            dx, df, dh0 = ceca.dsgd_recurrence_grad(s["x"], s["f"], s["dh"], marks, h0=s["h0_"], starts=s["starts_"], dh_last=s["dlast"])
            return {"h": h, "last": last, "dx": dx, "df": df, "dh0": dh0}
        more = {"teacher_lse": s["lse"], "weight": s["weight"], "temperature": s["temperature"]}
        if op == "distill_loss":
            return {"loss": ceca.dsgd_distill_loss(s["z"], s["idx"], s["t_"], **more)}
        loss, dz = ceca.dsgd_distill_grad(s["z"], s["idx"], s["t_"], **more)
        return {"loss": loss, "dz": dz}
    if op == "lookup":
        return _lookup(s)
    if op == "embed_grad":
        return _embed_grad(s)
    if op == "recur":
        return _recur(s)
    if op == "recur_train":
        return _recur_train(s)
    return _distill(s, op == "distill_grad")


# ------------------------------------------------------------------------------------------------- work


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    op = case["op"]
    if op in ("lookup", "embed_grad"):
        n, t, v, d = case["n"], case["t"], case["v"], case["d"]
        held = n * t * size[case["tokens"]] + n * t * d * size[case["out"]]
        if op == "embed_grad":
            return {"bytes": held + n * v * d * size[case["table"]], "flops": 2 * n * t * d}
        # distinct rows of t tokens whose frequency falls as 1 / rank, each read once
        seen = _distinct(t, v)
        return {"bytes": held + n * seen * d * size[case["table"]], "flops": n * t * d}
    if op in ("recur", "recur_train"):
        b, t, d, e = case["b"], case["t"], case["d"], size[case["dtype"]]
        small = b * d * 4 * (1 + case["h0"]) + (b * t if case["starts"] else 0)
        if op == "recur":
            return {"bytes": 3 * b * t * d * e + small, "flops": 8 * b * t * d}
        # forward: x, f read, h written; backward: x, f, dh read, dx, df written
        return {"bytes": 8 * b * t * d * e + 2 * small + 2 * b * d * 4, "flops": 24 * b * t * d}
    r, v, k, e = case["r"], case["v"], case["k"], size[case["dtype"]]
    live = r - r // EMPTY
    small = r * (8 * k + 8 + (4 if case["tail"] else 0))
    if op == "distill_loss":
        return {"bytes": live * v * e + small, "flops": 4 * live * v}
    return {"bytes": (live + r) * v * e + small, "flops": 8 * live * v}


def _distinct(t, v):
    """The expected number of distinct rows among t log-uniform tokens of v (98 % of them not empty)."""
    total, lo, scale = 0.0, 0, math.log(v + 1)
    while lo < v:  # rows in groups of like frequency
        hi = min(v, lo + max(1, lo // 64))
        p = math.log((hi + 1) / (lo + 1)) / scale / (hi - lo)
        total += (hi - lo) * -math.expm1(0.98 * t * math.log1p(-p)) if p < 1 else 1.0
        lo = hi
    return int(total)


# ------------------------------------------------------------------------------------------------- 64 bits


def _exact_lookup(s):
    out = torch.zeros((s["n"], s["t"], s["d"]), dtype=torch.float64, device=DEV)
    for i in range(s["n"]):
        at = torch.nonzero(s["tok"][i] >= 0)[:, 0]
        out[i, at] = torch.index_select(s["table_"][i], 0, s["tok"][i][at].long()).double() * s["scale"]
    return out


def _exact_embed_grad(s):
    out = torch.zeros((s["n"], s["v"], s["d"]), dtype=torch.float64, device=DEV)
    for i in range(s["n"]):
        tok, order = torch.sort(s["tok"][i].long(), stable=True)
        skip = int((tok < 0).sum())
        tok, order = tok[skip:], order[skip:]
        if not tok.numel():
            continue
        rows, counts = torch.unique_consecutive(tok, return_counts=True)
        upto = torch.cumsum(s["dout"][i][order].double(), 0)
        ends = torch.cumsum(counts, 0) - 1
        sums = upto[ends]
        sums[1:] -= upto[ends[:-1]]
        out[i, rows] = sums * s["scale"]
    return out


def _exact_recur(s, grad):
    x, f = s["x"], s["f"]
    b, t, d = x.shape
    h = torch.zeros((b, d), dtype=torch.float64, device=DEV) if s["h0_"] is None else s["h0_"].double()
    first = h
    hs = torch.empty((b, t, d), dtype=torch.float64, device=DEV)
    a = 1 / (1 + torch.exp(-f.double()))
    na = 1 / (1 + torch.exp(f.double()))
    took = na * x.double()
    go = None if s["starts_"] is None else 1.0 - s["starts_"].double()[:, :, None]
    kept = a if go is None else a * go
    for j in range(t):
        torch.addcmul(took[:, j], kept[:, j], h, out=hs[:, j])
        h = hs[:, j]
    out = {"h": hs, "last": h.clone()}
    if grad:
        lam = torch.empty_like(hs)
        dh = s["dh"].double()
        lam[:, t - 1] = dh[:, t - 1] + s["dlast"].double()
        for j in range(t - 2, -1, -1):
            torch.addcmul(dh[:, j], kept[:, j + 1], lam[:, j + 1], out=lam[:, j])
        out["dx"] = na * lam
        prev = torch.cat([first[:, None], hs[:, :-1]], 1)
        prev = prev if go is None else prev * go
        out["df"] = lam * (prev - x.double()) * a * na
        out["dh0"] = kept[:, 0] * lam[:, 0]
    return out


def _exact_distill(s, grad):
    tau = s["temperature"]
    loss = torch.zeros(s["r"], dtype=torch.float64, device=DEV)
    dz = torch.zeros((s["r"], s["v"]), dtype=torch.float64, device=DEV) if grad else None
    for r0 in range(0, s["r"], 512):
        at = slice(r0, r0 + 512)
        z = s["z"][at].double() / tau
        logq = z - torch.logsumexp(z, 1, keepdim=True)
        held = s["idx"][at] >= 0
        t = (s["t_"][at].double() / tau).masked_fill(~held, -math.inf)
        norm = s["lse"][at].double()[:, None] if s["tail"] else torch.logsumexp(t, 1, keepdim=True)
        logp = t - norm
        idx = s["idx"][at].long().clamp_min(0)
        p = logp.exp()
        terms = p * (logp - logq.gather(1, idx))
        kl = terms.masked_fill(~held, 0.0).sum(1)
        target = torch.zeros_like(z).scatter_add_(1, idx, p)
        if s["tail"]:
            inside = torch.zeros_like(z).scatter_add_(1, idx, held.double()) > 0
            rest = 1 - p.sum(1)
            logrest = torch.logsumexp(logq.masked_fill(inside, -math.inf), 1)
            kl = kl + torch.where(rest > 0, rest * (rest.clamp_min(1e-300).log() - logrest), 0.0)
            target = torch.where(inside, target, (logq - logrest[:, None]).exp() * rest.clamp_min(0)[:, None])
        w = s["weight"][at].double()
        loss[at] = torch.where(w != 0, w * kl, 0.0)
        if grad:
            dz[at] = torch.where(w[:, None] != 0, (logq.exp() - target) * (w / tau)[:, None], 0.0)
    return {"loss": loss, "dz": dz} if grad else {"loss": loss}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lookup":
        return _exact_lookup(s)
    if case["op"] == "embed_grad":
        return _exact_embed_grad(s)
    if case["op"] in ("recur", "recur_train"):
        return _exact_recur(s, case["op"] == "recur_train")
    return _exact_distill(s, case["op"] == "distill_grad")
