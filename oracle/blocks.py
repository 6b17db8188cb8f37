"""TEST INFRASTRUCTURE: 64-bit statements of the operators around a model's blocks and behind its logits, straight from their
definitions, and bounds on how far an fp32 evaluation may be from them (see oracle/lm.py for how they are counted).

Sums over d channels run over at most d / 64 terms in a row and a tree of less than 40, sums over rows over all of them.
"""
import numpy as np

from .lm import U, _gates, _out

SIGMOID, SILU = 0, 1


# ------------------------------------------------------------------------------------------- 8 bits


def kept(x):
    """The whole numbers, the powers E and the values of x's blocks of 32 along the last axis."""
    d = x.shape[-1]
    q, v = np.zeros(x.shape), np.zeros(x.shape)
    powers = []
    for c in range(0, d, 32):
        part = x[..., c:c + 32].astype(np.float64)
        bad = ~np.isfinite(part).all(-1, keepdims=True)
        top = np.where(bad, 1.0, np.abs(np.where(bad, 0.0, part)).max(-1, keepdims=True))
        e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1, -200)
        e = np.maximum(e, -121)
        unit = np.ldexp(1.0, e - 6)
        whole = np.clip(np.rint(np.where(bad, 0.0, part) / unit), -127, 127)
        q[..., c:c + 32] = whole
        v[..., c:c + 32] = np.where(bad, np.nan, whole * unit)
        powers.append(np.where(bad, 128, e)[..., 0])
    return q, np.stack(powers, -1), v


def kept_bytes(x):
    """The kept rows of x as they lie in memory."""
    q, powers, _ = kept(x)
    d = x.shape[-1]
    width = -(-(d + powers.shape[-1]) // 16) * 16
    out = np.zeros(x.shape[:-1] + (width,), np.uint8)
    out[..., :d] = q.astype(np.int8).view(np.uint8)
    out[..., d:d + powers.shape[-1]] = powers + 127
    return out


# ------------------------------------------------------------------------------------------- block norms


def _gate(a, act):
    """(factor, its error, derivative, its error)"""
    s, ns, eg = _gates(a)
    slope, es = s * ns, 2 * eg + 4 * U
    if act == SIGMOID:
        return s, eg * s, slope, es * slope
    return a * s, (eg + U) * np.abs(a * s), s + a * slope, eg * s + (es + U) * np.abs(a * slope) + U * np.abs(s + a * slope)


def _norm_error(d):
    return U * (24 + d / 128)


def _out_row(h, y, gate, w_post, scale, act, rho, erho):
    """h_out, its error, and the parts it is made of; rho with relative error erho."""
    if y is None:
        return h, np.zeros_like(h), None
    g, eg, slope, es = (np.ones_like(y), np.zeros_like(y), np.zeros_like(y), np.zeros_like(y)) if gate is None else _gate(gate, act)
    yn = y * rho
    by = scale[:, None, None] * w_post[:, None, :]
    add = by * g * yn
    out = h + add
    err = np.abs(by * yn) * eg + (erho + 5 * U) * np.abs(add) + U * np.abs(out)
    return out, err, (g, eg, slope, es, yn, by)


def block_norm(h, y, w_pre, w_post, gate=None, act=SIGMOID, scale=None, eps=1e-6, stream16=False, act16=False):
    """{name: (want, tolerance)} of h_out, u and stats (only what there is)."""
    n, t, d = h.shape
    scale = np.ones(n) if scale is None else scale
    rel = _norm_error(d)
    rho = 0.0 if y is None else 1 / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    ho, eh, _ = _out_row(h, y, gate, w_post, scale, act, rho, rel)
    out = {}
    if y is not None:
        out["h"] = _out(ho, eh, stream16)
    stats = np.zeros((n, t, 2))
    es = np.zeros((n, t, 2))
    stats[..., :1], es[..., :1] = rho, rel * np.abs(rho)
    if w_pre is not None:
        ms = (ho * ho).mean(-1, keepdims=True) + eps
        r = 1 / np.sqrt(ms)
        er = rel + np.sqrt((eh * eh).mean(-1, keepdims=True) / ms)
        u = ho * r * w_pre[:, None, :]
        out["u"] = _out(u, np.abs(r * w_pre[:, None, :]) * eh + (er + 4 * U) * np.abs(u), act16)
        stats[..., 1:], es[..., 1:] = r, er * r
    out["stats"] = _out(stats, es, False)
    return out


def block_norm_grad(h, y, w_pre, w_post, stats, du, dh_out=None, gate=None, act=SIGMOID, scale=None, stream16=False, act16=False, weights16=False,
                    before=None):
    """{name: (want, tolerance)}; stats as given to the call, exact."""
    n, t, d = h.shape
    sc = np.ones(n) if scale is None else scale
    rho, r = stats[..., :1], stats[..., 1:]
    ho, eh, parts = _out_row(h, y, gate, w_post, sc, act, rho, U)
    rows = 43 + d / 64   # roundings of a mean over channels
    past = np.zeros_like(h) if dh_out is None else dh_out
    out = {}
    if w_pre is not None:
        wp = w_pre[:, None, :]
        hn, ehn = ho * r, eh * r + U * np.abs(ho * r)
        flow = wp * du
        m = (hn * flow).mean(-1, keepdims=True)
        em = (ehn * np.abs(flow)).mean(-1, keepdims=True) + rows * U * np.abs(hn * flow).mean(-1, keepdims=True)
        turn = r * (flow - hn * m)
        dh = past + turn
        edh = r * (3 * U * np.abs(flow) + np.abs(m) * ehn + np.abs(hn) * em + 3 * U * np.abs(hn * m)) + 2 * U * (np.abs(turn) + np.abs(dh))
        edw = (np.abs(du) * ehn).sum(1) + (t + 40) * U * np.abs(hn * du).sum(1)
        out["dw_pre"] = ((hn * du).sum(1), edw)
    else:
        dh, edh = past, np.zeros_like(h)
    out["dh"] = _out(dh, edh, stream16)
    if y is not None:
        g, eg, slope, es, yn, by = parts
        eyn = U * np.abs(yn)
        e = by * g * dh
        ee = np.abs(by * g) * edh + np.abs(by * dh) * eg + 4 * U * np.abs(e)
        m = (yn * e).mean(-1, keepdims=True)
        em = (np.abs(yn) * ee + np.abs(e) * eyn).mean(-1, keepdims=True) + rows * U * np.abs(yn * e).mean(-1, keepdims=True)
        if w_pre is not None:   # mean(yn e) may be mean(q (dh_out + r w_pre du)) - r mean(hn w_pre du) mean(q hn), q = s g w_post yn: sums of their own
            q, m1 = np.abs(by * g * yn), np.abs((hn * flow).mean(-1, keepdims=True))
            em = em + rows * U * ((q * (np.abs(past) + r * np.abs(flow))).mean(-1, keepdims=True) + r * m1 * (q * np.abs(hn)).mean(-1, keepdims=True))
        dy = rho * (e - yn * m)
        out["dy"] = _out(dy, rho * (ee + np.abs(m) * eyn + np.abs(yn) * em + 3 * U * (np.abs(e) + np.abs(yn * m))) + 2 * U * np.abs(dy), act16)
        if gate is not None:
            da = by * slope * yn * dh
            out["dgate"] = _out(da, np.abs(by * slope * yn) * edh + np.abs(by * yn * dh) * es + 5 * U * np.abs(da), act16)
        part = yn * g * dh
        ep = np.abs(yn * g) * edh + np.abs(yn * dh) * eg + 4 * U * np.abs(part)
        s, esum = part.sum(1), ep.sum(1) + (t + 40) * U * np.abs(part).sum(1)
        out["dw_post"] = (sc[:, None] * s, np.abs(sc[:, None]) * esum + 2 * U * np.abs(sc[:, None] * s))
        if scale is not None:
            w = w_post
            mag = (np.abs(part).sum(1) * np.abs(w)).sum(1)
            out["dscale"] = ((w * s).sum(1), (np.abs(w) * ep.sum(1)).sum(1) + (t + d + 60) * U * mag)
    for k in ("dw_pre", "dw_post", "dscale"):
        if k in out:
            want, err = out[k]
            if before is not None:
                want, err = want + before[k], err + U * (np.abs(want) + np.abs(before[k]))
            out[k] = _out(want, err, weights16)
    return out


# ------------------------------------------------------------------------------------------- tokens' log-probabilities


def _rows(z, tokens, temperature):
    """For each row: log q and 1 - q of its token with their errors, all q, and relative bounds of q elsewhere."""
    r, v = z.shape
    logp, elog, other, eother = (np.zeros(r) for _ in range(4))
    q, rq = np.zeros((r, v)), np.zeros((r, v))
    live = (tokens >= 0) & (tokens < v)
    for i in np.flatnonzero(live):
        k = int(tokens[i])
        if not np.isfinite(z[i][z[i] > -np.inf]).all():
            logp[i], other[i], q[i] = np.nan, np.nan, np.nan
            continue
        y = z[i] / temperature
        top = y.max()
        if top == -np.inf:
            logp[i], other[i] = -np.inf, 1.0
            continue
        e = np.exp(y - top)
        total = e.sum()
        q[i] = e / total
        rest = total - e[k] if e[k] < 0.5 * total else np.delete(e, k).sum()
        other[i] = rest / total
        logp[i] = y[k] - top - np.log(total) if other[i] > 0.5 else np.log1p(-other[i])   # (e[k] may be too small for 64 bits)
        away = np.where(e > 0, top - np.where(np.isfinite(y), y, top), 0.0)
        # an exponent's rounding grows with its distance from the frame, which is near the others' maximum
        own = top - np.delete(y, k).max() if v > 1 else 0.0
        own = own if np.isfinite(own) else 0.0
        dist = U * (4 * (away + own) + 100)
        rsum = (np.delete(e * dist, k).sum() / rest if rest > 0 else 0.0) + U * (40 + v / 64)
        delta = rsum + dist[k] + 8 * U * (1 + abs(logp[i]) + away[k] + own if np.isfinite(logp[i]) else 1)
        elog[i] = other[i] * delta + 4 * U * abs(logp[i]) if np.isfinite(logp[i]) else 0.0
        eother[i] = other[i] * ((1 - other[i]) * delta + 6 * U)
        rq[i] = dist + rsum + delta * (1 - other[i]) + 12 * U
    return live, logp, elog, other, eother, q, rq


def token_logprob(z, tokens, temperature=1.0):
    _, logp, elog, _, _, _, _ = _rows(z, tokens, temperature)
    return _out(logp, elog, False)


def _turned(tokens, c, ec, rows, temperature, bf16):
    live, _, _, other, eother, q, rq = rows
    with np.errstate(invalid="ignore"):
        dz = -(c[:, None] / temperature) * q
        tol = (np.abs(c[:, None]) * rq + ec[:, None]) * q / temperature
        for i in np.flatnonzero(live):
            k = int(tokens[i])
            dz[i, k] = c[i] / temperature * other[i]
            tol[i, k] = (abs(c[i]) * (eother[i] + 4 * U * other[i]) + ec[i] * other[i]) / temperature
        off = (c == 0) & (ec == 0)
        dz[off] = 0.0
        tol[off] = 0.0
        return _out(dz, tol + 4 * U * np.abs(dz), bf16)


def policy(z, tokens, old, adv, ref=None, weight=None, temperature=1.0, low=0.2, high=0.2, kl=0.0, bf16=False):
    """{name: (want, tolerance)} of loss, logp and dz."""
    r, v = z.shape
    w = np.ones(r) if weight is None else weight.astype(np.float64)
    tokens = np.where(w != 0, tokens, -1)
    rows = _rows(z, tokens, temperature)
    live, l, el = rows[0], rows[1], rows[2]
    lo, hi = np.float64(np.float32(1) - np.float32(low)), np.float64(np.float32(1) + np.float32(high))
    with np.errstate(over="ignore", invalid="ignore"):
        p = np.exp(l - old)
        ep = p * (el + U * (np.abs(l) + np.abs(old)) + 6 * U)
        free = ~(p * adv > np.clip(p, lo, hi) * adv)
        loss = -np.where(free, p, np.clip(p, lo, hi)) * adv
        eloss = np.where(free, ep, 0.0) * np.abs(adv) + 2 * U * np.abs(loss)
        c, ec = np.where(free, -p * adv, 0.0), np.where(free, ep * np.abs(adv) + 2 * U * np.abs(p * adv), 0.0)
        if ref is not None and kl:
            x = ref - l
            ex = el + U * (np.abs(ref) + np.abs(l))
            m = np.expm1(x)
            ekl = np.exp(x) * ex + 4 * U * np.abs(m)
            loss, eloss = loss + kl * (m - x), eloss + kl * (np.abs(m) * ex + 4 * U * np.abs(m) + 4 * U * (np.abs(m) + np.abs(x))) + 2 * U * np.abs(loss)
            c, ec = c - kl * m, ec + kl * ekl + 4 * U * (np.abs(c) + np.abs(kl * m))
        loss, eloss, c, ec = w * loss, np.abs(w) * (eloss + 2 * U * np.abs(loss)), w * c, np.abs(w) * (ec + 2 * U * np.abs(c))
    for a in (loss, eloss, c, ec):
        a[~live] = 0.0
    return {"loss": _out(loss, eloss, False), "logp": _out(l, el, False), "dz": _turned(tokens, c, ec, rows, temperature, bf16)}


def preference(z, tokens, bounds, ref=None, weight=None, temperature=1.0, beta=0.1, smoothing=0.0, average=False, bf16=False):
    """{name: (want, tolerance)} of loss, logp and dz."""
    r, v = z.shape
    rows = _rows(z, tokens, temperature)
    live, l, el = rows[0], rows[1], rows[2]
    pairs = len(bounds) // 2
    w = np.ones(pairs) if weight is None else weight.astype(np.float64)
    cut = np.clip(np.asarray(bounds, np.int64), 0, r)
    spans = [slice(cut[j], max(cut[j], cut[j + 1])) for j in range(2 * pairs)]
    count = np.array([max(1, int(live[s].sum())) if average else 1 for s in spans], np.float64)
    L = np.array([l[s].sum() for s in spans]) / count
    eL = np.array([(el[s] + U * np.abs(l[s])).sum() for s in spans]) / count   # each row's is held in fp32
    R = np.zeros(2 * pairs) if ref is None else ref
    with np.errstate(over="ignore", invalid="ignore"):
        m = beta * ((L[0::2] - R[0::2]) - (L[1::2] - R[1::2]))
        em = abs(beta) * (eL[0::2] + eL[1::2]) + 1e-15 * (np.abs(m) + abs(beta) * (np.abs(L[0::2]) + np.abs(L[1::2])))
        up, down = np.logaddexp(0, -m), np.logaddexp(0, m)
        sig, nsig = 1 / (1 + np.exp(-m)), 1 / (1 + np.exp(m))
    eps = smoothing
    loss = w * ((1 - eps) * up + (eps * down if eps else 0.0))
    eloss = np.abs(w) * ((1 - eps) * nsig + eps * sig) * em + U * np.abs(loss)
    slope = w * beta * (eps * sig - (1 - eps) * nsig)
    eslope = np.abs(w * beta) * np.minimum(sig, nsig) * em * (1 + em) + U * np.abs(slope)
    loss, eloss, slope, eslope = (np.where(w == 0, 0.0, a) for a in (loss, eloss, slope, eslope))
    c, ec = np.zeros(r), np.zeros(r)
    for j, s in enumerate(spans):
        c[s] = (slope[j // 2] if j % 2 == 0 else -slope[j // 2]) / count[j]
        ec[s] = eslope[j // 2] / count[j]
    c[~live], ec[~live] = 0.0, 0.0
    return {"loss": _out(loss, eloss, False), "logp": _out(L, eL, False), "dz": _turned(tokens, c, ec, rows, temperature, bf16)}
