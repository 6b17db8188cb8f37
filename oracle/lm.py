"""TEST INFRASTRUCTURE: 64-bit statements of the language-model operators, straight from their definitions, and
bounds on how far an fp32 evaluation may be from them.

U is the unit roundoff of fp32, UB that of bf16.  Each bound is a first-order running bound: the error that
a quantity inherits plus one term for every rounding on the way, with these constants of the arithmetic:
  sums: an fp32 sum of m terms in any order is off by at most (m - 1) U times the sum of their magnitudes
  __expf(x): 2 + floor(1.16 |x|) ulp, division 2 ulp, ex2.approx and lg2.approx 2 ulp (an ulp is 2 U at most)
and a bf16 output adds UB times its magnitude.  SLACK covers second-order terms and subnormal results.
"""
import numpy as np

U, UB = 2.0 ** -24, 2.0 ** -8
SLACK = 1.01
TINY = 1e-37


def _out(want, err, bf16):
    return want, SLACK * (err + (UB if bf16 else U) * (np.abs(want) + err)) + TINY


# ------------------------------------------------------------------------------------------- embedding


def embed_lookup(E, tokens, scale, bf16=False):
    n, v, d = E.shape
    want = np.zeros((n, tokens.shape[1], d))
    for i in range(n):
        for s, w in enumerate(tokens[i]):
            if 0 <= w < v:
                want[i, s] = scale * E[i, w]
    return _out(want, U * np.abs(want), bf16)


def embed_grad(dout, tokens, v, scale, before=None, bf16=False):
    n, t, d = dout.shape
    sums, mags, many = np.zeros((n, v, d)), np.zeros((n, v, d)), np.zeros((n, v, 1))
    for i in range(n):
        at = np.flatnonzero((tokens[i] >= 0) & (tokens[i] < v))
        np.add.at(sums[i], tokens[i][at], dout[i][at])
        np.add.at(mags[i], tokens[i][at], np.abs(dout[i][at]))
        np.add.at(many[i], tokens[i][at], 1.0)
    want, err = scale * sums, abs(scale) * (many + 1) * U * mags   # m - 1 additions, the product
    if before is not None:
        err = err + np.where(many > 0, U * (np.abs(want) + np.abs(before)), 0.0)
        want = want + before
    want, tol = _out(want, err, bf16)
    if before is not None:
        tol = np.where(many > 0, tol, 0.0)   # a row without a token is not touched
    return want, tol


# ------------------------------------------------------------------------------------------- recurrence


def _gates(f):
    with np.errstate(over="ignore"):
        a, na = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    return a, na, U * (12 + 2.4 * np.minimum(np.abs(f), 90.0))   # exp, 1 + e, the quotient, a product


def recurrence(x, f, h0=None, starts=None, bf16=False):
    """{name: (want, tolerance)} of h and last; also h and its bound in 64 bits for the gradient."""
    b, t, d = x.shape
    a, na, eg = _gates(f)
    h = np.zeros((b, d)) if h0 is None else h0.astype(np.float64)
    e = np.zeros((b, d))
    go = np.ones((b, t, 1), bool) if starts is None else (starts == 0)[:, :, None]
    hs, es, ps, eps = (np.zeros((b, t, d)) for _ in range(4))
    for s in range(t):
        ps[:, s], eps[:, s] = np.where(go[:, s], h, 0.0), np.where(go[:, s], e, 0.0)
        p, ep = ps[:, s], eps[:, s]
        h = a[:, s] * p + na[:, s] * x[:, s]
        # two gates, the product with x, and the additions and products of the scan: 4 roundings a step
        e = a[:, s] * ep + (eg[:, s] + 4 * U) * (a[:, s] * np.abs(p) + na[:, s] * np.abs(x[:, s]))
        hs[:, s], es[:, s] = h, e
    return {"h": _out(hs, es, bf16), "last": _out(h, e, False)}, (ps, eps)


def recurrence_grad(x, f, dh, h0=None, starts=None, dh_last=None, bf16=False):
    b, t, d = x.shape
    _, (ps, eps) = recurrence(x, f, h0, starts)
    a, na, eg = _gates(f)
    go = np.ones((b, t, 1), bool) if starts is None else (starts == 0)[:, :, None]
    c = np.zeros((b, d)) if dh_last is None else dh_last.astype(np.float64)
    ec = np.zeros((b, d))
    ls, el = np.zeros((b, t, d)), np.zeros((b, t, d))
    for s in range(t - 1, -1, -1):
        ls[:, s] = dh[:, s] + c
        el[:, s] = ec + U * (np.abs(dh[:, s]) + np.abs(c))
        c = np.where(go[:, s], a[:, s] * ls[:, s], 0.0)
        ec = np.where(go[:, s], a[:, s] * el[:, s] + (eg[:, s] + 4 * U) * a[:, s] * (np.abs(dh[:, s]) + np.abs(ls[:, s])), 0.0)
    dx, df = na * ls, a * na * ls * (ps - x)
    edx = na * el + (eg + U) * np.abs(dx)
    edf = a * na * (el * np.abs(ps - x) + np.abs(ls) * (eps + U * (np.abs(ps) + np.abs(x)))) + (2 * eg + 4 * U) * np.abs(df)
    return {"dx": _out(dx, edx, bf16), "df": _out(df, edf, bf16), "dh0": _out(c, ec, False)}


# ------------------------------------------------------------------------------------------- distillation


def _logsumexp(x):
    top = x.max() if x.size else -np.inf
    return top if top == -np.inf else top + np.log(np.exp(x - top).sum())


def distill(z, idx, t, teacher_lse=None, weight=None, temperature=1.0, bf16=False):
    """{name: (want, tolerance)} of loss and dz, row by row."""
    r, v = z.shape
    loss, dz = np.zeros(r), np.zeros((r, v))
    tl, tz = np.zeros(r), np.zeros((r, v))
    for i in range(r):
        w = 1.0 if weight is None else float(weight[i])
        with np.errstate(over="ignore", invalid="ignore"):
            ti = t[i] / temperature
        js = [j for j in range(len(idx[i])) if 0 <= idx[i][j] < v and not ti[j] == -np.inf]
        if w == 0.0 or not js:
            continue
        at = np.array([int(idx[i][j]) for j in js])
        ti = ti[js]
        y = z[i] / temperature
        top = y.max()
        fin = y[np.isfinite(y)]
        if top == -np.inf:
            q, logq = np.zeros(v), np.full(v, -np.inf)
        else:
            lse = top + np.log(np.exp(y - top).sum())
            logq = y - lse
            q = np.exp(logq)
        # relative bound of an exponential and of the sum: the scaled exponent's rounding (two roundings of at most its
        # range), ex2, v / 128 additions in a row and a tree of less than 40, the quotient
        reach = float(top - fin.min()) if fin.size else 0.0
        rq = U * (4 * reach + 16 + v / 128 + 40)
        if teacher_lse is None:
            tt = ti.max()
            norm = tt + np.log(np.exp(ti - tt).sum())
        else:
            norm = float(teacher_lse[i])
        lp = ti - norm
        p = np.exp(lp)
        rp = U * (4 * (np.abs(ti).max() + abs(norm)) + 20 + len(js))
        p0 = 1.0 - p.sum() if teacher_lse is not None and not p.sum() >= 1.0 else 0.0   # NaN for a NaN
        ep0 = (rp + len(js) * U) * p.sum() + U if teacher_lse is not None else 0.0
        inside = np.zeros(v, bool)
        inside[at] = True
        pc = np.zeros(v)
        np.add.at(pc, at, p)
        use = p > 0
        # the logarithms: exponent roundings as above, lg2 and its argument
        elog = rp + rq + 8 * U * (np.abs(lp) + np.abs(logq[at]) + 1)
        with np.errstate(invalid="ignore", divide="ignore"):
            terms = np.where(use, p * (lp - logq[at]), 0.0)
            kl = terms.sum()
            ekl = np.where(use, p * (rp * np.abs(lp - logq[at]) + elog), 0.0).sum() + (len(js) + 4) * U * np.abs(terms).sum()
            target = pc
            et = rp * pc + len(js) * U * pc
            if teacher_lse is not None:
                lq0 = _logsumexp(logq[~inside])   # q0 itself may be too small for 64 bits
                share = np.where(~inside, np.exp(logq - lq0), 0.0) if lq0 > -np.inf else np.zeros(v)
                if p0 > 0:
                    lr = np.log(p0) - lq0
                    kl += p0 * lr
                    ekl += ep0 * (abs(lr) + 1) + p0 * (2 * rq + 8 * U * (abs(lr) + 1)) + U * abs(p0 * lr)
                    target = np.where(inside, pc, p0 * share)
                    et = np.where(inside, et, share * (ep0 + p0 * 3 * rq))
                elif ep0 > 0 and lq0 > -np.inf:   # the true rest may be rounded up to ep0
                    ekl += ep0 * (abs(np.log(ep0) - lq0) + 1)
                    et = np.where(inside, et, share * ep0)
        loss[i], tl[i] = w * kl, abs(w) * ekl
        # all the mass that is compared is 1, or what the top holds where that is more (or may be rounded to more)
        all_mass, e_mass = 1.0, 0.0
        if teacher_lse is not None:
            all_mass = p.sum() + p0
            e_mass = ep0 if p.sum() > 1.0 - ep0 else 0.0
        dz[i] = w / temperature * (all_mass * q - target)
        tz[i] = abs(w) / temperature * ((3 * rq * all_mass + e_mass) * q + et + 3 * U * (all_mass * q + target))
    with np.errstate(invalid="ignore"):
        return {"loss": _out(loss, tl, False), "dz": _out(dz, tz, bf16)}
