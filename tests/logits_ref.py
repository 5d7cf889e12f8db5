"""Plain 64-bit forms of the operators on rows of logits, on the CPU.

Written from the definitions in ``include/bitlogic.h``; one row at a time.
"""
import math

import numpy as np

LOG2E = np.float32(1.4426950408889634)


def values(x):
    """Logits as the operators read them, float64 [T, V]."""
    z = x.detach().cpu()
    if z.dtype.is_floating_point:
        return z.double().numpy()
    z = z.numpy()
    return np.where(z == np.iinfo(np.int32).min, -np.inf, z.astype(np.float32).astype(np.float64))


def order(z):
    """Classes that rank, largest first, equal ones by class."""
    ok = np.flatnonzero(~np.isnan(z) & (z > -np.inf))
    return ok[np.argsort(-z[ok], kind="stable")]


def lse(z):
    if np.isnan(z).any():
        return math.nan
    m = z.max()
    if np.isinf(m):
        return m
    return m + math.log(np.exp(z - m).sum())


def log_softmax(z):
    d = z - z.max()          # no digits of the classes' differences lost in a large maximum
    return d - math.log(np.exp(d).sum())


def top(z, K, tau):
    val, idx = np.full(K, -np.inf), np.full(K, -1)
    o = order(z)[:K]
    val[:len(o)], idx[:len(o)] = z[o], o
    return val, idx, lse(z / tau)


def distill(z, val, idx, t_lse, label, w, tau, kd, ce, scale):
    """Loss, gradient and the magnitude of the gradient's terms of one row."""
    V = len(z)
    zero = np.zeros(V)
    if w == 0 or np.all(z == -np.inf):
        return 0.0, zero, zero
    if np.isnan(z).any() or np.isposinf(z).any():
        return math.nan, np.full(V, math.nan), zero
    with np.errstate(divide="ignore", invalid="ignore"):
        y = z / tau
        logp = log_softmax(y)
        p = np.exp(logp)
        on = np.zeros(V, bool)
        q = np.zeros(V)
        use = [(int(v), float(a) / tau) for v, a in zip(idx, val) if 0 <= v < V]
        for v, _ in use:
            on[v] = True
        live = [(v, a) for v, a in use if a > -np.inf]
        if live:
            norm = t_lse if t_lse is not None else lse(np.array([a for _, a in live]))
        kl = 0.0
        for v, a in live:
            qk = math.exp(a - norm)
            q[v] += qk
            if qk > 0:
                kl += qk * ((a - norm) - logp[v])
        Q = q.sum()
        rest = p[~on].sum()
        qr = max(0.0, 1.0 - Q) if t_lse is not None and on.any() and rest > 0 else 0.0
        if qr > 0:
            kl += qr * (math.log(qr) - math.log(rest))
        g = (Q + qr) * p - q
        mag = (Q + qr) * p + q
        if qr > 0:
            g[~on] -= qr * p[~on] / rest
            mag[~on] += qr * p[~on] / rest
        loss = kd * tau * tau * kl if kd else 0.0
        g, mag = g * kd * tau, mag * abs(kd) * tau
        if label is not None and 0 <= label < V and ce:
            s = np.exp(log_softmax(z))
            loss -= ce * log_softmax(z)[label]
            g, mag = g + ce * s, mag + abs(ce) * s
            g[label] -= ce
            mag[label] += abs(ce)
    return loss, g * (w * scale), mag * abs(w * scale)


def weights(z, temperature):
    """e (float64 of the exact power) and whole weights of one row; the
    argument of the power is rounded as the definition says."""
    z32 = z.astype(np.float32)
    ok = ~np.isnan(z) & (z > -np.inf)
    m = z32[ok].max()
    with np.errstate(invalid="ignore", over="ignore"):
        slope = np.float32(np.float32(1) / np.float32(temperature)) * LOG2E
        y = ((z32 - m) * slope).astype(np.float64)
        e = np.where(ok, np.exp2(np.where(ok, y, -np.inf)), 0.0)
    return e, [int(v) for v in np.rint(e * 2.0 ** 40)]


def share(total, x):
    return (total * int(np.float32(x) * np.float32(16777216.0))) >> 24


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The class drawn and the logarithm of its probability, in whole numbers."""
    o = order(z)
    if len(o) == 0:
        return -1, -math.inf
    if not temperature > 0 or np.isposinf(z[o[0]]):
        return int(o[0]), 0.0
    e, w = weights(z, temperature)
    kept = list(o[:top_k]) if 0 < top_k < len(o) else list(o)
    if top_p < 1:
        want = max(1, share(sum(w[v] for v in kept), max(top_p, 0.0)))
        run, n = 0, 0
        while run < want:
            run += w[kept[n]]
            n += 1
        kept = kept[:n]
    if min_p > 0:
        kept = [v for v in kept if e[v] >= min(np.float32(min_p), np.float32(1))]
    total = sum(w[v] for v in kept)
    target, run = share(total, u), 0
    for v in sorted(kept):
        run += w[v]
        if run > target:
            return int(v), math.log(w[v] / total)
    raise AssertionError("the draw passed the end of the row")
