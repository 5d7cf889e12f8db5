"""Plain 64-bit forms of the operators beside a larger model (draft verification,
supports, dropout, norms to 8 bits), on the CPU, from ``include/bitlogic.h``."""
import math

import numpy as np

import logits_ref as ref

E4M3_MAX = 448.0


# ------------------------------------------------------- supports and drafts --

def kept_set(z, floor=-np.inf, last=-1):
    """Classes of one row (float64) that a support leaves, with a weight or not."""
    with np.errstate(invalid="ignore"):
        return (z > floor) | ((z == floor) & (np.arange(len(z)) <= last) & (z > -np.inf))


def probs(z, temperature=1.0, floor=-np.inf, last=-1):
    """The softmax of the kept logits of one row; None when nothing ranks."""
    keep = kept_set(z, floor, last) & ~np.isnan(z)
    if not keep.any():
        return None
    m = z[keep].max()
    if not temperature > 0 or m == np.inf:
        p = np.zeros(len(z))
        p[np.flatnonzero(keep & (z == m))[0]] = 1.0
        return p
    e = np.where(keep, np.exp((np.where(keep, z, m) - m) / float(temperature)), 0.0)
    return e / e.sum()


def verdicts(rows, tokens, logprobs, u, draw_u, drafts, tol=2e-6):
    """Every (accepted, next class) that the definition allows for one sequence
    when p, q and the sums carry a relative error of `tol`.

    rows: per target row (z, temperature, floor, last); drafts: the same per
    draft, or None for drafts without a distribution."""
    allowed = set()
    for a, token in enumerate(tokens):
        p = probs(*rows[a])
        V = len(rows[a][0])
        q = math.exp(logprobs[a]) if logprobs is not None else 1.0
        pd = p[token] if p is not None and 0 <= token < V else 0.0
        uq = float(u[a]) * q
        near = pd > 0 and abs(uq - pd) <= tol * pd
        if near or not uq < pd:
            allowed |= {(a, t) for t in draws(refused_weights(p, drafts[a] if drafts is not None else None, token, V), draw_u, tol)}
        if not near and not uq < pd:
            return allowed
    p = probs(*rows[len(tokens)])
    return allowed | {(len(tokens), t) for t in draws(p, draw_u, tol)}


def refused_weights(p, draft, token, V):
    if p is None:
        return None
    q = np.zeros(V)
    if draft is None or not draft[1] > 0:
        if 0 <= token < V:
            q[token] = 1.0
    else:
        qd = probs(*draft)
        if qd is not None:
            q = qd
            kept = draft[0][kept_set(*draft[:1], *draft[2:])]
            if np.isposinf(kept).any():
                q = np.zeros(V)
                q[token] = 1.0
    left = np.maximum(p - q, 0.0)
    return left if left.sum() > 0 else p


def draws(w, u, tol):
    """Classes that floor(u sum) can fall in when every share of w is off by up to
    tol of its own and by 2^-41, and the sums with them."""
    if w is None:
        return {-1}
    sums = np.cumsum(w)
    total = sums[-1]
    slack = tol * (1.0 + 1.0 / total) * total + len(w) * 2.0 ** -41 + 2.0 ** -23 * total
    goal = float(u) * total
    lo, hi = goal - slack, goal + slack
    ok = (sums > lo) & (sums - w <= hi) & (w > 0)
    return set(np.flatnonzero(ok).tolist())


def support(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """floor and last of one row, in the whole numbers of a draw, and whether the
    cut lies so near a border that a rounding of the powers may move it."""
    V = len(z)
    o = ref.order(z)
    if len(o) == 0:
        return -math.inf, -1, False
    one = not temperature > 0 or np.isposinf(z[o[0]])
    if not 0 < (1 if one else top_k) < V and not top_p < 1 and not min_p > 0:
        return -math.inf, -1, False
    if one:
        return z[o[0]], int(o[0]), False
    e, w = ref.weights(z, temperature)
    kept = list(o[:top_k]) if 0 < top_k < len(o) else list(o)
    near = False
    if top_p < 1:
        total = sum(w[v] for v in kept)
        want = max(1, ref.share(total, max(top_p, 0.0)))
        run, n = 0, 0
        while run < want:
            run += w[kept[n]]
            n += 1
        # (the first class alone, where top_p is 0, is no border)
        near = top_p > 0 and min(abs(run - want), abs(run - w[kept[n - 1]] - want)) <= 4e-6 * total
        kept = kept[:n]
    if min_p > 0:
        bar = float(min(np.float32(min_p), np.float32(1)))
        # (the power of the largest is exactly 1)
        near = near or any(abs(e[v] - bar) <= 1e-6 * bar and e[v] < 1 for v in kept)
        kept = [v for v in kept if e[v] >= bar]
    return z[kept[-1]], int(kept[-1]), near


# ----------------------------------------------------------------- dropout --

def philox(block, step, stream, seed):
    """Philox4x32-10: the four words of every counter, uint64 arrays of 32-bit values."""
    M = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    block = np.asarray(block, np.uint64)
    c = [block & M, block >> sh, np.full_like(block, step & 0xFFFFFFFF), np.full_like(block, stream)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> sh) ^ c[1] ^ np.uint64(k[0]), b & M, (a >> sh) ^ c[3] ^ np.uint64(k[1]), a & M]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept_values(i0, n, seed, step, p, site):
    """Whether elements i0 .. i0 + n - 1 are kept."""
    b0, b1 = i0 // 8, (i0 + n + 7) // 8
    block = np.arange(b0, b1, dtype=np.uint64)

    def halves(stream):
        w = philox(block, step, stream, seed)
        return np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=1).reshape(-1)

    number = (halves(2 * site) << np.uint64(16)) | halves(2 * site + 1)
    return (number >= np.uint64(round(p * 2.0 ** 32)))[i0 - 8 * b0:i0 - 8 * b0 + n]


# ------------------------------------------------------------------- norms --

def norm(h, weight, eps):
    """y of rows h (float64)."""
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return y if weight is None else y * weight


def groups(d, group):
    return [(0, d)] if group == 0 else [(c, min(d, c + group)) for c in range(0, d, group)]


def norm_backward(dy, h, weight, eps):
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    xh = h * r
    g = dy if weight is None else dy * weight
    return r * (g - xh * (g * xh).mean(1, keepdims=True)), (dy * xh).sum(0)
