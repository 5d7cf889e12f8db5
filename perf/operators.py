"""Cases of the operators at a model's logits: what a student learns from a
teacher's answers, the record of those answers, and answers drawn by chance.

``bitlogic_top_logits`` keeps the largest logits of every row with their
classes and the row's log-sum-exp: a teacher's record.
``bitlogic_distill_loss`` is the loss of a student's logits against such a
record and against labels, with its gradient.  ``bitlogic_sample_logits``
draws a class per row under temperature, top-k, top-p and min-p from given
random numbers.

``listed`` names the cases, ``draw`` gives further ones of the same ranges,
``prepare`` makes a case's inputs and output buffers on the GPU, ``run`` is
one pass (plain torch, or the framework's call when ``own`` is set), ``work``
its least bytes and operations, ``exact`` the outputs in 64 bits.

The teacher's record and the random numbers are inputs.  Classes are whole
numbers: equal logits rank by the lower class, and the draw's weights are
whole multiples of 2^-40 of the largest one, so that their sums are exact in
any order.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
LOG2E = 1.4426950408889634
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4}


# ------------------------------------------------------------------- cases --

def _top(rows, classes, top, dtype, pad=0, masked=0, temperature=1.0):
    return dict(kind="top", rows=rows, classes=classes, top=top, dtype=dtype, pad=pad, masked=masked,
                temperature=temperature)


def _distill(rows, classes, top, dtype, pad=0, masked=0, temperature=1.0, tail=False, labels=False, weights=False,
             class_major=False):
    return dict(kind="distill", rows=rows, classes=classes, top=top, dtype=dtype, pad=pad, masked=masked,
                temperature=temperature, tail=tail, labels=labels, weights=weights, class_major=class_major)


def _sample(rows, classes, dtype, mode, pad=0, masked=0):
    return dict(kind="sample", rows=rows, classes=classes, dtype=dtype, mode=mode, pad=pad, masked=masked)


def listed():
    def named(name, case):
        return dict(name=name, **case)

    return [
        # one request's next answer at a small vocabulary: latency
        named("sample_one", _sample(1, 32768, "bf16", "mixed")),
        # the hard head's counts over a test split of 10000, ten classes
        named("sample_counts_10", _sample(10000, 10, "i32", "plain")),
        # a served batch, nucleus sampling, rows of odd length
        named("sample_nucleus_odd", _sample(96, 50001, "f32", "nucleus")),
        # a large batch whose requests each bring their own settings
        named("sample_mixed_large", _sample(1024, 131072, "bf16", "mixed", masked=64)),
        # a teacher's record of one position, as it is served
        named("top_one", _top(1, 131072, 64, "f16")),
        # a teacher LUT network's counts of 100 classes over 10000 samples
        named("top_counts_100", _top(10000, 100, 10, "i32", temperature=100.0)),
        # a teacher's record of a training batch
        named("top_large", _top(4096, 131072, 128, "bf16", masked=64)),
        # the LUT network's ten-class head: labels and a teacher, gradient
        # rows per class as the layer-2 backward reads them
        named("distill_head_10", _distill(1024, 10, 4, "f32", temperature=2.0, labels=True, class_major=True)),
        # the hundred-class head on the odd last batch of an epoch
        named("distill_head_100_odd", _distill(2047, 100, 10, "f32", temperature=4.0, tail=True, labels=True,
                                               class_major=True)),
        # odd rows in full precision, labels and teacher, some rows left out
        named("distill_f32_odd", _distill(509, 50001, 50, "f32", temperature=2.0, labels=True, weights=True)),
        # an ordinary vocabulary batch against the record alone
        named("distill_f16", _distill(2048, 32768, 64, "f16", tail=True, weights=True)),
        # the largest training batch, a padded vocabulary
        named("distill_large", _distill(8192, 131072, 128, "bf16", masked=64, tail=True, weights=True)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "distill", "distill", "sample", "sample"])
    classes = _log(rng, 10, 131072)
    if classes > 64 and rng.random() < 0.4:
        classes = classes // 32 * 32
    # no drawn case has more logits than the largest listed one of its kind
    most = {"top": 1 << 29, "distill": 1 << 30, "sample": 1 << 27}[kind]
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"] + ([] if kind == "distill" else ["i32"] * (classes < 2000)))
    if BYTES[dtype] == 4:
        most //= 2
    rows = _log(rng, 1, max(1, min(16384, most // classes)))
    pad = rng.choice([0, 0, 0, 8, 3, 32])
    masked = rng.choice([0, 0, min(64, classes // 8)])
    if kind == "sample":
        return _sample(rows, classes, dtype, rng.choice(["plain", "nucleus", "top", "mixed", "mixed"]), pad, masked)
    top = min(classes - masked, _log(rng, 1, 256))
    if kind == "top":
        return _top(rows, classes, top, dtype, pad, masked, rng.choice([1.0, 2.0, 0.7]) * (50.0 if dtype == "i32" else 1.0))
    return _distill(rows, classes, top, dtype, pad, masked, rng.choice([1.0, 1.0, 2.0, 3.5]), rng.random() < 0.5,
                    rng.random() < 0.5, rng.random() < 0.5, classes <= 1000 and rng.random() < 0.4)


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rows_at_once(classes):
    return max(1, (1 << 27) // classes)


def _logits(case, g):
    """[rows, classes] in the case's type, `pad` unused values after each row."""
    R, V, dtype, pad = case["rows"], case["classes"], DTYPES[case["dtype"]], case["pad"]
    buf = torch.empty(R, V + pad, dtype=dtype, device=DEV)
    x = buf[:, :V]
    hot = max(1, min(16, V // 8))
    for r in range(0, R, _rows_at_once(V)):
        part = x[r:r + _rows_at_once(V)]
        n = part.shape[0]
        z = torch.randn(n, V, generator=g, device=DEV).mul_(2.0)
        at = torch.randint(0, V, (n, hot), generator=g, device=DEV)
        up = torch.empty(n, hot, device=DEV).exponential_(0.25, generator=g)
        z.scatter_add_(1, at, up)
        if dtype is torch.int32:   # group sums of a hard head: ones among 6400 nodes
            part.copy_(z.mul_(50.0).add_(3200.0).round_().clamp_(0.0, 6400.0))
            if case["masked"]:
                part[:, V - case["masked"]:] = 0
        else:
            part.copy_(z)
            if case["masked"]:     # classes that only pad the vocabulary
                part[:, V - case["masked"]:] = float("-inf")
    if pad:
        buf[:, V:] = 1 << 20 if dtype is torch.int32 else float("inf")
    return x


def _teacher(case, x, g):
    """A record of the K largest logits of a teacher that mostly agrees with
    the student, and the log-sum-exp of all of them."""
    R, V, K, tau = case["rows"], case["classes"], case["top"], case["temperature"]
    val = torch.empty(R, K, device=DEV)
    idx = torch.empty(R, K, dtype=torch.int32, device=DEV)
    lse = torch.empty(R, device=DEV)
    for r in range(0, R, _rows_at_once(V)):
        s = slice(r, r + _rows_at_once(V))
        y = x[s].float() * 0.9
        y += torch.randn(y.shape, generator=g, device=DEV)
        v, i = y.topk(K, dim=1)
        val[s], idx[s], lse[s] = v, i.to(torch.int32), torch.logsumexp(y / tau, dim=1)
    # a twentieth of the rows has a shorter record, down to none
    short = torch.rand(R, 1, generator=g, device=DEV) < 0.05
    left = torch.randint(0, K + 1, (R, 1), generator=g, device=DEV)
    gone = short & (torch.arange(K, device=DEV) >= left)
    idx[gone], val[gone] = -1, float("-inf")
    return val, idx, lse


def _settings(case, g):
    """Per-row temperature, top_k, top_p and min_p (None where unused)."""
    R, mode = case["rows"], case["mode"]
    rand = lambda: torch.rand(R, generator=g, device=DEV)   # noqa: E731

    def pick(values, dtype):
        return torch.tensor(values, dtype=dtype, device=DEV)[torch.randint(0, len(values), (R,), generator=g, device=DEV)]

    unit = 50.0 if case["dtype"] == "i32" else 1.0
    s = dict(temperature=(0.6 + 0.8 * rand()) * unit, top_k=None, top_p=None, min_p=None)
    if mode == "nucleus":
        s["top_p"] = 0.8 + 0.19 * rand()
    elif mode == "top":
        s["top_k"] = pick([20, 40, 50, 100], torch.int32)
    elif mode == "mixed":
        s["temperature"] = torch.where(rand() < 0.05, torch.zeros((), device=DEV), s["temperature"])   # greedy requests
        s["top_k"] = pick([0, 0, 1, 5, 40, 200, 1000], torch.int32)
        s["top_p"] = pick([1.0, 0.5, 0.9, 0.95, 0.99], torch.float32)
        s["min_p"] = pick([0.0, 0.0, 0.02, 0.1], torch.float32)
    return s


def _inputs(case, seed):
    g = _gen(seed)
    R, kind = case["rows"], case["kind"]
    v = dict(logits=_logits(case, g))
    if kind == "distill":
        v["val"], v["idx"], lse = _teacher(case, v["logits"], g)
        v["lse"] = lse if case["tail"] else None
        v["labels"] = v["weight"] = None
        if case["labels"]:   # some samples carry no label
            labels = torch.randint(0, case["classes"] - case["masked"], (R,), generator=g, device=DEV).to(torch.int32)
            v["labels"] = torch.where(torch.rand(R, generator=g, device=DEV) < 0.05, torch.full_like(labels, -1), labels)
        if case["weights"]:  # rows left out of the loss
            keep = (torch.rand(R, generator=g, device=DEV) >= 0.1).float()
            v["weight"] = keep / keep.sum().clamp_(min=1.0)
    elif kind == "sample":
        v["u"] = torch.rand(R, generator=g, device=DEV)
        v.update(_settings(case, g))
    return v


def _mix(case):
    """kd_weight, ce_weight, grad_scale: a class-major gradient goes on to the
    nodes of a group-sum head of temperature 20."""
    return (0.7 if case["labels"] else 1.0), (0.3 if case["labels"] else 0.0), (0.05 if case["class_major"] else 1.0)


def prepare(case, seed):
    s = _inputs(case, seed)
    R, V = case["rows"], case["classes"]
    s["case"] = case
    if case["kind"] == "top":
        s["val"] = torch.empty(R, case["top"], device=DEV)
        s["idx"] = torch.empty(R, case["top"], dtype=torch.int32, device=DEV)
        s["lse"] = torch.empty(R, device=DEV)
    elif case["kind"] == "distill":
        s["row_loss"], s["loss"] = torch.empty(R, device=DEV), torch.empty(1, device=DEV)
        dtype = DTYPES[case["dtype"]]
        if case["class_major"]:
            s["grad"] = torch.empty(V, R, dtype=dtype, device=DEV).t()
        else:
            s["grad"] = torch.empty(R, V + case["pad"], dtype=dtype, device=DEV)[:, :V]
    else:
        s["token"], s["logprob"] = torch.empty(R, dtype=torch.int32, device=DEV), torch.empty(R, device=DEV)
    return s


# --------------------------------------------------------------------- run --

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_top(s):
    import paper_2602_07400_gb300 as bl
    bl.bitlogic_top_logits(s["logits"], s["val"], s["idx"], s["lse"], temperature=s["case"]["temperature"])
    return dict(val=s["val"], idx=s["idx"], lse=s["lse"])


def _own_distill(s):
    import paper_2602_07400_gb300 as bl
    kd, ce, scale = _mix(s["case"])
    bl.bitlogic_distill_loss(s["logits"], s["val"], s["idx"], s["row_loss"], s["loss"], s["grad"],
                             teacher_lse=s["lse"], labels=s["labels"], row_weight=s["weight"],
                             temperature=s["case"]["temperature"], kd_weight=kd, ce_weight=ce, grad_scale=scale)
    return dict(loss=s["loss"], row_loss=s["row_loss"], grad=s["grad"])


def _own_sample(s):
    import paper_2602_07400_gb300 as bl
    bl.bitlogic_sample_logits(s["logits"], s["u"], s["token"], s["logprob"], temperature=s["temperature"],
                              top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return dict(token=s["token"], logprob=s["logprob"])


_OWN = dict(top=_own_top, distill=_own_distill, sample=_own_sample)


def _lse(y):
    """ln sum exp of the rows of y, -inf for a row of -inf."""
    m = y.amax(dim=1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    return (m + (y - m).exp().sum(dim=1, keepdim=True).log()).squeeze(1)


def _plain_top(s):
    K, tau = s["case"]["top"], s["case"]["temperature"]
    z = s["logits"].float()
    val, idx = torch.sort(z, dim=1, descending=True, stable=True)
    val = val[:, :K].contiguous()
    idx = torch.where(val > float("-inf"), idx[:, :K], -torch.ones_like(idx[:, :K])).to(torch.int32)
    return dict(val=val, idx=idx, lse=_lse(z * (1.0 / tau)))


def _plain_distill(s):
    case = s["case"]
    tau, (kd, ce, scale) = case["temperature"], _mix(case)
    z = s["logits"].float()
    R, V = z.shape
    zero = torch.zeros((), device=DEV)
    weight = s["weight"] if s["weight"] is not None else torch.full((R,), 1.0 / R, device=DEV)
    y = z * (1.0 / tau)
    m = y.amax(dim=1, keepdim=True)
    e = (y - m).exp()
    total = e.sum(dim=1, keepdim=True)
    lse = m + total.log()
    # teacher
    listed_ = s["idx"] >= 0
    at = s["idx"].clamp(min=0).long()
    a = torch.where(listed_, s["val"], torch.full_like(s["val"], float("-inf"))) * (1.0 / tau)
    log_norm = s["lse"][:, None] if s["lse"] is not None else _lse(a)[:, None]
    q = torch.where(a > float("-inf"), (a - log_norm).exp(), zero)
    Q = q.sum(dim=1, keepdim=True)
    kl = torch.where(q > 0, q * ((a - log_norm) - (y.gather(1, at) - lse)), zero).sum(dim=1)
    # classes on the record (its unused places go to a column past the last)
    member = torch.zeros(R, V + 1, dtype=torch.bool, device=DEV).scatter_(1, torch.where(listed_, at, V), True)[:, :V]
    qd = torch.zeros(R, V + 1, device=DEV).scatter_add_(1, torch.where(listed_, at, V), q)[:, :V]
    p = e / total
    if s["lse"] is not None:
        any_q = listed_.any(dim=1, keepdim=True)
        rest = torch.where(member, zero, e).sum(dim=1, keepdim=True)
        qr = torch.where(any_q & (rest > 0), (1.0 - Q).clamp(min=0.0), zero)
        kl = kl + torch.where(qr > 0, qr * (qr.log() - (rest / total).log()), zero).squeeze(1)
        W = Q + qr
        g = p * W - qd - torch.where(member | (qr <= 0), zero, qr * e / rest)
    else:
        g = p * Q - qd
    row = kd * tau * tau * kl
    g = g * (kd * tau)
    if s["labels"] is not None:
        has = s["labels"] >= 0
        lab = s["labels"].clamp(min=0).long()[:, None]
        mz = z.amax(dim=1, keepdim=True)
        ez = (z - mz).exp()
        sz = ez.sum(dim=1, keepdim=True)
        row = row + torch.where(has, ce * (mz + sz.log() - z.gather(1, lab)).squeeze(1), zero)
        d = (ez / sz).scatter_add_(1, lab, torch.full((R, 1), -1.0, device=DEV))
        g = g + torch.where(has[:, None], ce * d, zero)
    row = torch.where(weight != 0, row, zero)
    grad = torch.where(weight[:, None] != 0, g * (weight * scale)[:, None], zero)
    return dict(loss=(weight * row).sum().reshape(1), row_loss=row, grad=grad.to(DTYPES[case["dtype"]]))


def _share(total, x):
    """floor(total * x) for x in [0, 1) held to 24 bits; total below 2^62."""
    x24 = (x * 16777216.0).long()[:, None]
    return (((total >> 32) * x24) << 8) + (((total & 0xFFFFFFFF) * x24) >> 24)


def _plain_sample(s):
    z = s["logits"].float()
    R, V = z.shape
    m = z.amax(dim=1, keepdim=True)
    T = s["temperature"]
    slope = torch.where(T > 0, LOG2E / T, torch.zeros_like(T))[:, None]
    e = torch.where(z > float("-inf"), ((z - m) * slope).exp2(), torch.zeros((), device=DEV))
    w = (e * 2.0 ** 40).round().long()
    k = s["top_k"].long() if s["top_k"] is not None else torch.zeros(R, dtype=torch.long, device=DEV)
    k = torch.where(T > 0, torch.where(k > 0, k, V), 1)[:, None]
    kept = w > 0
    if s["top_k"] is not None or s["top_p"] is not None:
        _, order = torch.sort(z, dim=1, descending=True, stable=True)
        ws = w.gather(1, order)
        keep = torch.arange(V, device=DEV)[None, :] < k
        if s["top_p"] is not None:
            ws = torch.where(keep, ws, 0)
            mass = _share(ws.sum(dim=1, keepdim=True), s["top_p"].clamp(max=1.0)).clamp(min=1)
            keep &= (ws.cumsum(dim=1) - ws < mass) | (s["top_p"] >= 1)[:, None]
        kept &= torch.zeros_like(keep).scatter_(1, order, keep)
    if s["min_p"] is not None:
        kept &= e >= s["min_p"][:, None]
    sums = torch.where(kept, w, 0).cumsum(dim=1)
    total = sums[:, -1:]
    token = (sums <= _share(total, s["u"])).sum(dim=1, keepdim=True)
    logprob = (w.gather(1, token).float() / total.float()).log()
    return dict(token=token.squeeze(1).to(torch.int32), logprob=logprob.squeeze(1))


_PLAIN = dict(top=_plain_top, distill=_plain_distill, sample=_plain_sample)


# -------------------------------------------------------------------- work --

def work(case):
    R, V, kind = case["rows"], case["classes"], case["kind"]
    n = R * V
    read = n * BYTES[case["dtype"]]
    if kind == "top":   # an exponential, a multiply-add and a comparison per logit
        return dict(bytes=read + R * case["top"] * 8 + 4 * R, flops=4 * n)
    if kind == "sample":
        return dict(bytes=read + 8 * R + 4 * R * (2 + 2 * (case["mode"] == "mixed") + (case["mode"] in ("mixed", "nucleus"))),
                    flops=4 * n)
    two = case["labels"] and case["temperature"] != 1.0   # two softmaxes
    return dict(bytes=2 * read + R * case["top"] * 8 + 4 * R * (1 + case["tail"] + case["labels"] + case["weights"]) + 4,
                flops=n * (12 if two else 6))


# ------------------------------------------------------------------- exact --

def exact(case, seed):
    v = _inputs(case, seed)
    R, V = case["rows"], case["classes"]
    step = max(1, (1 << 26) // V)
    parts = [_EXACT[case["kind"]](case, v, slice(r, min(R, r + step))) for r in range(0, R, step)]
    out = {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
    if case["kind"] == "distill":
        weight = v["weight"].double() if v["weight"] is not None else torch.full((R,), 1.0 / R, dtype=torch.float64, device=DEV)
        out["loss"] = (weight * out["row_loss"]).sum().reshape(1)
    return out


def _exact_top(case, v, s):
    z, K = v["logits"][s].double(), case["top"]
    # by class first, then a stable order by value
    val, idx = torch.sort(-z, dim=1, stable=True)
    val = -val[:, :K]
    idx = idx[:, :K].masked_fill(torch.isinf(val), -1).to(torch.int32)
    return dict(val=val, idx=idx, lse=torch.logsumexp(z / case["temperature"], dim=1))


def _exact_distill(case, v, s):
    tau, (kd, ce, scale) = case["temperature"], _mix(case)
    z = v["logits"][s].double()
    R, V = z.shape
    logp = torch.log_softmax(z / tau, dim=1)
    val, idx = v["val"][s].double() / tau, v["idx"][s].long()
    none = idx < 0
    norm = v["lse"][s].double() if v["lse"] is not None else torch.logsumexp(val, dim=1)
    q = torch.exp(val - norm[:, None]).masked_fill(none, 0.0).nan_to_num(0.0)
    cols = idx.masked_fill(none, V)
    dense = torch.zeros(R, V + 1, dtype=torch.float64, device=DEV).scatter_(1, cols, q)[:, :V]
    on = torch.zeros(R, V + 1, dtype=torch.bool, device=DEV).scatter_(1, cols, True)[:, :V]
    p = logp.exp()
    kl = torch.special.xlogy(dense, dense).sum(1) - (dense * logp.masked_fill(dense == 0, 0.0)).sum(1)
    off = p * dense.sum(1, keepdim=True) - dense
    if case["tail"]:
        left = p.masked_fill(on, 0.0).sum(1)
        other = (1.0 - dense.sum(1)).clamp(min=0.0) * on.any(1) * (left > 0)
        kl = kl + torch.special.xlogy(other, other) - torch.special.xlogy(other, left)
        share = other / left.clamp(min=1e-300)
        off = p * (dense.sum(1) + other)[:, None] - dense - (p * share[:, None]).masked_fill(on, 0.0)
    row, grad = kd * tau ** 2 * kl, kd * tau * off
    if v["labels"] is not None:
        labels = v["labels"][s].long()
        logs = torch.log_softmax(z, dim=1)
        has = (labels >= 0).double()
        hit = torch.zeros_like(z).scatter_(1, labels.clamp(min=0)[:, None], 1.0)
        row = row - ce * has * logs.gather(1, labels.clamp(min=0)[:, None]).squeeze(1)
        grad = grad + ce * has[:, None] * (logs.exp() - hit)
    weight = v["weight"][s].double() if v["weight"] is not None else torch.full((R,), 1.0 / case["rows"], dtype=torch.float64, device=DEV)
    used = (weight != 0).double()
    return dict(row_loss=row * used, grad=grad * (scale * weight)[:, None])


def _exact_sample(case, v, s):
    z = v["logits"][s].double()
    R, V = z.shape
    T = v["temperature"][s].double()
    greedy = T <= 0
    # relative to the largest, so that equal logits have equal whole-number shares
    p = torch.exp((z - z.amax(1, keepdim=True)) / T.masked_fill(greedy, 1.0)[:, None])
    order = torch.argsort(-z, dim=1, stable=True)
    ps = p.gather(1, order)
    rank = torch.arange(V, device=DEV)[None, :]
    k = torch.full((R,), V, device=DEV) if v["top_k"] is None else v["top_k"][s].long()
    k = k.masked_fill(k <= 0, V).masked_fill(greedy, 1)
    ps = ps * (rank < k[:, None])
    keep = ps > 0
    if v["top_p"] is not None:
        top_p = v["top_p"][s].double()[:, None]
        before = ps.cumsum(1) - ps
        keep &= (before < top_p * ps.sum(1, keepdim=True)) | (top_p >= 1.0) | (rank == 0)
    if v["min_p"] is not None:
        keep &= ps >= v["min_p"][s].double()[:, None] * ps[:, :1]
    p = p * torch.zeros_like(keep).scatter_(1, order, keep)
    sums = p.cumsum(1)
    token = torch.searchsorted(sums, v["u"][s].double()[:, None] * sums[:, -1:], right=True).clamp_(max=V - 1)
    return dict(token=token.squeeze(1).to(torch.int32), logprob=(p.gather(1, token) / sums[:, -1:]).log().squeeze(1))


_EXACT = dict(top=_exact_top, distill=_exact_distill, sample=_exact_sample)
