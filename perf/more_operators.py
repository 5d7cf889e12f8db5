"""Cases of the operators that put a small network beside a large model: its
answers as drafts that the large model checks, dropout while it learns, and
hidden states of the large model as its 8-bit inputs.

``bitlogic_support_logits`` gives the classes that top-k, top-p and min-p leave
of each row of logits.  ``bitlogic_verify_drafts`` accepts or rejects drafted
classes by the target's logits and given random numbers and draws the class
that follows.  ``bitlogic_dropout`` drops and scales values by a counter-based
generator, forward and backward from the same counter.  ``bitlogic_norm_bytes``
adds a residual, divides rows by their root mean square and rounds them to 8
bits with scales; ``bitlogic_norm_backward`` is its gradient.

``listed`` names the cases, ``draw`` gives further ones of the same ranges,
``prepare`` makes a case's inputs and output buffers on the GPU, ``run`` is one
pass (plain torch, or the framework's call when ``own`` is set), ``work`` its
least bytes and operations, ``exact`` the outputs in 64 bits.

Random numbers, seeds and counters are inputs.  Equal logits rank by the lower
class, and a draw's weights are whole multiples of 2^-40, so that their sums
are exact in any order.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
LOG2E = 1.4426950408889634
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4}
NEG = float("-inf")


# ------------------------------------------------------------------- cases --

def _verify(seqs, drafts, classes, dtype, draft, ragged=False, cut=0, pad=0):
    """`draft`: the type of the draft's logits, or "none" for drafts without a
    distribution; `cut`: top_k of both sides (0: all classes)."""
    return dict(kind="verify", seqs=seqs, drafts=drafts, classes=classes, dtype=dtype, draft=draft, ragged=ragged,
                cut=cut, pad=pad)


def _support(rows, classes, dtype, mode, pad=0):
    return dict(kind="support", rows=rows, classes=classes, dtype=dtype, mode=mode, pad=pad)


def _dropout(rows, cols, dtype, p, residual=False, backward=False, pad=0):
    return dict(kind="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual, backward=backward, pad=pad)


def _norm(rows, cols, dtype, out, group=0, residual=True, pad=0):
    """`out`: "e4m3", or "u8" (codes, returned as the values they stand for)."""
    return dict(kind="norm", rows=rows, cols=cols, dtype=dtype, out=out, group=group, residual=residual, pad=pad)


def _norm_back(rows, cols, dtype, residual=True, pad=0):
    return dict(kind="norm_back", rows=rows, cols=cols, dtype=dtype, residual=residual, pad=pad)


def listed():
    def named(name, case):
        return dict(name=name, **case)

    return [
        # one request, four drafts, a small vocabulary: latency
        named("verify_one", _verify(1, 4, 32768, "bf16", "bf16")),
        # a hard LUT network's draws over 100 classes, checked by a wider one's head
        named("verify_counts_100", _verify(2048, 3, 100, "f32", "i32")),
        # a served batch: ragged drafts, odd rows in full precision, top-k on both sides
        named("verify_ragged_odd", _verify(61, 7, 50001, "f32", "f32", ragged=True, cut=50)),
        # a large served batch, every request with seven drafts of another model
        named("verify_large", _verify(256, 7, 131072, "bf16", "bf16")),
        # the settings of one request's rows of drafts: latency
        named("support_few", _support(8, 32768, "bf16", "mixed")),
        # a large batch whose requests each bring their own settings
        named("support_mixed_large", _support(1024, 131072, "bf16", "mixed")),
        # layer 1's output of the smallest training step, forward
        named("dropout_wires_small", _dropout(1000, 256, "f32", 0.1)),
        # hidden states of a training batch beside their residual, both directions
        named("dropout_hidden_large", _dropout(16384, 8192, "bf16", 0.1, residual=True, backward=True)),
        # one position's hidden state as it is served: latency
        named("norm_one", _norm(1, 8192, "bf16", "e4m3", group=128)),
        # the hidden states of a large batch, one scale per row
        named("norm_large", _norm(32768, 8192, "bf16", "e4m3")),
        # a short batch of odd rows in full precision, gradient
        named("norm_back_odd", _norm_back(509, 1001, "f32")),
        # the gradient of a training batch
        named("norm_back_large", _norm_back(16384, 8192, "bf16")),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "support", "dropout", "norm", "norm_back"])
    pad = rng.choice([0, 0, 0, 8, 3, 32])
    if kind in ("verify", "support"):
        classes = _log(rng, 10, 131072)
        if classes > 64 and rng.random() < 0.4:
            classes = classes // 32 * 32
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"] + ["i32"] * (classes < 2000))
        if kind == "support":
            rows = _log(rng, 1, max(1, min(8192, (1 << 26) // classes)))
            return _support(rows, classes, dtype, rng.choice(["nucleus", "top", "mixed", "mixed"]), pad)
        drafts = rng.randint(1, 8)
        seqs = _log(rng, 1, max(1, min(2048, (1 << 27) // (classes * (drafts + 1)))))
        draft = rng.choice([dtype, dtype, "none", "bf16", "f32"] + ["i32"] * (classes < 2000))
        return _verify(seqs, drafts, classes, dtype, draft, rng.random() < 0.5, rng.choice([0, 0, 0, 5, 40]), pad)
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    cols = _log(rng, 17, 16384)
    if cols > 64 and rng.random() < 0.5:
        cols = cols // 64 * 64
    rows = _log(rng, 1, max(1, min(65536, (1 << (26 if dtype == "f32" else 27)) // cols)))
    if kind == "dropout":
        return _dropout(rows, cols, dtype, rng.choice([0.05, 0.1, 0.25, 0.5, 0.003]), rng.random() < 0.5,
                        rng.random() < 0.5, pad)
    if kind == "norm":
        return _norm(rows, cols, dtype, rng.choice(["e4m3", "e4m3", "u8"]), rng.choice([0, 0, 128, 64]),
                     rng.random() < 0.7, pad)
    return _norm_back(rows, cols, dtype, rng.random() < 0.7, pad)


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _parts(rows, cols):
    step = max(1, (1 << 26) // cols)
    return [slice(r, min(rows, r + step)) for r in range(0, rows, step)]


def _matrix(rows, cols, dtype, pad):
    """Uninitialised [rows, cols] with `pad` unused values after each row."""
    buf = torch.empty(rows, cols + pad, dtype=DTYPES[dtype], device=DEV)
    if pad:
        buf[:, cols:] = 1 << 20 if dtype == "i32" else float("inf")
    return buf[:, :cols]


def _unit(dtype):
    return 50.0 if dtype == "i32" else 1.0     # a hard head's counts per unit of logit


def _store(z, dtype):
    if dtype == "i32":
        return z.mul(50.0).add_(3200.0).round_().clamp_(0.0, 6400.0).to(torch.int32)
    return z.to(DTYPES[dtype])


def _logits(rows, cols, dtype, pad, g):
    x = _matrix(rows, cols, dtype, pad)
    hot = max(1, min(16, cols // 8))
    for s in _parts(rows, cols):
        n = s.stop - s.start
        z = torch.randn(n, cols, generator=g, device=DEV).mul_(2.0)
        # likely classes, apart from each other
        at = torch.randint(0, cols, (n, 1), generator=g, device=DEV) + torch.arange(hot, device=DEV) * (cols // hot)
        z.scatter_add_(1, at % cols, torch.empty(n, hot, device=DEV).exponential_(0.25, generator=g))
        x[s] = _store(z, dtype)
    return x


def _top_support(x, k):
    """floor and last of the k largest logits of every row."""
    rows, cols = x.shape
    floor = torch.empty(rows, device=DEV)
    last = torch.empty(rows, dtype=torch.int32, device=DEV)
    k = min(k, cols)
    for s in _parts(rows, cols):
        v, i = torch.sort(x[s].float(), dim=1, descending=True, stable=True)
        floor[s], last[s] = v[:, k - 1], i[:, k - 1].to(torch.int32)
    return floor, last


def _verify_inputs(case, g):
    S, K, V, pad = case["seqs"], case["drafts"], case["classes"], case["pad"]
    n = torch.full((S,), K, dtype=torch.int64)
    if case["ragged"]:     # from no draft up to K, by the seed alone
        n = torch.randint(0, K + 1, (S,), generator=g, device=DEV).cpu()
        n[0] = K
    first = torch.zeros(S + 1, dtype=torch.int64)
    first[1:] = n.cumsum(0)
    D = int(first[-1])
    target = _logits(D + S, V, case["dtype"], pad, g)
    # target row of every draft
    at = (torch.arange(D) + torch.repeat_interleave(torch.arange(S), n)).to(DEV)
    s = dict(target=target, first=first.to(torch.int32).to(DEV),
             temperature=(0.7 + 0.6 * torch.rand(D + S, generator=g, device=DEV)) * _unit(case["dtype"]))
    s["floor"], s["last"] = _top_support(target, case["cut"]) if case["cut"] else (None, None)
    s["token"] = torch.zeros(D, dtype=torch.int32, device=DEV)
    s["draft"] = s["draft_logprob"] = s["draft_temperature"] = s["draft_floor"] = s["draft_last"] = None
    shift = 3200.0 / 50.0 if case["dtype"] == "i32" else 0.0
    if case["draft"] == "none":        # copied from the prompt: right about every second time
        for p in _parts(D, V):
            z = target[at[p]].float()
            likely = z.argmax(dim=1)
            other = torch.randint(0, V, likely.shape, generator=g, device=DEV)
            s["token"][p] = torch.where(torch.rand(likely.shape, generator=g, device=DEV) < 0.6, likely, other).to(torch.int32)
    else:
        d = case["draft"]
        s["draft"] = _matrix(D, V, d, pad)
        for p in _parts(D, V):         # mostly of the target's opinion
            z = target[at[p]].float() / _unit(case["dtype"]) - shift
            z += 0.5 * torch.randn(z.shape, generator=g, device=DEV)
            s["draft"][p] = _store(z, d)
        T = s["draft_temperature"] = (0.7 + 0.6 * torch.rand(D, generator=g, device=DEV)) * _unit(d)
        if case["cut"]:
            s["draft_floor"], s["draft_last"] = _top_support(s["draft"], case["cut"])
        lp = s["draft_logprob"] = torch.zeros(D, device=DEV)
        cls = torch.arange(V, device=DEV)[None, :]
        for p in _parts(D, V):         # drawn from the draft's kept classes
            z = s["draft"][p].float()
            if case["cut"]:
                f, l = s["draft_floor"][p, None], s["draft_last"][p, None]
                z = torch.where((z > f) | ((z == f) & (cls <= l)), z, NEG)
            y = torch.log_softmax(z / T[p, None], dim=1)
            noise = torch.empty_like(y).exponential_(generator=g).log_()
            tok = (y - noise).argmax(dim=1)
            s["token"][p] = tok.to(torch.int32)
            lp[p] = y.gather(1, tok[:, None]).squeeze(1)
    s["u"] = torch.rand(D, generator=g, device=DEV)
    s["draw_u"] = torch.rand(S, generator=g, device=DEV)
    return s


def _settings(case, g):
    """Per-row temperature, top_k, top_p and min_p (None where unused)."""
    R, mode = case["rows"], case["mode"]
    rand = lambda: torch.rand(R, generator=g, device=DEV)   # noqa: E731

    def pick(values, dtype):
        return torch.tensor(values, dtype=dtype, device=DEV)[torch.randint(0, len(values), (R,), generator=g, device=DEV)]

    s = dict(temperature=(0.6 + 0.8 * rand()) * _unit(case["dtype"]), top_k=None, top_p=None, min_p=None)
    if mode == "nucleus":
        s["top_p"] = 0.8 + 0.19 * rand()
    elif mode == "top":
        s["top_k"] = pick([20, 40, 50, 100], torch.int32)
    else:
        s["temperature"] = torch.where(rand() < 0.05, torch.zeros((), device=DEV), s["temperature"])   # greedy requests
        s["top_k"] = pick([0, 0, 1, 5, 40, 200, 1000], torch.int32)
        s["top_p"] = pick([1.0, 0.5, 0.9, 0.95, 0.99], torch.float32)
        s["min_p"] = pick([0.0, 0.0, 0.02, 0.1], torch.float32)
    return s


def _values(rows, cols, dtype, pad, g, spread=1.0):
    x = _matrix(rows, cols, dtype, pad)
    for s in _parts(rows, cols):
        x[s] = torch.randn(s.stop - s.start, cols, generator=g, device=DEV).mul_(spread).to(DTYPES[dtype])
    return x


def _inputs(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "verify":
        return _verify_inputs(case, g)
    R, pad, dtype = case["rows"], case["pad"], case["dtype"]
    if kind == "support":
        return dict(logits=_logits(R, case["classes"], dtype, pad, g), **_settings(case, g))
    C = case["cols"]
    if kind == "dropout":
        s = dict(x=_values(R, C, dtype, pad, g), residual=_values(R, C, dtype, pad, g) if case["residual"] else None,
                 counter=torch.tensor([(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 62), 3 + int(seed) % 1000],
                                      dtype=torch.int64, device=DEV))
        s["dout"] = _values(R, C, dtype, pad, g) if case["backward"] else None
        return s
    weight = 1.0 + 0.2 * torch.randn(C, generator=g, device=DEV)
    s = dict(weight=weight.to(DTYPES[dtype]), residual=_values(R, C, dtype, pad, g) if case["residual"] else None)
    # some columns of a hidden state stand out
    x = _values(R, C, dtype, pad, g)
    out = torch.randint(0, C, (max(1, C // 256),), generator=g, device=DEV)
    x[:, out] = (x[:, out].float() * 8.0).to(DTYPES[dtype])
    if kind == "norm":
        s["x"] = x
    else:
        s["h"], s["dy"] = x, _values(R, C, dtype, pad, g)
    return s


def _groups(case):
    return -(-case["cols"] // case["group"]) if case["group"] else 1


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "verify":
        S, D = s["draw_u"].numel(), s["u"].numel()
        s["accepted"] = torch.empty(S, dtype=torch.int32, device=DEV)
        s["next_token"] = torch.empty(S, dtype=torch.int32, device=DEV)
        s["logprob"] = torch.empty(S, device=DEV)
        # a generous scratch of any framework's call: 2 KB a row
        s["workspace"] = torch.empty(2048 * (S + D), dtype=torch.uint8, device=DEV)
        return s
    R, pad, dtype = case["rows"], case["pad"], case["dtype"]
    if kind == "support":
        s["floor"], s["last"] = torch.empty(R, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)
        return s
    C = case["cols"]
    if kind == "dropout":
        s["out"] = _matrix(R, C, dtype, pad)
        s["dx"] = _matrix(R, C, dtype, pad) if case["backward"] else None
    elif kind == "norm":
        s["total"] = _matrix(R, C, dtype, pad) if case["residual"] else None
        s["out"] = torch.empty(R, C, dtype=torch.uint8 if case["out"] == "u8" else torch.float8_e4m3fn, device=DEV)
        s["scale"] = torch.empty(R, _groups(case), device=DEV)
    else:
        s["dx"], s["dweight"] = _matrix(R, C, dtype, pad), torch.empty(C, device=DEV)
        # partial sums of the weight's gradient: 4 bytes for each column of up to 1024 blocks
        s["workspace"] = torch.empty(4096 * C, dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------- run --

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_verify(s):
    import paper_2602_07400_gb300 as bl
    bl.bitlogic_verify_drafts(s["target"], s["first"], s["token"], s["u"], s["draw_u"], s["accepted"], s["next_token"],
                              s["workspace"], logprob=s["logprob"], draft=s["draft"], draft_logprob=s["draft_logprob"],
                              temperature=s["temperature"], floor=s["floor"], last=s["last"],
                              draft_temperature=s["draft_temperature"], draft_floor=s["draft_floor"],
                              draft_last=s["draft_last"])
    return dict(accepted=s["accepted"], next_token=s["next_token"], logprob=s["logprob"])


def _own_support(s):
    import paper_2602_07400_gb300 as bl
    bl.bitlogic_support_logits(s["logits"], s["floor"], s["last"], temperature=s["temperature"], top_k=s["top_k"],
                               top_p=s["top_p"], min_p=s["min_p"])
    return dict(floor=s["floor"], last=s["last"])


def _own_dropout(s):
    import paper_2602_07400_gb300 as bl
    p = s["case"]["p"]
    bl.bitlogic_dropout(s["x"], s["out"], s["counter"], p, site=1, residual=s["residual"])
    if s["dout"] is None:
        return dict(out=s["out"])
    bl.bitlogic_dropout(s["dout"], s["dx"], s["counter"], p, site=1)
    return dict(out=s["out"], dx=s["dx"])


def _own_norm(s):
    import paper_2602_07400_gb300 as bl
    case = s["case"]
    bl.bitlogic_norm_bytes(s["x"], s["out"], s["scale"], weight=s["weight"], residual=s["residual"], total=s["total"],
                           group=case["group"], eps=1e-6)
    out = _meaning(s["out"], s["scale"], case) if case["out"] == "u8" else s["out"]
    return dict(out=out, scale=s["scale"], **(dict(total=s["total"]) if case["residual"] else {}))


def _own_norm_back(s):
    import paper_2602_07400_gb300 as bl
    bl.bitlogic_norm_backward(s["dy"], s["h"], s["dx"], weight=s["weight"], dweight=s["dweight"],
                              residual_grad=s["residual"], workspace=s["workspace"], eps=1e-6)
    return dict(dx=s["dx"], dweight=s["dweight"])


_OWN = dict(verify=_own_verify, support=_own_support, dropout=_own_dropout, norm=_own_norm, norm_back=_own_norm_back)


def _per_column(scale, case):
    """Scales [rows, groups] for every column, where there is more than one."""
    return scale.repeat_interleave(case["group"], dim=1)[:, :case["cols"]] if scale.shape[1] > 1 else scale


def _meaning(codes, scale, case):
    # eight bits of meaning, in a type that holds them
    return ((codes.float() - 128.0) * _per_column(scale, case)).to(torch.bfloat16)


def _share(total, x):
    """floor(total * x) for x in [0, 1) held to 24 bits; total below 2^62."""
    x24 = (x * 16777216.0).long()[:, None]
    return (((total >> 32) * x24) << 8) + (((total & 0xFFFFFFFF) * x24) >> 24)


def _weights(z, T, floor, last):
    """The kept logits' powers and whole weights about the row's largest."""
    if floor is not None:
        cls = torch.arange(z.shape[1], device=DEV)[None, :]
        z = torch.where((z > floor[:, None]) | ((z == floor[:, None]) & (cls <= last[:, None])), z, NEG)
    m = z.amax(dim=1, keepdim=True)
    e = torch.where(z > NEG, ((z - m) * (LOG2E / T)[:, None]).exp2(), torch.zeros((), device=DEV))
    return e, (e * 2.0 ** 40).round().long()


def _pick(row, x):
    return row[x] if row is not None else None


def _plain_verify(s):
    V = s["target"].shape[1]
    first = s["first"].long()
    S, D = first.numel() - 1, s["u"].numel()
    n = first[1:] - first[:-1]
    seq = torch.repeat_interleave(torch.arange(S, device=DEV), n, output_size=D)
    at = torch.arange(D, device=DEV) + seq
    # the target's probability of every draft against the draft's own
    _, w = _weights(s["target"].float(), s["temperature"], s["floor"], s["last"])
    total = w.sum(dim=1)
    p = w[at].gather(1, s["token"].long()[:, None]).squeeze(1).double() / total[at].double()
    q = s["draft_logprob"].double().exp() if s["draft"] is not None else torch.ones(D, dtype=torch.float64, device=DEV)
    refused = ~(s["u"].double() * q < p)
    # the first refused draft of every sequence, or all accepted
    order = torch.where(refused, torch.arange(D, device=DEV) - first[seq], D + 1)
    accepted = torch.full((S,), D + 1, device=DEV).scatter_reduce(0, seq, order, "amin")
    accepted = torch.minimum(accepted, n)
    row = first[:-1] + torch.arange(S, device=DEV) + accepted
    all_in = accepted == n
    e, w = _weights(s["target"][row].float(), s["temperature"][row], _pick(s["floor"], row), _pick(s["last"], row))
    total = w.sum(dim=1, keepdim=True)
    weight = w
    if D:
        j = (first[:-1] + accepted).clamp(max=D - 1)
        if s["draft"] is None:
            qv = torch.zeros_like(e).scatter_(1, s["token"][j].long()[:, None], 1.0)
        else:
            ed, wd = _weights(s["draft"][j].float(), s["draft_temperature"][j], _pick(s["draft_floor"], j),
                              _pick(s["draft_last"], j))
            qv = ed * (2.0 ** 40 / wd.sum(dim=1, keepdim=True).float())
        left = ((e * (2.0 ** 40 / total.float()) - qv) * 2.0 ** 40).round().clamp(min=0).long()
        take = ~all_in[:, None] & (left.sum(dim=1, keepdim=True) > 0)
        weight = torch.where(take, left, w)
    sums = weight.cumsum(dim=1)
    token = (sums <= _share(sums[:, -1:], s["draw_u"])).sum(dim=1, keepdim=True)
    logprob = (w.gather(1, token).float() / total.float()).log().squeeze(1)
    return dict(accepted=accepted.to(torch.int32), next_token=token.squeeze(1).to(torch.int32), logprob=logprob)


def _plain_support(s):
    z = s["logits"].float()
    R, V = z.shape
    T = s["temperature"]
    m = z.amax(dim=1, keepdim=True)
    slope = torch.where(T > 0, LOG2E / T, torch.zeros_like(T))[:, None]
    e = ((z - m) * slope).exp2()
    w = (e * 2.0 ** 40).round().long()
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    k = s["top_k"].long() if s["top_k"] is not None else torch.zeros(R, dtype=torch.long, device=DEV)
    k = torch.where(T > 0, torch.where(k > 0, k, V), 1)[:, None]
    keep = torch.arange(V, device=DEV)[None, :] < k
    cut = k < V
    if s["top_p"] is not None:
        ws = torch.where(keep, w.gather(1, order), 0)
        mass = _share(ws.sum(dim=1, keepdim=True), s["top_p"].clamp(max=1.0)).clamp(min=1)
        keep &= (ws.cumsum(dim=1) - ws < mass) | (s["top_p"] >= 1)[:, None]
        cut = cut | (s["top_p"] < 1)[:, None]
    if s["min_p"] is not None:
        keep &= e.gather(1, order) >= s["min_p"][:, None]
        cut = cut | (s["min_p"] > 0)[:, None]
    at = keep.sum(dim=1, keepdim=True) - 1
    floor = torch.where(cut, zs.gather(1, at), NEG)
    last = torch.where(cut, order.gather(1, at), -1)
    return dict(floor=floor.squeeze(1), last=last.squeeze(1).to(torch.int32))


def _philox(block, step, stream, seed):
    """Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011): four words of every
    counter (block, step, stream) under the key `seed`, as int64."""
    M = 0xFFFFFFFF

    def mul(a, b):   # high and low word of the product of 32-bit words
        return (a * (b >> 16) + ((a * (b & 0xFFFF)) >> 16)) >> 16, (a * b) & M

    c0, c1 = block & M, block >> 32
    c2, c3 = (step & M).expand_as(block), torch.full_like(block, stream)
    k0, k1 = seed & M, (seed >> 32) & M
    for _ in range(10):
        h0, l0 = mul(c0, 0xD2511F53)
        h1, l1 = mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    return c0, c1, c2, c3


def _kept(rows, cols, counter, p, site):
    """Element i takes half i % 8 of the words of block i / 8: of stream 2 site
    as its number's high half, of stream 2 site + 1 as the low one."""
    n = rows * cols
    block = torch.arange((n + 7) // 8, device=DEV)

    def halves(stream):
        w = torch.stack(_philox(block, counter[1], stream, counter[0]), dim=1)
        return torch.stack([w & 0xFFFF, w >> 16], dim=2).reshape(-1)[:n]

    number = (halves(2 * site) << 16) | halves(2 * site + 1)
    return (number >= round(p * 4294967296.0)).reshape(rows, cols)


def _plain_dropout(s):
    case = s["case"]
    p, dtype = case["p"], DTYPES[case["dtype"]]
    keep = _kept(case["rows"], case["cols"], s["counter"], p, 1)
    zero = torch.zeros((), device=DEV)
    out = torch.where(keep, s["x"].float() * (1.0 / (1.0 - p)), zero)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    if s["dout"] is None:
        return dict(out=out.to(dtype))
    return dict(out=out.to(dtype), dx=torch.where(keep, s["dout"].float() * (1.0 / (1.0 - p)), zero).to(dtype))


def _plain_norm(s):
    case = s["case"]
    dtype, group, G = DTYPES[case["dtype"]], case["group"], _groups(case)
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * s["weight"].float()
    if group:
        big = torch.nn.functional.pad(y.abs(), (0, G * group - case["cols"])).reshape(-1, G, group).amax(dim=2)
    else:
        big = y.abs().amax(dim=1, keepdim=True)
    most = 127.0 if case["out"] == "u8" else 448.0
    scale = big / most
    q = y * _per_column(torch.where(big > 0, most / big, torch.zeros((), device=DEV)), case)
    if case["out"] == "u8":
        out = _meaning((q.round().clamp(-127.0, 127.0) + 128.0).to(torch.uint8), scale, case)
    else:
        out = q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return dict(out=out, scale=scale, **(dict(total=h.to(dtype)) if s["residual"] is not None else {}))


def _plain_norm_back(s):
    h, dy = s["h"].float(), s["dy"].float()
    rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + 1e-6)
    xh = h * rstd
    gr = dy * s["weight"].float()
    dx = (gr - xh * (gr * xh).mean(dim=1, keepdim=True)) * rstd
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dict(dx=dx.to(DTYPES[s["case"]["dtype"]]), dweight=(dy * xh).sum(dim=0))


_PLAIN = dict(verify=_plain_verify, support=_plain_support, dropout=_plain_dropout, norm=_plain_norm,
              norm_back=_plain_norm_back)


# -------------------------------------------------------------------- work --

def work(case):
    kind, size = case["kind"], BYTES[case["dtype"]]
    if kind == "verify":
        # ragged drafts are half of the most on average; a sequence that meets a
        # refusal reads one row of the draft's
        S, V = case["seqs"], case["classes"]
        D = S * case["drafts"] // 2 if case["ragged"] else S * case["drafts"]
        n = (S + D) * V
        read = n * size + (S * V * BYTES[case["draft"]] // 2 if case["draft"] != "none" else 0)
        return dict(bytes=read + 12 * D + 4 * (S + D) * (1 + 2 * (case["cut"] > 0)) + 20 * S, flops=4 * n)
    if kind == "support":
        n = case["rows"] * case["classes"]
        return dict(bytes=n * size + case["rows"] * 20, flops=4 * n)
    n = case["rows"] * case["cols"]
    if kind == "dropout":
        moved = 2 + case["residual"] + 2 * case["backward"]
        return dict(bytes=moved * n * size, flops=n * 2 * (1 + case["backward"]))
    if kind == "norm":
        moved = 1 + 2 * case["residual"]
        return dict(bytes=moved * n * size + n + 4 * case["rows"] * _groups(case) + case["cols"] * size, flops=8 * n)
    return dict(bytes=(3 + case["residual"]) * n * size + case["cols"] * (size + 4), flops=12 * n)


# ------------------------------------------------------------------- exact --

def exact(case, seed):
    return _EXACT[case["kind"]](case, _inputs(case, seed))


def _exact_probs(z, T, floor, last):
    z = z.double()
    if floor is not None:
        cls = torch.arange(z.shape[1], device=DEV)
        gone = (z < floor.double()[:, None]) | ((z == floor.double()[:, None]) & (cls > last[:, None]))
        z = z.masked_fill(gone, NEG)
    return torch.softmax(z / T.double()[:, None], dim=1)


def _exact_verify(case, v):
    first = v["first"].tolist()
    S, D, V = len(first) - 1, v["u"].numel(), case["classes"]
    seq = [s for s in range(S) for _ in range(first[s + 1] - first[s])]
    rows = torch.tensor([j + s for j, s in enumerate(seq)], dtype=torch.long, device=DEV)
    ok = torch.zeros(D, dtype=torch.bool, device=DEV)
    for p in _parts(D, 2 * V):
        r = rows[p]
        prob = _exact_probs(v["target"][r], v["temperature"][r], _pick(v["floor"], r), _pick(v["last"], r))
        prob = prob.gather(1, v["token"][p].long()[:, None]).squeeze(1)
        q = 1.0 if v["draft"] is None else torch.exp(v["draft_logprob"][p].double())
        ok[p] = v["u"][p].double() * q < prob
    flags = ok.tolist()
    accepted = []
    for s in range(S):
        a = 0
        while first[s] + a < first[s + 1] and flags[first[s] + a]:
            a += 1
        accepted.append(a)
    row = torch.tensor([first[s] + s + accepted[s] for s in range(S)], device=DEV)
    token = []
    for p in _parts(S, 2 * V):
        r = row[p]
        prob = _exact_probs(v["target"][r], v["temperature"][r], _pick(v["floor"], r), _pick(v["last"], r))
        left = prob.clone()
        hit = [(i, first[s] + accepted[s]) for i, s in enumerate(range(p.start, p.stop)) if first[s] + accepted[s] < first[s + 1]]
        if hit:
            i, j = (torch.tensor(t, device=DEV) for t in zip(*hit))
            if v["draft"] is None:
                q = torch.nn.functional.one_hot(v["token"][j].long(), V).double()
            else:
                q = _exact_probs(v["draft"][j], v["draft_temperature"][j], _pick(v["draft_floor"], j), _pick(v["draft_last"], j))
            left[i] = (prob[i] - q).clamp(min=0.0)
        sums = left.cumsum(1)
        t = torch.searchsorted(sums, v["draw_u"][p].double()[:, None] * sums[:, -1:], right=True).clamp_(max=V - 1)
        token.append(t.squeeze(1))
    # a draw that falls on a border of 2^-40 takes another class here, whose
    # logarithm says nothing about theirs
    return dict(accepted=torch.tensor(accepted, dtype=torch.int32, device=DEV),
                next_token=torch.cat(token).to(torch.int32), logprob=None)


def _exact_support(case, v):
    R, V = case["rows"], case["classes"]
    floors, lasts = [], []
    for s in _parts(R, 2 * V):
        z, T = v["logits"][s].double(), v["temperature"][s].double()
        greedy = T <= 0
        prob = torch.softmax(z / T.masked_fill(greedy, 1.0)[:, None], dim=1)
        order = torch.argsort(-z, dim=1, stable=True)
        ps = prob.gather(1, order)
        k = torch.full_like(greedy, V, dtype=torch.long) if v["top_k"] is None else v["top_k"][s].long()
        k = k.masked_fill(k <= 0, V).masked_fill(greedy, 1)[:, None]
        rank = torch.arange(V, device=DEV)[None, :]
        ps = ps * (rank < k)
        kept, whole = rank < k, k >= V
        if v["top_p"] is not None:
            top_p = v["top_p"][s].double()[:, None]
            kept = kept & ((ps.cumsum(1) - ps < top_p * ps.sum(1, keepdim=True)) | (top_p >= 1.0) | (rank == 0))
            whole = whole & (top_p >= 1.0)
        if v["min_p"] is not None:
            min_p = v["min_p"][s].double()[:, None]
            kept = kept & (greedy[:, None] | (prob.gather(1, order) >= min_p * prob.amax(1, keepdim=True)))
            whole = whole & (min_p <= 0)
        at = order.gather(1, kept.sum(1, keepdim=True) - 1)
        floors.append(z.gather(1, at).masked_fill(whole, NEG).squeeze(1))
        lasts.append(at.masked_fill(whole, -1).squeeze(1).to(torch.int32))
    return dict(floor=torch.cat(floors), last=torch.cat(lasts))


def _exact_numbers(n, seed, step, stream):
    """The half words of a stream, from the definition of Philox4x32-10 with
    words cut in 16-bit parts."""
    c = [torch.arange((n + 7) // 8, device=DEV), None, None, None]
    zero = torch.zeros_like(c[0])
    c[1], c[2], c[3] = c[0] // 4294967296, zero + step, zero + stream
    c[0] = c[0] % 4294967296
    key = [seed % 4294967296, seed // 4294967296]
    for r in range(10):
        wide = []
        for word, factor in ((c[0], 0xD2511F53), (c[2], 0xCD9E8D57)):
            a1, a0, b1, b0 = word // 65536, word % 65536, factor // 65536, factor % 65536
            mid = a1 * b0 + (a0 * b0) // 65536
            mid2 = a0 * b1 + mid % 65536
            wide.append((a1 * b1 + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + (a0 * b0) % 65536))
        k = [(key[i] + r * (0x9E3779B9, 0xBB67AE85)[i]) % 4294967296 for i in (0, 1)]
        c = [wide[1][0].bitwise_xor(c[1]).bitwise_xor(k[0]), wide[1][1],
             wide[0][0].bitwise_xor(c[3]).bitwise_xor(k[1]), wide[0][1]]
    return torch.stack([part for w in c for part in (w % 65536, w // 65536)], dim=1).reshape(-1)[:n]


def _exact_dropout(case, v):
    R, C, p = case["rows"], case["cols"], case["p"]
    seed, step = v["counter"].tolist()
    high, low = (_exact_numbers(R * C, seed, step, 2 + i) for i in (0, 1))
    gone = (high * 65536 + low < round(p * 4294967296.0)).reshape(R, C)
    out = (v["x"].double() / (1.0 - p)).masked_fill(gone, 0.0)
    if case["residual"]:
        out += v["residual"].double()
    if not case["backward"]:
        return dict(out=out)
    return dict(out=out, dx=(v["dout"].double() / (1.0 - p)).masked_fill(gone, 0.0))


def _exact_norm(case, v):
    out, scales, totals = [], [], []
    most = 127.0 if case["out"] == "u8" else 448.0
    for s in _parts(case["rows"], 2 * case["cols"]):
        h = v["x"][s].double()
        if case["residual"]:
            h = h + v["residual"][s].double()
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6) * v["weight"].double()
        cols = y.split(case["group"], dim=1) if case["group"] else [y]
        scale = torch.stack([c.abs().amax(1) for c in cols], dim=1) / most
        q = torch.cat([c / scale[:, i, None] for i, c in enumerate(cols)], dim=1)
        out.append(q.round() * _per_column(scale, case) if case["out"] == "u8" else q)
        scales.append(scale)
        totals.append(h)
    return dict(out=torch.cat(out), scale=torch.cat(scales), **(dict(total=torch.cat(totals)) if case["residual"] else {}))


def _exact_norm_back(case, v):
    dx, dw = [], torch.zeros(case["cols"], dtype=torch.float64, device=DEV)
    w = v["weight"].double()
    for s in _parts(case["rows"], 2 * case["cols"]):
        h, dy = v["h"][s].double(), v["dy"][s].double()
        ms = h.square().mean(1, keepdim=True) + 1e-6
        root = ms.sqrt()
        # y = h w / root: d root / d h = h / (C root)
        along = (dy * w * h).sum(1, keepdim=True) / (case["cols"] * ms)
        g = (dy * w - h * along) / root
        dx.append(g + v["residual"][s].double() if case["residual"] else g)
        dw += (dy * h / root).sum(0)
    return dict(dx=torch.cat(dx), dweight=dw)


_EXACT = dict(verify=_exact_verify, support=_exact_support, dropout=_exact_dropout, norm=_exact_norm,
              norm_back=_exact_norm_back)
