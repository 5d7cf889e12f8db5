"""Operators on rows of logits (top logits, distillation, sampling) against
plain 64-bit forms (logits_ref), at the sizes, types and masks where they can
go wrong.

Tolerances: values and classes are exact.  A log-sum-exp or a loss is a sum of
terms of the logits' size over the temperature, each rounded a few times in
fp32: 2^-20 of the largest such term.  A gradient is a sum of probabilities
whose exponents (up to 80 in these rows) are rounded a few times in fp32:
2e-5 of the sum of their magnitudes, plus the one rounding to the type.
"""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2602_07400_gb300 as bl

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}
NEG = float("-inf")

# one class to 2^20, around the widths of warps, 16-byte pieces and blocks
SIZES = [1, 2, 3, 7, 10, 31, 32, 33, 64, 100, 127, 255, 257, 1000, 1023, 1024, 1025, 2049, 4099, 8192, 16385]
LONG = [32768, 50001, 65537, 131072, 131075, 262144, 1 << 20]


def logits(T, V, dtype, seed, pad=0, shift=0, scale=3.0, ties=False):
    """[T, V] with `pad` unread values after each row and `shift` before the first."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.empty(T * (V + pad) + shift, dtype=TYPES[dtype], device=DEV)
    x = buf[shift:].view(T, V + pad)[:, :V]
    z = torch.randn(T, V, generator=g, device=DEV) * scale
    z[:, torch.randint(0, V, (max(1, V // 50),), generator=g, device=DEV)] += 4.0
    if ties:
        z = z.round()
    if pad:
        buf.fill_(7 if dtype == "i32" else float("nan"))
    x.copy_((z * 40 + 500).round().clamp(min=0) if dtype == "i32" else z)
    return x


# ------------------------------------------------------------------ top --

def run_top(x, K, tau=1.0, want_lse=True):
    T = x.shape[0]
    val = torch.full((T, K), 777.0, device=DEV)
    idx = torch.full((T, K), 777, dtype=torch.int32, device=DEV)
    lse = torch.full((T,), 777.0, device=DEV) if want_lse else None
    bl.bitlogic_top_logits(x, val, idx, lse, temperature=tau)
    return val.cpu().numpy(), idx.cpu().numpy(), None if lse is None else lse.cpu().numpy()


def check_top(x, K, tau=1.0):
    val, idx, lse = run_top(x, K, tau)
    z = ref.values(x)
    for t in range(x.shape[0]):
        v, i, s = ref.top(z[t], K, tau)
        np.testing.assert_array_equal(idx[t], i, err_msg=f"row {t}")
        np.testing.assert_array_equal(val[t], v, err_msg=f"row {t}")
        if math.isfinite(s):
            fin = z[t][np.isfinite(z[t])]
            assert abs(lse[t] - s) <= 2.0 ** -20 * (1 + np.abs(fin).max() / tau), (t, lse[t], s)
        else:
            assert np.array_equal(lse[t], np.float32(s), equal_nan=True), (t, lse[t], s)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16", "i32"])
@pytest.mark.parametrize("V", SIZES + LONG)
def test_top(V, dtype):
    T = 5 if V < 5000 else 2
    for K in sorted({1, min(V, 10), min(V, 256)}):
        check_top(logits(T, V, dtype, V + K, pad=V % 3, shift=V % 5, scale=1.0 if dtype == "i32" else 3.0), K,
                  50.0 if dtype == "i32" else 1.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 100, 1024, 5000, 40000, 131072])
def test_top_of_equal_sorted_and_masked_rows(V, dtype):
    K = min(V, 200)
    x = logits(11, V, dtype, 5)
    x[0] = 1.0                                             # one value
    x[1] = torch.arange(V, device=DEV) / 8                 # rising (ties where rounded)
    x[2] = -torch.arange(V, device=DEV) / 8                # falling
    x[3] = NEG                                             # nothing ranks
    x[4, 1:] = NEG                                         # one class
    x[5, ::2] = float("nan")                               # NaN does not rank
    x[6, V // 2] = float("inf")
    x[7] = torch.finfo(x.dtype).min                        # the lowest value is a logit
    x[7, V // 3] = NEG
    x[8] = (torch.arange(V, device=DEV) % 2).to(x.dtype)   # two values
    x[9] = 0.0
    x[9, ::2] = -0.0                                       # zeros of both signs are equal
    x[10] = float("nan")
    check_top(x, K)
    check_top(x, 1)


def test_top_counts_masked():
    x = logits(4, 300, "i32", 3)
    x[1, 5:] = -2 ** 31
    x[2] = -2 ** 31
    x[3] = torch.arange(300, device=DEV, dtype=torch.int32) % 7 - 3
    check_top(x, 20, 10.0)


def test_top_many_rows_and_no_lse():
    x = logits(3000, 100, "f32", 9)
    check_top(x, 10)
    val, idx, lse = run_top(x, 10, want_lse=False)
    assert lse is None and (idx >= 0).all()


# -------------------------------------------------------------- distill --

def record(x, K, seed, tau, full_lse):
    """A teacher that mostly agrees with the student's rows."""
    T, V = x.shape
    g = torch.Generator(device=DEV).manual_seed(seed)
    y = 0.9 * x.float().nan_to_num(0.0, 0.0, -30.0) + torch.randn(T, V, generator=g, device=DEV)
    n = min(K, V)
    v, i = y.topk(n, dim=1)
    val = torch.full((T, K), NEG, device=DEV)
    idx = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    val[:, :n], idx[:, :n] = v, i.to(torch.int32)
    return val, idx, torch.logsumexp(y / tau, dim=1) if full_lse else None


def run_distill(x, val, idx, lse, labels=None, weight=None, tau=1.0, kd=1.0, ce=0.0, scale=1.0, grad="rows", **kw):
    T, V = x.shape
    row = torch.full((T,), 777.0, device=DEV)
    loss = torch.full((1,), 777.0, device=DEV)
    g = None
    if grad == "rows":
        g = torch.full((T, V), 777.0, dtype=x.dtype, device=DEV)
    elif grad == "padded":
        g = torch.full((T * (V + 5) + 3,), 777.0, dtype=x.dtype, device=DEV)[3:].view(T, V + 5)[:, :V]
    elif grad == "classes":
        g = torch.full((V, T), 777.0, dtype=x.dtype, device=DEV).t()
    elif grad == "same":
        g = x
    bl.bitlogic_distill_loss(x, val, idx, row, loss, g, teacher_lse=lse, labels=labels, row_weight=weight,
                             temperature=tau, kd_weight=kd, ce_weight=ce, grad_scale=scale, **kw)
    return loss, row, g


def check_distill(x, val, idx, lse, labels=None, weight=None, tau=1.0, kd=1.0, ce=0.0, scale=1.0, grad="rows"):
    T, V = x.shape
    z, v64, i64 = ref.values(x), val.double().cpu().numpy(), idx.cpu().numpy()
    l64 = None if lse is None else lse.double().cpu().numpy()
    loss, row, g = run_distill(x, val, idx, lse, labels, weight, tau, kd, ce, scale, grad)
    lab = None if labels is None else labels.cpu().numpy()
    w = np.full(T, 1.0 / T) if weight is None else weight.double().cpu().numpy()
    row, got = row.double().cpu().numpy(), None if g is None else g.double().cpu().numpy()
    total = tol_total = 0.0
    for t in range(T):
        l, gr, mag = ref.distill(z[t], v64[t], i64[t], None if l64 is None else l64[t],
                                 None if lab is None else int(lab[t]), w[t], tau, kd, ce, scale)
        fin = z[t][np.isfinite(z[t])]
        tv = v64[t][np.isfinite(v64[t])]
        size = 1 + (np.abs(fin).max() if fin.size else 0) + (np.abs(tv).max() if tv.size else 0) + math.log(V)
        tol = 2.0 ** -20 * size * (abs(kd) * tau * max(tau, 1.0) + abs(ce))
        if math.isfinite(l):
            assert abs(row[t] - l) <= tol, (t, row[t], l, tol)
        else:
            assert np.array_equal(row[t], l, equal_nan=True), (t, row[t], l)
        total += w[t] * l if w[t] else 0.0
        tol_total += abs(w[t]) * tol
        if got is not None:
            if math.isnan(l):
                assert np.isnan(got[t]).all(), t
                continue
            bound = 2e-5 * mag + HALF_ULP[x.dtype] * np.abs(gr) + TINY[x.dtype]
            bad = ~(np.abs(got[t] - gr) <= bound)
            assert not bad.any(), (t, np.flatnonzero(bad)[:5], got[t][bad][:5], gr[bad][:5])
    if math.isfinite(total):
        assert abs(float(loss) - total) <= tol_total + 2.0 ** -20 * abs(total), (float(loss), total)
    return loss, row, g


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", SIZES)
def test_distill(V, dtype):
    T = 6
    x = logits(T, V, dtype, V, pad=V % 3, shift=V % 5)
    g = torch.Generator(device=DEV).manual_seed(V)
    labels = torch.randint(-1, V, (T,), generator=g, device=DEV).to(torch.int32)
    weight = torch.rand(T, generator=g, device=DEV)
    weight[2] = 0.0
    # gradients of the size of a type's normal numbers
    for K, tau, tail, lab, wt, grad in [(min(V, 5), 1.0, False, None, None, "rows"),
                                        (min(V, 64), 2.0, True, labels, weight, "padded"),
                                        (min(V + 3, 256), 1.0, True, labels, None, "classes")]:
        val, idx, lse = record(x, K, V + K, tau, tail)
        check_distill(x, val, idx, lse, lab, wt, tau, kd=0.7, ce=0.3 if lab is not None else 0.0, scale=16.0,
                      grad=grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", LONG)
def test_distill_long_rows(V, dtype):
    T = 3
    x = logits(T, V, dtype, V, pad=V % 3, shift=V % 2)
    labels = torch.tensor([V - 1, -1, 0], dtype=torch.int32, device=DEV)
    for K, tau, tail, lab in [(100, 1.0, True, None), (256, 2.5, False, labels)]:
        val, idx, lse = record(x, K, V + K, tau, tail)
        check_distill(x, val, idx, lse, lab, None, tau, kd=0.7, ce=0.3 if lab is not None else 0.0, scale=64.0,
                      grad="padded" if lab is None else "rows")


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [12, 100, 3000, 70000])
def test_distill_masks_and_empty_rows(V, tail):
    T, K = 14, 10
    x = logits(T, V, "f32", V)
    val, idx, lse = record(x, K, 3, 1.0, tail)
    labels = (torch.arange(T, device=DEV) % V).to(torch.int32)
    weight = torch.full((T,), 0.25, device=DEV)
    weight[0] = 0.0
    x[0, 1] = float("nan")                 # a row left out, whatever it holds
    idx[1], val[1] = -1, NEG               # no record
    idx[2, 3:] = -1                        # a short record (its values are not read)
    val[2, 3:] = float("nan")
    x[3] = NEG                             # every class masked
    x[4, idx[4, 1:].long()] = NEG          # masked where the teacher answers: +inf
    val[5, 4:] = NEG                       # teacher probability 0
    off = torch.ones(V, dtype=torch.bool, device=DEV)
    off[idx[6].long()] = False
    x[6, off] = NEG                        # nothing off the record
    labels[6] = idx[6, 2]
    x[7, 3] = float("nan")
    x[8, 4] = float("inf")
    idx[9, 5] = idx[9, 1]                  # a class twice, one thrice
    idx[9, 7] = idx[9, 8] = idx[9, 0]
    labels[9] = idx[9, 0]
    x[10] = torch.finfo(torch.float32).min / 4   # equal and very low
    val[10] = 0.0
    labels[11] = -1
    labels[12] = idx[12, 0]                # the label on the record
    x[13, off] = -60.0                     # a small remainder: the record of row 6 off row 13
    check_distill(x, val, idx, lse, labels, weight, 1.0, kd=0.6, ce=0.4)
    check_distill(x, val, idx, lse, None, weight, 1.0, kd=0.6, grad="classes")
    check_distill(x, val, idx, lse, None, weight, 1.0, kd=0.6, grad=None)
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V", [40, 5000])
def test_distill_no_weight_on_a_term_and_no_teacher_probability(V):
    x = logits(5, V, "f32", 1)
    val, idx, lse = record(x, 8, 2, 1.0, True)
    labels = torch.arange(5, device=DEV).to(torch.int32)
    x[0, idx[0, 0].long()] = NEG
    check_distill(x, val, idx, lse, labels, None, 1.0, kd=0.0, ce=1.0)    # +inf without weight is none
    val[:] = NEG
    check_distill(x, val, idx, None, None, None, 2.0, kd=1.0)


@pytest.mark.parametrize("V", [100, 3001, 40000])
def test_distill_in_place_is_the_same(V):
    x = logits(7, V, "bf16", 4)
    val, idx, lse = record(x, 20, 5, 1.0, True)
    labels = torch.full((7,), 3, dtype=torch.int32, device=DEV)
    loss, row, g = run_distill(x, val, idx, lse, labels, ce=0.5)
    y = x.clone()
    loss2, row2, _ = run_distill(y, val, idx, lse, labels, ce=0.5, grad="same")
    assert torch.equal(y, g) and torch.equal(row, row2) and torch.equal(loss, loss2)


def test_distill_index_out_of_range_is_flagged_and_ignored():
    x = logits(4, 500, "f32", 4)
    val, idx, lse = record(x, 6, 5, 1.0, False)
    bad = idx.clone()
    bad[1, 0] = 500
    cut = idx.clone()
    cut[1, 0] = -1
    labels = torch.tensor([1, 2, 500, 3], dtype=torch.int32, device=DEV)
    none = torch.tensor([1, 2, -1, 3], dtype=torch.int32, device=DEV)
    assert bl.bitlogic_device_error() == 0
    got = run_distill(x, val, bad, lse, labels, ce=0.5)
    assert bl.bitlogic_device_error() == -8 and bl.bitlogic_device_error() == 0
    want = run_distill(x, val, cut, lse, none, ce=0.5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("V,K,tau,tail", [(12, 4, 1.0, True), (40, 8, 2.0, False), (3000, 16, 1.5, True)])
def test_distill_gradient_against_differences(V, K, tau, tail):
    """Central differences of the 64-bit loss, for the gradient's formula, and
    of the operator's own loss along the gradient."""
    x = logits(1, V, "f32", 8)
    val, idx, lse = record(x, K, 9, tau, tail)
    labels = torch.tensor([2], dtype=torch.int32, device=DEV)
    loss, row, g = run_distill(x, val, idx, lse, labels, None, tau, 0.7, 0.3)
    z = ref.values(x)[0]
    args = (val.double().cpu().numpy()[0], idx.cpu().numpy()[0],
            None if lse is None else float(lse[0]), 2, 1.0, tau, 0.7, 0.3, 1.0)
    got = g.double().cpu().numpy()[0]
    h = 1e-5
    for v in list(range(min(V, 12))) + [int(i) for i in idx[0, :4]]:
        a, b = z.copy(), z.copy()
        a[v] += h
        b[v] -= h
        d = (ref.distill(a, *args)[0] - ref.distill(b, *args)[0]) / (2 * h)
        # second differences of a softmax are below 2: h^2 error; 1e-16 / h of rounding
        assert abs(got[v] - d) <= 2e-5 * abs(d) + 1e-7, (v, got[v], d)
    step = 0.05 * g / g.norm()
    up, _, _ = run_distill(x + step, val, idx, lse, labels, None, tau, 0.7, 0.3, grad=None)
    dn, _, _ = run_distill(x - step, val, idx, lse, labels, None, tau, 0.7, 0.3, grad=None)
    want = 0.1 * float(g.norm())
    # third derivatives times 0.05^3 / 3, and fp32 losses
    assert abs(float(up - dn) - want) <= 2e-4 + 1e-2 * want


def test_distill_many_rows_class_major():
    T, V = 2047, 100
    x = logits(T, V, "f32", 3)
    val, idx, lse = record(x, 10, 4, 4.0, True)
    labels = (torch.arange(T, device=DEV) % V).to(torch.int32)
    check_distill(x, val, idx, lse, labels, None, 4.0, 0.7, 0.3, 0.05, grad="classes")


def test_distill_no_rows():
    x = torch.empty(0, 50, device=DEV)
    loss, _, _ = run_distill(x, torch.empty(0, 4, device=DEV), torch.empty(0, 4, dtype=torch.int32, device=DEV), None)
    assert float(loss) == 0.0


# --------------------------------------------------------------- sample --

def run_sample(x, u, **kw):
    T = x.shape[0]
    token = torch.full((T,), 777, dtype=torch.int32, device=DEV)
    logprob = torch.full((T,), 777.0, device=DEV)
    bl.bitlogic_sample_logits(x, u, token, logprob, **kw)
    return token.cpu().numpy(), logprob.cpu().numpy()


# with this temperature the slope is exactly 1, so whole logits give weights
# that are powers of two, exact on both sides
UNIT = 1.4426950408889634


def f32(values):
    return torch.tensor(values, dtype=torch.float32, device=DEV)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def check_exact_draws(x, us, temperature=UNIT, top_k=0, top_p=1.0, min_p=0.0):
    z = ref.values(x)
    T = x.shape[0]
    for u in us:
        token, logprob = run_sample(x, f32([u] * T), temperature=f32([temperature] * T), top_k=i32([top_k] * T),
                                    top_p=f32([top_p] * T), min_p=f32([min_p] * T))
        for t in range(T):
            want, lp = ref.sample(z[t], u, np.float32(temperature), top_k, np.float32(top_p), np.float32(min_p))
            assert token[t] == want, (t, u, top_k, top_p, min_p, token[t], want)
            if math.isfinite(lp):
                assert abs(logprob[t] - lp) <= 2.0 ** -21 * (1 + abs(lp)), (t, logprob[t], lp)
            else:
                assert logprob[t] == lp


US = [0.0, 0.1, 0.5, 0.77, 0.99999994]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16", "i32"])
@pytest.mark.parametrize("V", SIZES + [32768, 50001, 131072])
def test_sample_whole_logits(V, dtype):
    x = logits(3, V, "f32", V, ties=True, pad=V % 3, shift=V % 4)
    if dtype != "f32":
        y = torch.empty(3 * (V + V % 3) + V % 4, dtype=TYPES[dtype], device=DEV)[V % 4:].view(3, V + V % 3)[:, :V]
        y.copy_(x)
        x = y
    few = US if V < 5000 else US[1:4]
    check_exact_draws(x, few)
    check_exact_draws(x, few[1:3], top_k=min(V, 7))
    check_exact_draws(x, few[1:3], top_p=0.6)
    check_exact_draws(x, few[1:3], min_p=0.125)
    check_exact_draws(x, few[1:3], top_k=max(1, V // 3), top_p=0.9, min_p=2.0 ** -6)


@pytest.mark.parametrize("V", [6, 100, 1024, 1025, 20000, 131072])
def test_sample_equal_masked_and_odd_rows(V):
    x = torch.zeros(9, V, device=DEV)
    x[1] = NEG
    x[2, 1:] = NEG
    x[3] = torch.arange(V, device=DEV) % 2
    x[4] = float("nan")
    x[5, V // 2] = float("inf")
    x[6, ::2] = float("nan")
    x[7] = torch.finfo(torch.float32).min
    x[7, V // 2:] = NEG
    x[8] = -torch.arange(V, device=DEV).float()
    for kw in [{}, dict(top_k=3), dict(top_p=0.5), dict(top_k=max(2, V // 2), top_p=0.25), dict(min_p=0.3),
               dict(top_p=0.0), dict(min_p=2.0), dict(top_k=V + 5), dict(temperature=0.0), dict(temperature=-1.0)]:
        check_exact_draws(x, [0.0, 0.4, 0.99999994], **kw)


def test_sample_settings_off_and_u_outside():
    x = logits(4, 200, "f32", 6, ties=True)
    nan = float("nan")
    base = run_sample(x, f32([0.3] * 4), temperature=f32([UNIT] * 4))
    off = run_sample(x, f32([0.3] * 4), temperature=f32([UNIT] * 4), top_k=i32([0, -3, 200, 1 << 30]),
                     top_p=f32([1.0, 2.0, nan, 1.0]), min_p=f32([0.0, -1.0, nan, 0.0]))
    np.testing.assert_array_equal(base[0], off[0])
    np.testing.assert_array_equal(base[1], off[1])
    lo, hi = run_sample(x, f32([0.0] * 4)), run_sample(x, f32([0.99999994] * 4))
    a, b = run_sample(x, f32([-1.0, nan, -0.0, -5.0])), run_sample(x, f32([1.0, 2.0, float("inf"), 1.0]))
    np.testing.assert_array_equal(lo[0], a[0])
    np.testing.assert_array_equal(hi[0], b[0])
    # a temperature of NaN is not > 0; a very small one leaves the largest
    g = run_sample(x, f32([0.7] * 4), temperature=f32([nan, 1e-42, 0.0, 1e-30]))
    top = run_top(x, 1)[1][:, 0]
    assert g[0][0] == top[0] and g[0][2] == top[2]
    z = ref.values(x)
    assert all(z[t][g[0][t]] == z[t].max() for t in range(4))


@pytest.mark.parametrize("dtype,V", [("f32", 10), ("f32", 777), ("bf16", 5003), ("f32", 50001), ("f16", 131072)])
def test_sample_random_settings(dtype, V):
    """Ordinary logits.  The weights' powers are rounded to fp32 (2^-22), so a
    draw may differ from the 64-bit one only where u lies as close to the edge
    of its class's share, or the cut to a class: both are looked for with u
    moved by 2^-18."""
    T = 24
    x = logits(T, V, dtype, V)
    g = torch.Generator(device=DEV).manual_seed(V)
    u = (torch.rand(T, generator=g, device=DEV) * 0.99 + 0.005)
    temp = 0.5 + torch.rand(T, generator=g, device=DEV)
    k = torch.tensor([0, 1, 3, 40, 200, 2000] * 4, dtype=torch.int32, device=DEV)
    p = f32([1.0, 0.9, 0.5, 0.95] * 6)
    mp = f32([0.0, 0.0, 0.05] * 8)
    token, logprob = run_sample(x, u, temperature=temp, top_k=k, top_p=p, min_p=mp)
    z = ref.values(x)
    eps = 2.0 ** -18
    for t in range(T):
        ok = []
        for du in (0.0, -eps, eps):
            for dp in (0.0, -eps, eps):
                pp = np.float32(float(p[t]) + dp) if float(p[t]) < 1 else np.float32(1)
                ok.append(ref.sample(z[t], float(u[t]) + du, np.float32(temp[t].item()), int(k[t]), pp, np.float32(mp[t].item())))
        assert int(token[t]) in [a for a, _ in ok], (t, token[t], ok)
        lp = [b for a, b in ok if a == int(token[t])][0]
        assert abs(logprob[t] - lp) <= 1e-4 + 1e-5 * abs(lp)


def test_sample_draws_follow_the_probabilities():
    V, n = 37, 40000
    row = logits(1, V, "f32", 2)
    x = row.expand(n, V).contiguous()
    u = (torch.arange(n, device=DEV).float() + 0.5) / n
    token, _ = run_sample(x, u)
    share = np.bincount(token, minlength=V) / n
    p = torch.softmax(row[0].double(), 0).cpu().numpy()
    # equally spaced u: each class's share is met within one step at both edges
    np.testing.assert_allclose(share, p, atol=2.0 / n + 1e-6)


def test_sample_does_not_depend_on_the_batch():
    V = 9000
    x = logits(300, V, "bf16", 11)
    g = torch.Generator(device=DEV).manual_seed(1)
    u = torch.rand(300, generator=g, device=DEV)
    p = torch.full((300,), 0.9, device=DEV)
    a = run_sample(x, u, top_p=p)
    for t in (0, 7, 299):
        b = run_sample(x[t:t + 1], u[t:t + 1], top_p=p[t:t + 1])
        assert a[0][t] == b[0][0] and a[1][t] == b[1][0]


# ------------------------------------------------- streams, graphs, rows --

@pytest.mark.parametrize("V", [100, 40000])
def test_on_another_stream_and_in_a_graph(V):
    from paper_2602_07400_gb300.pipeline import capture_graph
    x = logits(8, V, "bf16", 3)
    val, idx, lse = torch.empty(8, 16, device=DEV), torch.empty(8, 16, dtype=torch.int32, device=DEV), torch.empty(8, device=DEV)
    row, loss, grad = torch.empty(8, device=DEV), torch.empty(1, device=DEV), torch.empty_like(x)
    token, logprob, u = torch.empty(8, dtype=torch.int32, device=DEV), torch.empty(8, device=DEV), torch.rand(8, device=DEV)
    p = torch.full((8,), 0.9, device=DEV)

    def all_three(stream=None):
        bl.bitlogic_top_logits(x, val, idx, lse, stream=stream)
        bl.bitlogic_distill_loss(x, val, idx, row, loss, grad, teacher_lse=lse, stream=stream)
        bl.bitlogic_sample_logits(x, u, token, logprob, top_p=p, stream=stream)
        return [t.clone() for t in (val, idx, lse, row, loss, grad, token, logprob)]

    want = all_three()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = all_three(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = capture_graph(lambda: all_three())
    for t in (val, idx, lse, row, loss, grad, token, logprob):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (val, idx, lse, row, loss, grad, token, logprob)))
    # a record of the row itself: no loss but rounding
    assert float(row.abs().max()) < 1e-5


def test_offsets_past_32_bits():
    """Rows far apart: the last one starts past 2^32 elements."""
    V, T = 1000, 3
    ld = (1 << 31) + 8
    buf = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (T, V), (ld, 1))
    small = logits(T, V, "bf16", 1)
    x.copy_(small)
    check_top(x, 10)
    val, idx, lse = record(small, 10, 5, 1.0, True)
    a, b = run_distill(x, val, idx, lse), run_distill(small, val, idx, lse)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    u = f32([0.2, 0.5, 0.9])
    np.testing.assert_array_equal(run_sample(x, u)[0], run_sample(small, u)[0])
    run_distill(x, val, idx, lse, grad="same")
    assert torch.equal(x, b[2])
