"""Operators on rows of logits where rows are many or longer than a cluster
holds: rows by one block that reads them several times, in batches of pieces and
groups of pieces.  Ordinary rows and the odd ones (equal, rising, masked, NaN,
infinite logits) against the plain 64-bit forms, at row ends off 16 bytes."""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
import test_gpu_logits as base
from test_gpu_logits import DEV, NEG, TYPES, UNIT, f32, i32, logits, record, run_distill, run_sample, run_top

pytestmark = pytest.mark.gpu

ODD = 12


def odd_rows(x):
    """The first rows of x (whole logits) made odd ones."""
    V = x.shape[1]
    at = torch.arange(V, device=DEV)
    x[0] = 1.0
    x[1] = (at * 64 // V).to(x.dtype)                 # rising in runs of equal logits
    x[2] = (-(at * 64 // V)).to(x.dtype)              # falling
    x[3] = NEG
    x[4, :V - 1] = NEG                                # the last class alone
    x[5, ::2] = float("nan")
    x[6, V // 2] = float("inf")
    x[7] = torch.finfo(x.dtype).min
    x[7, V // 3] = NEG
    x[8] = (at % 2).to(x.dtype)
    x[9, V // 3:] = NEG
    x[10] = float("nan")
    x[11, : V // 2] = NEG
    return x


def whole_rows(T, V, dtype, pad, shift):
    x = logits(T, V, "f32", V + T, ties=True)
    y = torch.full((T * (V + pad) + shift,), float("nan"), dtype=TYPES[dtype], device=DEV)[shift:].view(T, V + pad)[:, :V]
    y.copy_(x)
    return odd_rows(y)


def draw(z, u, temperature, top_k, top_p, min_p):
    """logits_ref.sample with its whole-number sums in 64 bits (weights of up to
    2^40, of fewer than 2^20 classes)."""
    o = ref.order(z)
    if len(o) == 0:
        return -1, -math.inf
    if not temperature > 0 or np.isposinf(z[o[0]]):
        return int(o[0]), 0.0
    ok = z > -np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        y = (z.astype(np.float32) - np.float32(z[o[0]])) * np.float32(np.float32(1) / np.float32(temperature) * ref.LOG2E)
        e = np.where(ok, np.exp2(np.where(ok, y.astype(np.float64), -np.inf)), 0.0)
    w = np.rint(e * 2.0 ** 40).astype(np.uint64)
    kept = o[:top_k] if 0 < top_k < len(o) else o
    if top_p < 1:
        sums = np.cumsum(w[kept])
        kept = kept[:int(np.searchsorted(sums, np.uint64(max(1, ref.share(int(sums[-1]), top_p))))) + 1]
    if min_p > 0:
        kept = kept[e[kept] >= min(np.float32(min_p), np.float32(1))]
    kept = np.sort(kept)
    sums = np.cumsum(w[kept])
    at = int(np.searchsorted(sums, np.uint64(ref.share(int(sums[-1]), u)), side="right"))
    return int(kept[at]), math.log(int(w[kept[at]]) / int(sums[-1]))


SETTINGS = [dict(), dict(top_k=7), dict(top_k=1000), dict(top_k=1500), dict(top_p=0.6), dict(top_p=0.97), dict(min_p=0.125),
            dict(top_p=0.9, min_p=2.0 ** -4), dict(top_k=900, top_p=0.5, min_p=2.0 ** -5), dict(temperature=0.0)]


@pytest.mark.parametrize("V,dtype,pad,shift", [(1500, "f32", 1, 1), (16385, "bf16", 3, 5), (50001, "f32", 2, 3), (131072, "bf16", 0, 0),
                                               (70001, "f16", 1, 7)])
def test_sample(V, dtype, pad, shift):
    """More rows than the card has SMs: a block per row."""
    T = torch.cuda.get_device_properties(0).multi_processor_count + 9
    x = whole_rows(T, V, dtype, pad, shift)
    rows = list(range(ODD)) + [ODD, T // 2, T - 1]
    z = ref.values(x[rows])
    for n, kw in enumerate(SETTINGS):
        for u in (0.0, 0.3, 0.77, 0.99999994)[n % 2::2]:
            s = dict(temperature=UNIT, top_k=0, top_p=1.0, min_p=0.0)
            s.update(kw)
            token, logprob = run_sample(x, f32([u] * T), temperature=f32([s["temperature"]] * T), top_k=i32([s["top_k"]] * T),
                                        top_p=f32([s["top_p"]] * T), min_p=f32([s["min_p"]] * T))
            for i, t in enumerate(rows):
                args = z[i], u, np.float32(s["temperature"]), s["top_k"], np.float32(s["top_p"]), np.float32(s["min_p"])
                want, lp = draw(*args)
                assert V > 2000 or (want, lp) == ref.sample(*args)
                assert token[t] == want, (t, u, kw, token[t], want)
                if math.isfinite(lp):
                    assert abs(logprob[t] - lp) <= 2.0 ** -21 * (1 + abs(lp)), (t, kw, logprob[t], lp)
                else:
                    assert logprob[t] == lp


def test_sample_settings_of_each_row():
    """Rows of one batch under settings of their own: as each draws alone."""
    T, V = 200, 40000
    x = whole_rows(T, V, "bf16", 1, 2)
    g = torch.Generator(device=DEV).manual_seed(3)
    u = torch.rand(T, generator=g, device=DEV)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device=DEV)[torch.randint(0, len(values), (T,), generator=g, device=DEV)]   # noqa: E731
    kw = dict(temperature=pick([UNIT, 0.0, 2 * UNIT], torch.float32), top_k=pick([0, 0, 1, 50, 1000, 3000], torch.int32),
              top_p=pick([1.0, 0.5, 0.9, 0.99], torch.float32), min_p=pick([0.0, 0.0, 0.125], torch.float32))
    token, logprob = run_sample(x, u, **kw)
    for t in range(T):
        a, b = run_sample(x[t:t + 1], u[t:t + 1], **{n: v[t:t + 1] for n, v in kw.items()})
        assert a[0] == token[t] and b[0] == logprob[t], (t, {n: float(v[t]) for n, v in kw.items()})


@pytest.mark.parametrize("V,dtype,pad,shift", [(1500, "f32", 1, 1), (4099, "bf16", 3, 5), (20000, "f32", 0, 0), (50001, "f32", 2, 3),
                                               (131072, "bf16", 0, 0), (131075, "f16", 1, 7)])
def test_top(V, dtype, pad, shift):
    """Rows from half a row per SM on: a block per row."""
    T = torch.cuda.get_device_properties(0).multi_processor_count
    rows = list(range(ODD)) + [ODD, T // 2, T - 1]
    for x in (whole_rows(T, V, dtype, pad, shift), odd_rows(logits(T, V, dtype, 7, pad=pad, shift=shift))):
        z = ref.values(x[rows])
        for K in (1, 200, 256):
            val, idx, lse = run_top(x, K, 1.5)
            for i, t in enumerate(rows):
                v, j, s = ref.top(z[i], K, 1.5)
                np.testing.assert_array_equal(idx[t], j, err_msg=f"row {t}")
                np.testing.assert_array_equal(val[t], v, err_msg=f"row {t}")
                if math.isfinite(s):
                    fin = z[i][np.isfinite(z[i])]
                    assert abs(lse[t] - s) <= 2.0 ** -20 * (1 + np.abs(fin).max() / 1.5), (t, lse[t], s)
                else:
                    assert np.array_equal(lse[t], np.float32(s), equal_nan=True), (t, lse[t], s)


def test_top_counts():
    x = logits(200, 5000, "i32", 5, pad=1, shift=3)
    x[1, 100:] = -2 ** 31
    x[2] = -2 ** 31
    x[3] = torch.arange(5000, device=DEV, dtype=torch.int32) % 7 - 3
    val, idx, lse = run_top(x, 100, 50.0)
    z = ref.values(x)
    for t in (0, 1, 2, 3, 100, 199):
        v, i, s = ref.top(z[t], 100, 50.0)
        np.testing.assert_array_equal(idx[t], i)
        np.testing.assert_array_equal(val[t], v)
        assert (lse[t] == s) if math.isinf(s) else abs(lse[t] - s) <= 2.0 ** -20 * (1 + np.abs(z[t][np.isfinite(z[t])]).max() / 50.0)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_odd_rows_longer_than_a_cluster(tail):
    base.test_distill_masks_and_empty_rows(430001, tail)


@pytest.mark.parametrize("V", [430001, 860003])
def test_distill_longer_than_a_cluster_in_place(V):
    base.test_distill_in_place_is_the_same(V)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_distill_longer_than_a_cluster(dtype):
    """Labels, weights and the gradient's layouts."""
    T, V = 4, 860003
    x = logits(T, V, dtype, 1, pad=3, shift=5)
    val, idx, lse = record(x, 200, 2, 2.0, True)
    labels = torch.tensor([V - 1, int(idx[1, 7]), -1, 0], dtype=torch.int32, device=DEV)
    weight = torch.tensor([0.5, 0.25, 0.0, 0.25], device=DEV)
    for grad in ("rows", "padded", "classes"):
        base.check_distill(x, val, idx, lse, labels, weight, 2.0, kd=0.7, ce=0.3, scale=64.0, grad=grad)


@pytest.mark.parametrize("dtype,V", [("f32", 3000), ("f32", 8000), ("f32", 20000), ("f32", 50000), ("bf16", 12000), ("bf16", 40000),
                                     ("f16", 131072)])
@pytest.mark.parametrize("grad", ["rows", "classes"])
def test_distill_many_odd_rows(dtype, V, grad):
    """Rows by 64, 128 and 256 threads and by clusters of two and four: the odd
    rows once against the 64-bit form, and each of their copies the same."""
    n, times, K = 12, 14, 50
    g = torch.Generator(device=DEV).manual_seed(V)
    x = logits(n, V, dtype, V)
    val, idx, lse = record(x, K, 3, 1.0, True)
    labels = torch.randint(0, V, (n,), generator=g, device=DEV).to(torch.int32)
    weight = torch.full((n,), 1.0 / n, device=DEV)
    weight[0], x[0, 1] = 0.0, float("nan")
    idx[1], val[1] = -1, NEG
    idx[2, 9:] = -1
    x[3] = NEG
    x[4, idx[4, 1:].long()] = NEG
    val[5, 4:] = NEG
    off = torch.ones(V, dtype=torch.bool, device=DEV)
    off[idx[6].long()] = False
    x[6, off] = NEG
    labels[6] = idx[6, 2]
    x[7, V - 1] = float("nan")
    x[8, V // 2] = float("inf")
    idx[9, 5] = idx[9, 1]
    idx[9, 7:9] = idx[9, 0]
    labels[9] = idx[9, 0]
    labels[10] = -1
    x[11] = 2.0
    base.check_distill(x, val, idx, lse, labels, weight, 1.0, 0.6, 0.4, 16.0, grad)
    many = lambda t: t.repeat(times, *[1] * (t.dim() - 1))   # noqa: E731
    X, args = many(x), (many(val), many(idx), many(lse), many(labels), many(weight) / times)
    loss, row, out = run_distill(X, *args, 1.0, 0.6, 0.4, 16.0 * times, grad)
    z, i64, l64 = ref.values(x), idx.cpu().numpy(), lse.double().cpu().numpy()
    v64, w64 = val.double().cpu().numpy(), args[4][:n].double().cpu().numpy()
    got = out.double().cpu().numpy()
    for t in range(n):
        for copy in range(1, times):
            assert torch.equal(row[t].nan_to_num(-5.0), row[copy * n + t].nan_to_num(-5.0))
        same = torch.as_strided(out, (times, V), (n * out.stride(0), out.stride(1)), out.storage_offset() + t * out.stride(0))
        assert torch.equal(same.nan_to_num(-5.0, 7e4, -7e4), same[:1].nan_to_num(-5.0, 7e4, -7e4).expand_as(same)), t
        l, gr, mag = ref.distill(z[t], v64[t], i64[t], l64[t], int(labels[t]), w64[t], 1.0, 0.6, 0.4, 16.0 * times)
        if math.isnan(l):
            assert np.isnan(got[t]).all() and math.isnan(float(row[t]))
            continue
        assert float(row[t]) == l if math.isinf(l) else abs(float(row[t]) - l) <= 2.0 ** -20 * 64   # terms of up to 64
        assert (np.abs(got[t] - gr) <= 2e-5 * mag + base.HALF_ULP[x.dtype] * np.abs(gr) + base.TINY[x.dtype]).all(), t


def test_rows_around_a_row():
    """A record's values and classes and a draw are the same in any batch; sums
    are up to their rounding."""
    T, V = 200, 30000
    x = logits(T, V, "bf16", 9)
    u, p = torch.rand(T, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV), torch.full((T,), 0.9, device=DEV)
    top, draw = run_top(x, 50), run_sample(x, u, top_p=p)
    val, idx, lse = record(x, 50, 4, 1.0, True)
    weight = torch.ones(T, device=DEV)
    _, row, grad = run_distill(x, val, idx, lse, None, weight)
    for t in (0, 99, T - 1):
        one = slice(t, t + 1)
        a, b = run_top(x[one], 50), run_sample(x[one], u[one], top_p=p[one])
        assert np.array_equal(a[0][0], top[0][t]) and np.array_equal(a[1][0], top[1][t])
        assert b[0][0] == draw[0][t] and b[1][0] == draw[1][t]
        assert abs(a[2][0] - top[2][t]) <= 2.0 ** -20 * (1 + np.abs(ref.values(x[one])).max())
        _, r, g = run_distill(x[one], val[one], idx[one], lse[one], None, weight[one])
        assert abs(float(r[0] - row[t])) <= 2.0 ** -20 * 64
        # one more rounding to bf16 on each side where sums differ
        assert (g[0].float() - grad[t].float()).abs().max() <= 2.0 ** -7 * grad[t].float().abs().max()
