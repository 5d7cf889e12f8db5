"""Distillation against records whose values are large: only their differences
count, so neither a loss nor a gradient may lose digits to their size."""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
from test_gpu_distill_remainder import on_gpu, row64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BASES = [0.0, 6e3, 1e5, 2.0 ** 25, -(2.0 ** 25), -1e30]
STEPS = [[0, 0, 0, 0, 0], [0, -4, -8, 4, 4], [0, 0, -64, -64, -400]]


def large_records(V, device):
    """A row per base and pattern of differences (whole multiples of 4: exact in
    fp32 up to 2^25; -1e30 swallows them)."""
    g = torch.Generator().manual_seed(V)
    T = len(BASES) * len(STEPS)
    x = torch.randn(T, V, generator=g) * 2
    idx = torch.stack([torch.randperm(V, generator=g)[:5] for _ in range(T)]).to(torch.int32)
    val = torch.tensor([[b + s for s in steps] for b in BASES for steps in STEPS], dtype=torch.float32)
    return x.to(device), val.to(device), idx.to(device)


def check_large(call, x, val, idx, tau):
    row, grad = call(x, val, idx, None, None, tau, 1.0, 0.0, 1.0)
    z, v64, i64 = ref.values(x), val.double().cpu().numpy(), idx.cpu().numpy().astype(np.int64)
    v64 -= v64.max(axis=1, keepdims=True)   # a softmax of them is the same
    for t in range(x.shape[0]):
        l, g, mag = row64(z[t], v64[t], i64[t], None, None, 0.125, tau, 1.0, 0.0, 1.0)
        # terms: q ln q with differences up to 408 / tau, and the student's logits
        size = 1 + 408 / tau + np.abs(z[t]).max() + math.log(x.shape[1])
        assert abs(row[t] - l) <= 2.0 ** -20 * size * tau * max(tau, 1.0), (t, row[t], l)
        bad = ~(np.abs(grad[t] - g) <= 2e-5 * mag + 2.0 ** -24 * np.abs(g) + 1e-37)
        assert not bad.any(), (t, np.flatnonzero(bad)[:5], grad[t][bad][:5], g[bad][:5])


@pytest.mark.parametrize("V", [12, 1000, 3000, 70000, 430001])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
def test_large_values_of_a_record(V, tau):
    check_large(on_gpu("rows"), *large_records(V, DEV), tau)


@pytest.mark.parametrize("V", [12, 1000, 3000, 70000, 430001])
def test_values_far_above_the_log_sum_exp_show(V):
    """A record under a log-sum-exp that is not its own: q = exp(a) as long as
    fp32 holds it, and no finite loss or gradient beyond."""
    above = [0.5, 3.0, 60.0, 87.0, 90.0, 100.0, 177.5, 1e4]
    T = len(above)
    g = torch.Generator().manual_seed(V)
    x = torch.randn(T, V, generator=g).to(DEV)
    idx = torch.randint(0, V, (T, 1), generator=g).to(torch.int32).to(DEV)
    val = torch.tensor(above, dtype=torch.float32, device=DEV)[:, None] + 2.0
    lse = torch.full((T,), 2.0, device=DEV)
    row, grad = on_gpu("rows")(x, val, idx, lse, None, 1.0, 1.0, 0.0, 1.0)
    z, v64 = ref.values(x), val.double().cpu().numpy()
    for t, a in enumerate(above):
        if a > 88:
            assert not np.isfinite(row[t]) and not np.isfinite(grad[t]).any(), a
            continue
        l, gr, mag = row64(z[t], v64[t], idx[t].cpu().numpy().astype(np.int64), 2.0, None, 0.125, 1.0, 1.0, 0.0, 1.0)
        # q is as exact as its exponent, off by a 2^-24 at most, beside the loss's own terms
        size = 1 + a + np.abs(z[t]).max() + math.log(V)
        if abs(l) > np.finfo(np.float32).max:   # past what a loss is held in
            assert row[t] == math.inf
        else:
            assert abs(row[t] - l) <= (2.0 ** -20 + a * 2.0 ** -24) * size * math.exp(a), (a, row[t], l)
        assert (np.abs(grad[t] - gr) <= (2e-5 + a * 2.0 ** -24) * mag + 1e-37).all(), a


@pytest.mark.parametrize("V", [12, 1000, 3000, 70000, 430001])
def test_nan_of_a_record_shows(V):
    """A NaN among a row's entries, or in its log-sum-exp, is in the row's loss
    and gradient and in no other row's; a place without an entry is not read."""
    T, nan = 6, math.nan
    g = torch.Generator().manual_seed(V)
    x = torch.randn(T, V, generator=g).to(DEV)
    idx = torch.stack([torch.randperm(V, generator=g)[:4] for _ in range(T)]).to(torch.int32).to(DEV)
    val = torch.randn(T, 4, generator=g).to(DEV)
    lse = torch.full((T,), 3.0, device=DEV)
    call = on_gpu("rows")
    for own in (None, lse):
        v, i = val.clone(), idx.clone()
        v[1, 2] = nan
        v[2, :] = nan
        v[3, 3], i[3, 3] = nan, -1
        want = [False, True, True, False, False, False]
        if own is not None:
            own = own.clone()
            own[4] = nan
            want[4] = True
        row, grad = call(x, v, i, own, None, 1.0, 1.0, 0.0, 1.0)
        for t in range(T):
            assert np.isnan(row[t]) == want[t], (t, row)
            assert (np.isnan(grad[t]).all() if want[t] else np.isfinite(grad[t]).all()), t
