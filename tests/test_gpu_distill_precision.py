"""Distillation where nearly all probability lies off the record: the remainder's
share r is near 1, and ln r is small beside the logarithms that it is made of."""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
from test_gpu_distill_remainder import log_sum, on_gpu, row64
from test_gpu_logits import DEV, logits, record

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1000, 3000, 16000, 70000, 430001])
def test_most_of_a_row_off_its_record(V):
    """The record's terms are as exact as their logarithms, 2^-20 of ln V and the
    logits, weighted by q; the remainder's are weighted by q_r, and ln r is off by
    2^-21 of itself or 1 and by what the record's share of the row is off (2^-18)."""
    T, K, tau = 6, 2, 3.5
    x = logits(T, V, "f32", V, scale=1.0)
    val, idx, lse = record(x, K, V + 1, tau, True)
    row, grad = on_gpu("rows")(x, val, idx, lse, None, tau, 1.0, 0.0, 1.0)
    z, v64, i64 = ref.values(x), val.double().cpu().numpy(), idx.cpu().numpy().astype(np.int64)
    for t in range(T):
        l, g, mag = row64(z[t], v64[t], i64[t], float(lse[t]), None, 0.125, tau, 1.0, 0.0, 1.0)
        Q = np.exp(v64[t] / tau - float(lse[t])).sum()
        on = math.exp(log_sum(z[t][i64[t]] / tau) - log_sum(z[t] / tau))
        assert Q < 0.2 and on < 0.2
        size = 1 + np.abs(z[t]).max() / tau + np.abs(v64[t]).max() / tau + math.log(V)
        tol = tau * tau * (Q * 2.0 ** -20 * size + (1 - Q) * (on * 2.0 ** -18 + 2.0 ** -21))
        assert abs(row[t] - l) <= tol, (t, row[t], l, tol)
        assert (np.abs(grad[t] - g) <= 2e-5 * mag + 2.0 ** -24 * np.abs(g) + 1e-37).all(), t
