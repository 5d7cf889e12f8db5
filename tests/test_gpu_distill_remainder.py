"""Distillation where the classes off the record lie far below the record's, by
up to the type's lowest value: the remainder's loss and gradient against a
64-bit form that carries the remainder's logarithm.

Tolerances: a loss is a sum of differences of logits over the temperature, each
rounded a few times in fp32: 2^-20 of the largest such term.  A gradient is a sum
of powers: 2e-5 of the sum of their magnitudes, the rounding to the type, and
what a probability below 2^-126 (which counts as 0) may be off by.
"""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2602_07400_gb300 as bl

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALL = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}
GAPS = [0.0, 60.0, 80.0, 84.0, 86.5, 88.0, 90.0, 104.0, 200.0, 2000.0, 1e4, math.inf]   # inf: the type's lowest value
Q = [0.5, 0.2, 0.07, 0.03]


def log_sum(z):
    m = z.max() if len(z) else -math.inf
    return m if math.isinf(m) else m + math.log(np.exp(z - m).sum())


def row64(z, val, idx, t_lse, label, w, tau, kd, ce, scale):
    """Loss, gradient and the magnitude of its terms of a row of finite or
    masked logits and a record of different classes."""
    y = z / tau - (z / tau).max()
    logp = y - log_sum(y)
    on = np.zeros(len(z), bool)
    on[idx] = True
    norm = t_lse if t_lse is not None else log_sum(val / tau)
    logq = val / tau - norm
    q = np.zeros(len(z))
    q[idx] = np.exp(logq)
    kl = (np.exp(logq) * (logq - logp[idx])).sum()
    logr = log_sum(logp[~on])
    qr = max(0.0, 1.0 - q.sum()) if t_lse is not None and logr > -math.inf else 0.0
    p = np.exp(logp)
    g, mag = (q.sum() + qr) * p - q, (q.sum() + qr) * p + q
    if qr > 0:
        kl += qr * (math.log(qr) - logr)
        share = np.exp(y[~on] - y[~on].max())   # about their own largest: its digits hide their sum's
        share *= qr / share.sum()
        g[~on] -= share
        mag[~on] += share
    loss, g, mag = kd * tau * tau * kl, kd * tau * g, kd * tau * mag
    if label is not None:
        x = z - z.max()
        logs = x - log_sum(x)
        s = np.exp(logs)
        loss -= ce * logs[label]
        g, mag = g + ce * s, mag + ce * s
        g[label] -= ce
        mag[label] += ce
    return loss, g * (w * scale), mag * (w * scale)


def far_rows(V, dtype, tau, device, seed=0):
    """A row per gap: the record's classes near 0, the rest `gap` times the
    temperature below, every third of them masked in every second row; one more
    row has nothing off the record."""
    g = torch.Generator().manual_seed(seed + V)
    T, K = len(GAPS) + 1, len(Q)
    z = torch.randn(T, V, generator=g)
    idx = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)])
    low = torch.finfo(TYPES[dtype]).min
    for t, gap in enumerate(GAPS):
        on = z[t, idx[t]].clone()
        z[t] = low if math.isinf(gap) else (z[t] - gap * tau).clamp(min=low)
        if t % 2:
            z[t, ::3] = -math.inf
        z[t, idx[t]] = on
    z[T - 1] = -math.inf
    z[T - 1, idx[T - 1]] = 0.25
    val = (tau * torch.tensor(Q).double().log()).float().expand(T, K).contiguous()
    return z.to(TYPES[dtype]).to(device), val.to(device), idx.to(torch.int32).to(device)


def check_rows(call, x, dtype, val, idx, lse, labels, tau, kd, ce, scale, w):
    row, grad = call(x, val, idx, lse, labels, tau, kd, ce, scale)
    z = ref.values(x)
    v64, i64 = val.double().cpu().numpy(), idx.cpu().numpy().astype(np.int64)
    for t in range(x.shape[0]):
        label = None if labels is None else int(labels[t])
        l, g, mag = row64(z[t], v64[t], i64[t], None if lse is None else float(lse[t]), label, w, tau, kd, ce, scale)
        if label is not None and z[t][label] == -math.inf:
            assert row[t] == math.inf
        else:
            fin = z[t][np.isfinite(z[t])]
            size = 1 + np.abs(fin).max() + math.log(len(z[t]))
            assert abs(row[t] - l) <= 2.0 ** -20 * size * (kd * tau * max(tau, 1.0) + ce), (t, row[t], l)
        flush = 2.0 ** -126 * w * scale * (kd * tau + ce)
        bad = ~(np.abs(grad[t] - g) <= 2e-5 * mag + HALF_ULP[dtype] * np.abs(g) + SMALL[dtype] + flush)
        assert not bad.any(), (t, np.flatnonzero(bad)[:5], grad[t][bad][:5], g[bad][:5])


def on_gpu(major):
    def call(x, val, idx, lse, labels, tau, kd, ce, scale):
        T, V = x.shape
        row, loss = torch.empty(T, device=DEV), torch.empty(1, device=DEV)
        g = torch.empty(V, T, dtype=x.dtype, device=DEV).t() if major == "classes" else torch.empty_like(x)
        weight = torch.full((T,), 0.125, device=DEV)
        bl.bitlogic_distill_loss(x, val, idx, row, loss, g, teacher_lse=lse, labels=labels, row_weight=weight,
                                 temperature=tau, kd_weight=kd, ce_weight=ce, grad_scale=scale)
        return row.double().cpu().numpy(), g.double().cpu().numpy()
    return call


def label_of(x, idx):
    """A class off the record, masked in no row but the last two kinds."""
    T, V = x.shape
    return torch.tensor([next(v for v in range(1, V) if v % 3 and v not in set(idx[t].tolist())) for t in range(T)],
                        dtype=torch.int32, device=x.device)


@pytest.mark.gpu
# a warp per row; a block; a cluster; rows streamed twice
@pytest.mark.parametrize("V,dtype", [(12, "f32"), (1000, "bf16"), (3000, "f32"), (8000, "f16"), (70000, "f32"), (131072, "bf16"),
                                     (430001, "f32"), (860003, "bf16")])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_classes_off_the_record_far_below(V, dtype, tau):
    x, val, idx = far_rows(V, dtype, tau, DEV)
    lse = torch.zeros(x.shape[0], device=DEV)
    scale = 1024.0 if dtype == "f16" else 65536.0
    check_rows(on_gpu("rows"), x, dtype, val, idx, lse, None, tau, 1.0, 0.0, scale, 0.125)
    check_rows(on_gpu("classes"), x, dtype, val, idx, lse, label_of(x, idx), tau, 0.7, 0.3, scale, 0.125)
    check_rows(on_gpu("rows"), x, dtype, val, idx, None, label_of(x, idx), tau, 0.7, 0.3, scale, 0.125)
