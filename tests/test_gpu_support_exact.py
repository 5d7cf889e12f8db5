"""Supports of rows to the class, of any length and under any settings: the cut in
whole numbers from the powers as a draw rounds them (2^y in fp32, of which CUDA's
exp2f gives the same bits from -64 to 0; below that a weight is 0), so that no
row is too near a border to be held against it."""
import numpy as np
import pytest
import torch

import paper_2602_07400_gb300 as bl
from test_gpu_verify import _f32, _i32, _logits, _unit

pytestmark = pytest.mark.gpu
LOG2E = np.float32(1.4426950408889634)


def _support(z, temperature, top_k, top_p, min_p):
    """(floor, last) of one row of fp32 logits without NaN."""
    V = z.numel()
    zs, order = torch.sort(z, descending=True, stable=True)
    one = not temperature > 0
    k = 1 if one else top_k
    if not (0 < k < V or top_p < 1 or min_p > 0):
        return -np.inf, -1
    if one:
        return float(zs[0]), int(order[0])
    slope = np.float32(np.float32(1) / np.float32(temperature)) * LOG2E
    e = torch.exp2((zs - zs[0]) * float(slope))
    n = k if 0 < k < V else V
    n = min(n, int((zs > -np.inf).sum()))
    if top_p < 1:
        upto = (e[:n].double() * 2.0 ** 40).round().long().cumsum(0)
        want = max(1, (int(upto[-1]) * int(np.float32(top_p) * np.float32(2 ** 24))) >> 24)
        n = int(torch.searchsorted(upto, want)) + 1
    if min_p > 0:
        n = min(n, int((e >= min(float(min_p), 1.0)).sum()))
    return float(zs[n - 1]), int(order[n - 1])


def _check(x, s):
    T = x.shape[0]
    floor, last = torch.full((T,), 7.0, device="cuda"), torch.full((T,), -7, dtype=torch.int32, device="cuda")
    bl.bitlogic_support_logits(x, floor, last, **s)
    torch.cuda.synchronize()
    z = x.float()
    if x.dtype == torch.int32:
        z = torch.where(x == torch.iinfo(torch.int32).min, torch.tensor(-float("inf"), device="cuda"), z)
    h = {n: t.cpu().numpy() for n, t in s.items()}
    f, l = floor.cpu().numpy(), last.cpu().numpy()
    for t in range(T):
        want = _support(z[t], h["temperature"][t], int(h["top_k"][t]), h["top_p"][t], h["min_p"][t])
        assert (f[t], l[t]) == want, (t, (f[t], l[t]), want, {n: v[t] for n, v in h.items()})


CASES = [(80, 7, "f32"), (80, 100, "i32"), (80, 1000, "bf16"), (80, 1025, "f32"), (60, 5000, "bf16"), (60, 20011, "f16"),
         (24, 50001, "f32"), (24, 131072, "bf16"), (24, 131072, "f32"), (8, 300001, "f32"), (4, 1 << 20, "bf16"),
         # a block per row
         (400, 3001, "f16"), (200, 40000, "bf16"), (180, 131072, "bf16"), (180, 50001, "f32")]


@pytest.mark.parametrize("T,V,dtype", CASES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 3)])
def test_any_settings(T, V, dtype, pad, shift):
    rng = np.random.default_rng(V + T)
    x = _logits(T, V, dtype, rng, pad, shift)
    s = dict(temperature=_f32(np.where(rng.random(T) < 0.1, 0.0, 0.5 + rng.random(T)) * _unit(dtype)),
             top_k=_i32(rng.choice([0, 0, 0, 1, 3, 50, 700, 1024, 1025, V - 1, V, V + 5], T)),
             top_p=_f32(rng.choice([1.0, 0.0, 0.3, 0.7, 0.9, 0.99, 0.9999], T)), min_p=_f32(rng.choice([0.0, 0.0, 0.0, 0.05, 1e-6, 1.0], T)))
    _check(x, s)


@pytest.mark.parametrize("T,V,dtype", CASES)
def test_mass_alone(T, V, dtype):
    rng = np.random.default_rng(V)
    x = _logits(T, V, dtype, rng)
    n = lambda v: _f32(np.full(T, v))   # noqa: E731
    for temp in (0.4, 1.0, 3.0):           # heads of few classes, and flat rows
        _check(x, dict(temperature=n(temp * _unit(dtype)), top_k=_i32([0] * T), top_p=_f32(0.02 + 0.979 * rng.random(T)), min_p=n(0.0)))


@pytest.mark.parametrize("T,V,dtype", [c for c in CASES if c[1] > 7])
def test_equal_and_masked_logits(T, V, dtype):
    # few values, so that the cut falls among equal ones; a third of the classes masked
    rng = np.random.default_rng(V + 1)
    z = rng.integers(0, 9, (T, V)) * (40 if dtype == "i32" else 0.75)
    x = torch.from_numpy(z).to(dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16, i32=torch.int32)[dtype]).cuda()
    x[:, ::3] = torch.iinfo(torch.int32).min if dtype == "i32" else float("-inf")
    s = dict(temperature=_f32(np.full(T, _unit(dtype))), top_k=_i32(rng.choice([0, 0, 2, 40, 900, V // 2], T)),
             top_p=_f32(rng.choice([1.0, 0.2, 0.8, 0.95], T)), min_p=_f32(rng.choice([0.0, 0.0, 0.3], T)))
    _check(x, s)
