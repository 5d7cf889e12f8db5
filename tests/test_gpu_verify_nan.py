"""A NaN among the target's logits is never weighed by the draw, wherever a row's
threads meet it: before their first finite logit, and at the row's ends."""
import numpy as np
import pytest
import torch

import paper_2602_07400_gb300 as bl
from test_gpu_verify import DTYPES, Batch

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
LANES = {"f32": 4, "bf16": 8, "f16": 8}     # classes of 16 bytes


def _spoil(x, r, kind, V, N):
    """Row r of x with NaN where all threads that meet one go on to finite logits,
    or only one of them does; a thread starts with the pieces of N classes
    128 (t / 32) + t % 32 + 32 i of the row, i < 4."""
    first = min(1024 * N, V // 2)
    if kind == 0:                       # the first batch of every thread
        x[r, :first] = NAN
    elif kind == 1:                     # one among masked ones
        x[r, :first] = -INF
        x[r, 37] = NAN
    elif kind == 2:                     # the first 512 classes
        x[r, :512] = NAN
    elif kind == 3:                     # the first classes of every warp's run
        x[r, :first] = -INF
        x[r, 0:first:128 * N] = NAN
    elif kind == 4:                     # the row's last piece alone is finite, behind a NaN of the same thread
        x[r, :V - V % N - (N if V % N == 0 else 0)] = -INF
        x[r, 128 * N + 1] = NAN
    elif kind == 5:                     # the same at its beginning
        x[r, 1:] = -INF
        x[r, N:2 * N] = NAN
        x[r, 32 * N:33 * N] = NAN
    elif kind == 6:                     # every second batch, from the first on
        for a in range(0, V - first, 2 * first):
            x[r, a:a + first] = NAN
    elif kind == 7:                     # all but the last class
        x[r, :V - 1] = NAN


def _batch(S, V, dtype, draft, seed, shift):
    b = Batch([1] * S, V, dtype, draft, seed, 3 * shift, shift)
    b.u.fill_(0.97)                     # refused mostly, and drawn from the row that refused
    if draft is None:
        b.token.fill_(5)
    else:
        b.lp.fill_(-0.1)
    for s in range(S):
        _spoil(b.target, 2 * s, s % 8, V, LANES[dtype])
        _spoil(b.target, 2 * s + 1, (s + 3) % 8, V, LANES[dtype])
    return b


@pytest.mark.parametrize("V", [1030, 9001, 20011, 60000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_whole_rows(V, dtype, shift):
    # as many rows as a block takes whole
    b = _batch(176, V, dtype, dtype, 7, shift)
    b.run().check(range(0, 176, 7))
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V,dtype", [(20011, "f32"), (60000, "bf16")])
def test_drafts_that_were_not_drawn(V, dtype):
    _batch(176, V, dtype, None, 8, 1).run().check(range(0, 176, 7))
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V,dtype", [(1 << 20, "f32"), ((1 << 20) - 3, "bf16"), (300001, "f16"), (131072, "bf16")])
@pytest.mark.parametrize("S", [1, 4, 16])
def test_rows_in_parts(V, dtype, S):
    for seed in range(2 if S < 16 else 1):
        b = Batch([1] * S, V, dtype, dtype, seed, 3, 1)
        b.u.fill_(0.97)
        b.lp.fill_(-0.1)
        for s in range(S):
            _spoil(b.target, 2 * s, (s + 4 * seed) % 8, V, LANES[dtype])
            part = V // 32              # and where a later part begins
            b.target[2 * s + 1, 5 * part:5 * part + 1024 * LANES[dtype]] = -INF
            b.target[2 * s + 1, 5 * part + 300] = NAN
        b.run().check(range(0, S, max(1, S // 4)))
    assert bl.bitlogic_device_error() == 0


def test_rows_that_hold_nothing_else():
    # NaN and -inf alone: no class
    b = Batch([0] * 320, 20011, "bf16", None, 9)
    b.target.fill_(-INF)
    b.target[::2, ::3] = NAN
    b.target[::4] = NAN
    b.run()
    torch.cuda.synchronize()
    assert (b.next == -1).all() and (b.logprob == -np.inf).all()
