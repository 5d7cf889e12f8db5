"""The clusters of the kernels over rows of logits: a block touches another
block's shared memory only after it knows that the other one runs."""
import os
import re

import numpy as np
import pytest
import torch

import logits_ref as ref
from test_gpu_logits import DEV, logits, record, run_distill, run_sample, run_top

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2602_07400_gb300", "csrc")


@pytest.mark.parametrize("name", ["top", "distill", "sample"])
def test_other_blocks_are_waited_for(name):
    with open(os.path.join(CSRC, name + ".cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    kernels = [k for k in text.split("__global__")[1:] if "cluster_size()" in k]
    assert kernels
    for k in kernels:
        first = min(m.start() for m in re.finditer(r"\b(put|store|add)_in_block\(", k))
        report, wait = k.find("report_running(blocks)"), k.find("wait_all_running(blocks)")
        assert 0 <= report < wait < first


@pytest.mark.gpu
def test_rows_over_clusters_in_many_waves():
    """More clusters than fit the card at once, so that blocks start while
    others are far into their rows; every pass over the same rows is the same."""
    T, V = 700, 70000
    x = logits(T, V, "f32", 1, pad=3, shift=1)
    val, idx, lse = record(x, 20, 2, 1.0, True)
    loss, row, g = run_distill(x, val, idx, lse, scale=float(T))
    for t in (0, 151, 152, 350, T - 1):
        l, want, mag = ref.distill(ref.values(x[t:t + 1])[0], val[t].double().cpu().numpy(), idx[t].cpu().numpy(),
                                   float(lse[t]), None, 1.0, 1.0, 1.0, 0.0, 1.0)
        assert abs(float(row[t]) - l) <= 2.0 ** -20 * 64
        assert (np.abs(g[t].double().cpu().numpy() - want) <= 2e-5 * mag + 2.0 ** -24 * np.abs(want) + 1e-37).all()
    for _ in range(5):
        again = run_distill(x, val, idx, lse, scale=float(T))
        assert all(torch.equal(a, b) for a, b in zip((loss, row, g), again))


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(1, 20000), (16, 131072), (75, 131072), (150, 50001)])
def test_record_and_draw_over_clusters(T, V):
    x = logits(T, V, "bf16", V)
    u = torch.rand(T, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    p = torch.full((T,), 0.9, device=DEV)
    top, draw = run_top(x, 40), run_sample(x, u, top_p=p)
    z = ref.values(x[:1])[0]
    np.testing.assert_array_equal(top[1][0], ref.top(z, 40, 1.0)[1])
    assert draw[0][0] in {ref.sample(z, float(u[0]) + d, top_p=np.float32(0.9 + e))[0]
                          for d in (-2.0 ** -18, 0, 2.0 ** -18) for e in (-2.0 ** -18, 0, 2.0 ** -18)}
    for _ in range(10):
        assert all(np.array_equal(a, b) for a, b in zip(top, run_top(x, 40)))
        assert all(np.array_equal(a, b) for a, b in zip(draw, run_sample(x, u, top_p=p)))
