"""A training step with dropout: passes without it, and its gradient down to the wires."""
import numpy as np
import pytest
import torch

import beside_ref as bref
import oracle
from paper_2602_07400_gb300.pipeline import Network, TrainStep
from test_gpu_dropout import _small

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k,B", [(6, 96), (6, 97), (2, 50)])
def test_a_pass_without_dropout_in_between(k, B):
    wl, conn1, th1, conn2, th2, x, labels = _small(k, B=B)
    make = lambda **kw: TrainStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau,   # noqa: E731
                                  through=False, fuse_dy1=False, codes1=False, **kw)
    a, b = make(), make(dropout=0.5, seed=3)
    for st in (a, b):
        st.load(x.cuda(), labels.cuda())
    b.run()
    torch.cuda.synchronize()
    dropped = b.y1.clone()
    b.dropout = 0.0
    for st in (a, b):
        st.run()
    torch.cuda.synchronize()
    for name in ("y1", "y2", "logits", "loss", "dth1", "dth2", "dy1"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    b.dropout = 0.5
    b.run()                      # the counter has not moved: the same mask
    torch.cuda.synchronize()
    assert torch.equal(b.y1, dropped) and not torch.equal(b.dth1, a.dth1)


@pytest.mark.parametrize("k,B", [(6, 96), (2, 50)])
def test_the_input_gradient(k, B):
    wl, conn1, th1, conn2, th2, x, labels = _small(k, B=B)
    st = TrainStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau, want_dx1=True,
                   dropout=0.25, seed=77)
    st.load(x.cuda(), labels.cuda())
    st.run()
    torch.cuda.synchronize()
    theta1, theta2 = st.net.theta1.cpu().numpy(), st.net.theta2.cpu().numpy()
    bits = oracle.encode_thermometer(x.numpy(), wl.thresholds)
    keep = bref.kept_values(0, wl.widths[0] * B, 77, 0, 0.25, 0).reshape(wl.widths[0], B)
    y1 = oracle.lut_forward(bits, conn1, theta1) * keep / 0.75
    _, _, dY = oracle.head_loss(oracle.lut_forward(y1, conn2, theta2), labels.numpy(), wl.classes, wl.tau)
    _, dy1 = oracle.lut_backward(y1, conn2, theta2, dY)
    dth1, dbits = oracle.lut_backward(bits, conn1, theta1, dy1 * keep / 0.75)
    for got, want in ((st.dy1, dy1 * keep / 0.75), (st.dbits, dbits), (st.dth1, dth1)):
        assert np.abs(got.cpu().numpy() - want).max() <= 1e-4 * np.abs(want).max()
