"""A student LUT network trained on a teacher's record, and answers drawn from
a hard network's counts, through the pipeline's classes."""
import math

import numpy as np
import pytest
import torch

import logits_ref as ref
import oracle
import paper_2602_07400_gb300 as bl
from paper_2602_07400_gb300 import synth
from paper_2602_07400_gb300.pipeline import DistillStep, HardInfer, Network, TeacherRecord, TrainStep
from parity_util import check_fwd, check_grad

pytestmark = pytest.mark.gpu


def _workload(k, batch=100, classes=10):
    return synth.Workload("t", batch, 40, classes, 40.0, (64, 128, 192), (240, 40 * classes // 2), k, 6.0)


def _step(wl, K, temperature, seed=0, **kw):
    conn1, th1, conn2, th2 = synth.network(wl, seed=seed)
    net = Network(conn1, th1, conn2, th2, wl.w_in)
    teacher = TeacherRecord(wl.batch, K, temperature)
    st = DistillStep(net, wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau, teacher, **kw)
    x, labels = synth.blob_batch(wl.batch, wl.d, wl.classes, wl.sigma, seed=seed + 1)
    st.load(x.cuda(), labels.cuda())
    return st, teacher, x, labels, (conn1, th1, conn2, th2)


@pytest.mark.parametrize("k,batch,tail", [(6, 100, True), (6, 101, False), (2, 100, True), (4, 67, True)])
def test_step_against_the_oracle(k, batch, tail):
    """Class gradients from the 64-bit form on the step's logits; table
    gradients from the oracle's backward on those class gradients."""
    wl = _workload(k, batch)
    tau_d = 2.0
    st, teacher, x, labels, (conn1, th1, conn2, th2) = _step(wl, 4, tau_d, kd_weight=0.7, ce_weight=0.3, tail=tail)
    g = torch.Generator(device="cuda").manual_seed(3)
    teacher.take(torch.randn(batch, wl.classes, generator=g, device="cuda") * 3)
    st.labels[5] = -1                      # a sample without a label
    st.row_weight = torch.full((batch,), 1.0 / batch, device="cuda")
    st.row_weight[7] = 0.0
    st.run()
    torch.cuda.synchronize()
    assert bl.bitlogic_device_error() == 0
    r = oracle.train_step(x.numpy(), labels.numpy(), wl.thresholds, conn1, th1, conn2, th2, wl.classes, wl.tau)
    check_fwd(st.logits, r["logits"], "logits")
    z = st.logits.double().cpu().numpy()
    dyg = np.zeros((wl.classes, batch))
    total = 0.0
    for s in range(batch):
        w = float(st.row_weight[s])
        l, gr, _ = ref.distill(z[s], teacher.val[s].double().cpu().numpy(), teacher.idx[s].cpu().numpy(),
                               float(teacher.lse[s]) if tail else None, int(st.labels[s]), w, tau_d, 0.7, 0.3, 1 / wl.tau)
        total += w * l
        dyg[:, s] = gr
    assert abs(float(st.loss) - total) <= 1e-5 * abs(total)
    check_grad(st.dyg, dyg, "class gradients")
    y1, bits = r["y1"], r["bits"]
    dth2, dy1 = oracle.lut_backward(y1, conn2, th2, np.repeat(dyg, st.net.w2 // wl.classes, axis=0), want_dx=True)
    dth1, _ = oracle.lut_backward(bits, conn1, th1, dy1, want_dx=False)
    check_grad(st.dth2, dth2, "dtheta2")
    check_grad(st.dth1, dth1, "dtheta1")


def test_without_a_teacher_it_is_the_training_step():
    wl = _workload(6)
    st, teacher, x, labels, params = _step(wl, 3, 1.0, kd_weight=0.0, ce_weight=1.0)
    st.run()
    plain = TrainStep(Network(*params, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau)
    plain.load(x.cuda(), labels.cuda())
    plain.run()
    torch.cuda.synchronize()
    assert abs(float(st.loss) - float(plain.loss)) <= 1e-5 * float(plain.loss)
    for n in ("dyg", "dth1", "dth2"):
        a, b = getattr(st, n), getattr(plain, n)
        assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max()), n


def test_graph_replay_is_the_step():
    wl = _workload(6)
    st, teacher, *_ = _step(wl, 4, 2.0)
    teacher.take(torch.randn(wl.batch, wl.classes, device="cuda"))
    st.run()
    want = [t.clone() for t in (st.loss, st.row_loss, st.dth1, st.dth2)]
    graph = st.capture()
    for t in (st.loss, st.row_loss, st.dth1, st.dth2):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (st.loss, st.row_loss, st.dth1, st.dth2)))


def test_a_hard_teachers_record_and_the_loss_along_the_gradient():
    """A wide hard network's counts are recorded, and the student's loss moves
    along the step's table gradients as they say: L(theta + h g) - L(theta - h g)
    = 2 h |g|^2, with h for a change of a hundredth of the loss.  The third-order
    term of so small a step is below that fraction squared, and the losses are
    fp32 (1e-5 of the change each): 2e-3 of the change."""
    wl = _workload(4, batch=512)
    conn1, th1, conn2, th2 = synth.network(synth.Workload("w", 512, 40, 10, 40.0, (64, 128, 192), (600, 500), 4, 6.0), seed=9)
    hard = HardInfer(Network(conn1, th1, conn2, th2, wl.w_in), 512, wl.d, wl.thresholds, wl.classes)
    st, teacher, x, labels, _ = _step(wl, 5, 1.0, seed=4, kd_weight=1.0, ce_weight=0.0)
    hard.x.copy_(x.cuda())
    hard.binarize()
    hard.run()
    teacher.take(hard.counts, unit=2.0)
    counts = hard.counts.double().cpu().numpy() / 2.0
    for s in (0, 100, 511):
        v, i, lse = ref.top(counts[s], 5, 1.0)
        np.testing.assert_array_equal(teacher.idx[s].cpu().numpy(), i)
        np.testing.assert_allclose(teacher.val[s].cpu().numpy(), v, rtol=1e-6)
        assert abs(float(teacher.lse[s]) - lse) <= 1e-4
    st.run()
    g1, g2, base = st.dth1.clone(), st.dth2.clone(), float(st.loss)
    norm2 = float(g1.double().square().sum() + g2.double().square().sum())
    h = 0.01 * base / (2 * norm2)
    th1, th2 = st.net.theta1.clone(), st.net.theta2.clone()
    got = []
    for sign in (1.0, -1.0):
        st.net.theta1.copy_(th1 + sign * h * g1)
        st.net.theta2.copy_(th2 + sign * h * g2)
        st.run()
        got.append(float(st.row_loss.double().mean()))
    want = 2 * h * norm2
    assert abs((got[0] - got[1]) - want) <= 2e-3 * want, (got, want)


def test_answers_drawn_from_counts():
    wl = _workload(4, batch=3000)
    conn1, th1, conn2, th2 = synth.network(wl, seed=2)
    hard = HardInfer(Network(conn1, th1, conn2, th2, wl.w_in), 3000, wl.d, wl.thresholds, wl.classes)
    x, _ = synth.blob_batch(3000, wl.d, wl.classes, wl.sigma, seed=3)
    hard.x.copy_(x.cuda())
    hard.binarize()
    hard.run()
    token = torch.empty(3000, dtype=torch.int32, device="cuda")
    logprob = torch.empty(3000, device="cuda")
    u = torch.rand(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    # greedy answers are the argmax, first maximum included
    hard.draw(u, token, temperature=torch.zeros(3000, device="cuda"))
    assert torch.equal(token, hard.pred)
    t = torch.full((3000,), 6.0, device="cuda")
    k = torch.full((3000,), 4, dtype=torch.int32, device="cuda")
    hard.draw(u, token, logprob, temperature=t, top_k=k)
    z = hard.counts.double().cpu().numpy()
    kept = np.stack([np.isin(np.arange(wl.classes), ref.order(row)[:4]) for row in z])
    p = np.exp((z - z.max(1, keepdims=True)) / 6.0) * kept
    p /= p.sum(1, keepdims=True)
    got = token.cpu().numpy()
    assert kept[np.arange(3000), got].all()
    np.testing.assert_allclose(logprob.cpu().numpy(), np.log(p[np.arange(3000), got]), atol=1e-5)
    # the mean probability of what was drawn: sum p^2 on average, within four
    # standard errors of 3000 draws of numbers in [0, 1]
    assert abs(p[np.arange(3000), got].mean() - (p ** 2).sum(1).mean()) <= 4 * 0.5 / math.sqrt(3000)
