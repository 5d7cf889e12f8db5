"""A small LUT network beside a larger model, as the operators are used together:
hidden states as samples, a step that learns from the larger model's record with
dropout, drafts drawn from the hard network's counts, and their check."""
import numpy as np
import pytest
import torch

import beside_ref as bref
import paper_2602_07400_gb300 as bl
from paper_2602_07400_gb300 import synth
from paper_2602_07400_gb300.pipeline import (DistillStep, DraftCheck, Features, HardInfer, Network, TeacherRecord,
                                             capture_graph, fit_quantile_thresholds)

D, C, S, K = 48, 20, 30, 4


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
def test_a_network_learns_from_hidden_states_and_drafts(captured):
    B = S * K
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")   # noqa: E731
    hidden, residual = rand(B, D).to(torch.bfloat16), rand(B, D).to(torch.bfloat16)
    weight = 1.0 + 0.1 * rand(D)
    features = Features(D, weight=weight)
    # codes and their thresholds
    codes, total = torch.empty(B, D, dtype=torch.uint8, device="cuda"), torch.empty_like(hidden)
    features.take(hidden, codes, residual=residual, total=total)
    thresholds = fit_quantile_thresholds([codes], 3)
    y = bref.norm(hidden.double().cpu().numpy() + residual.double().cpu().numpy(), weight.double().cpu().numpy(), 1e-6)
    torch.cuda.synchronize()
    want = 128 + np.clip(y / np.float64(np.float32(features.scale)), -127, 127)
    assert np.abs(codes.cpu().numpy() - want).max() <= 0.5 + 1e-3
    # the larger model's answers, from its hidden states
    head = rand(D, C).double()
    def answers(h):
        return (h.double() @ head).float().to(torch.bfloat16)
    wl = synth.Workload("beside", B, D, C, 40.0, tuple(thresholds), (300, 200), 6, 4.0)
    conn1, th1, conn2, th2 = synth.network(wl, seed=0)
    net = Network(conn1, th1, conn2, th2, wl.w_in)
    teacher = TeacherRecord(B, 8, 1.0)
    teacher.take(answers(total))
    step = DistillStep(net, B, D, wl.thresholds, C, wl.tau, teacher, kd_weight=1.0, ce_weight=0.0, dropout=0.1, seed=3)
    features.take(hidden, step.x, residual=residual)
    assert torch.equal(step.x, codes)
    step.labels.fill_(-1)
    run = step.capture().replay if captured else step.run
    masks = []
    for _ in range(3):
        run()
        torch.cuda.synchronize()
        assert torch.isfinite(step.loss).all() and step.dth1.abs().sum() > 0
        masks.append(step.y1 == 0)
        step.update()
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])
    # drafts from the hard network's counts, checked by the larger model
    hard = HardInfer(net, B, D, wl.thresholds, C)
    hard.binarize()
    check = DraftCheck(S, B, C)
    check.first.copy_(torch.arange(0, B + 1, K, dtype=torch.int32))
    T = torch.full((B,), wl.tau, device="cuda")
    k = torch.full((B,), 6, dtype=torch.int32, device="cuda")
    floor, last = torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    u = [torch.rand(n, generator=g, device="cuda") for n in (B, B, S)]
    at = (torch.arange(S * (K + 1), device="cuda") * K // (K + 1)).clamp(max=B - 1)
    target = answers(total)[at].contiguous()

    def serve():
        features.take(hidden, hard.x, residual=residual)
        hard.run()
        hard.draw(u[0], check.token, check.logprob, temperature=T, top_k=k)
        hard.support(floor, last, temperature=T, top_k=k)
        check.run(target, u[1], u[2], draft=hard.counts, draft_temperature=T, draft_floor=floor, draft_last=last)

    if captured:
        graph = capture_graph(serve)
        check.accepted.fill_(-1)
        check.next_token.fill_(-5)
        graph.replay()
    else:
        serve()
    torch.cuda.synchronize()
    z, zd = target.double().cpu().numpy(), hard.counts.double().cpu().numpy()
    tok, lp, fl, la = (t.cpu().numpy() for t in (check.token, check.logprob, floor, last))
    uu, du = u[1].cpu().numpy(), u[2].cpu().numpy()
    for s in range(S):
        rows = [(z[s * (K + 1) + i], 1.0, -np.inf, -1) for i in range(K + 1)]
        j = range(s * K, (s + 1) * K)
        drafts = [(zd[i], wl.tau, fl[i], la[i]) for i in j]
        ok = bref.verdicts(rows, tok[j], lp[j].astype(float), uu[j], du[s], drafts)
        assert (int(check.accepted[s]), int(check.next_token[s])) in ok
    assert bl.bitlogic_device_error() == 0
    # and the features' gradient
    dy, dx, dw = rand(B, D).to(torch.bfloat16), torch.empty_like(hidden), torch.empty(D, device="cuda")
    features.backward(dy, total, dx, dw)
    torch.cuda.synchronize()
    gx, gw = bref.norm_backward(dy.double().cpu().numpy(), total.double().cpu().numpy(), weight.double().cpu().numpy(), 1e-6)
    assert np.abs(dx.double().cpu().numpy() - gx).max() <= 2.0 ** -8 * np.abs(gx).max()
    assert np.abs(dw.double().cpu().numpy() - gw).max() <= 1e-5 * np.abs(gw).max()


@pytest.mark.gpu
def test_dropout_refuses_routes_without_rows():
    wl = synth.Workload("refuse", 16, D, C, 40.0, (64, 128, 192), (100, 40), 6, 4.0)
    net = Network(*synth.network(wl, seed=0), wl.w_in)
    from paper_2602_07400_gb300.pipeline import TrainStep
    for bad in (dict(codes1=True), dict(fuse_dy1=True), dict(through=True)):
        with pytest.raises(ValueError):
            TrainStep(net, 16, D, wl.thresholds, C, wl.tau, dropout=0.1, **bad)
    for p in (-0.1, 1.0, float("nan")):
        with pytest.raises(ValueError):
            TrainStep(net, 16, D, wl.thresholds, C, wl.tau, dropout=p)
    with pytest.raises(ValueError):
        Features(D, scale=0.0)
