"""Dropout on the GPU against Philox4x32-10 on the CPU, and in the training step."""
import numpy as np
import pytest
import torch

import beside_ref as bref
import oracle
import paper_2602_07400_gb300 as bl
from paper_2602_07400_gb300 import synth
from paper_2602_07400_gb300.pipeline import DistillStep, Network, TeacherRecord, TrainStep

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def test_the_reference_generator_gives_the_published_words():
    # known answers of Philox4x32-10: counter and key all 0, and all ones
    w = [int(x[0]) for x in bref.philox([0], 0, 0, 0)]
    assert w == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    w = [int(x[0]) for x in bref.philox([(1 << 64) - 1], 0xFFFFFFFF, 0xFFFFFFFF, (1 << 64) - 1)]
    assert w == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def _counter(seed, step):
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


def _matrix(R, C, dtype, pad=0, shift=0, fill=None):
    buf = torch.empty(R * (C + pad) + shift + 16, dtype=dtype, device="cuda")
    x = buf[shift:shift + R * (C + pad)].view(R, C + pad)[:, :C]
    if fill is None:
        x.normal_()
    else:
        x.fill_(fill)
    return x


def _expected(x, keep, p, residual):
    y = np.where(keep, x.double().cpu().numpy() * (1.0 / (1.0 - p)), 0.0)
    return y if residual is None else y + residual.double().cpu().numpy()


def _check(out, want, terms):
    # the scale, the product and the sum are rounded to fp32 (2^-24 each of the
    # terms), the result to its type by half a step (of a subnormal one at least)
    eps = torch.finfo(out.dtype).eps / 2
    got = out.double().cpu().numpy()
    tol = eps * np.abs(want) * 1.0001 + 3 * 2.0 ** -24 * terms + torch.finfo(out.dtype).smallest_normal * eps * 2
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


SHAPES = [(1, 1), (1, 7), (3, 8), (1, 8), (2, 9), (5, 1001), (1000, 256), (64, 4096), (7, 33), (3, 70001), (0, 5), (5, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("R,C", SHAPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1), (0, 1)])
def test_dropout_against_its_definition(R, C, dtype, pad, shift):
    for i, (p, residual, site) in enumerate([(0.1, False, 0), (0.5, True, 3), (0.9, True, 1 << 30), (0.0, False, 7)]):
        x = _matrix(R, C, dtype, pad, shift)
        r = _matrix(R, C, dtype, pad, shift) if residual else None
        out = _matrix(R, C, dtype, pad, shift, 7.0)
        seed, step = -5 - i * (1 << 40), (1 << 33) + i
        bl.bitlogic_dropout(x, out, _counter(seed, step), p, site, residual=r)
        torch.cuda.synchronize()
        keep = bref.kept_values(0, R * C, seed & ((1 << 64) - 1), step, p, site).reshape(R, C)
        want = _expected(x, keep, p, r)
        terms = np.abs(x.double().cpu().numpy()) / (1 - p) + (np.abs(r.double().cpu().numpy()) if residual else 0)
        _check(out, want, terms)
        if not residual and p:
            assert ((out == 0).cpu().numpy() >= ~keep).all()
        # in place, and on the residual's place
        for at in ("x", "r") if residual else ("x",):
            y = _matrix(R, C, dtype, pad, shift, 0.0)
            y.copy_(x if at == "x" else r)
            bl.bitlogic_dropout(y if at == "x" else x, y, _counter(seed, step), p, site, residual=r if at == "x" else (y if residual else None))
            torch.cuda.synchronize()
            assert torch.equal(y, out)


@pytest.mark.gpu
def test_the_low_halves_decide_where_the_high_ones_are_level():
    # thresholds whose high half is one value: about n / 2^16 elements are level
    n = 1 << 20
    x = torch.ones(1, n, device="cuda")
    for p in (0.5 + 2.0 ** -18, 0.25 + 2.0 ** -17 + 2.0 ** -32, 2.0 ** -20, 1.0 - 2.0 ** -20, 2.0 ** -32, 2.0 ** -34):
        out = torch.empty_like(x)
        bl.bitlogic_dropout(x, out, _counter(99, 1), p)
        torch.cuda.synchronize()
        keep = bref.kept_values(0, n, 99, 1, p, 0)
        assert np.array_equal(out.cpu().numpy()[0] != 0, keep)


@pytest.mark.gpu
def test_dropped_values_are_zero_whatever_they_hold():
    x = torch.full((4, 1000), float("nan"), device="cuda")
    out = torch.empty_like(x)
    bl.bitlogic_dropout(x, out, _counter(1, 2), 0.5)
    torch.cuda.synchronize()
    keep = bref.kept_values(0, 4000, 1, 2, 0.5, 0).reshape(4, 1000)
    assert np.array_equal(np.isnan(out.cpu().numpy()), keep) and (out.cpu().numpy()[~keep] == 0).all()


@pytest.mark.gpu
def test_the_mask_does_not_go_by_type_or_strides():
    want = None
    for dtype in DTYPES:
        for pad, shift in ((0, 0), (8, 0), (1, 0), (0, 3)):
            x = _matrix(37, 1024, dtype, pad, shift, 1.0)
            out = _matrix(37, 1024, dtype, pad, shift, 0.0)
            bl.bitlogic_dropout(x, out, _counter(7, 7), 0.3, 2)
            torch.cuda.synchronize()
            mask = (out != 0).cpu()
            want = mask if want is None else want
            assert torch.equal(mask, want)
    for seed, step, site in ((8, 7, 2), (7, 8, 2), (7, 7, 3), (7 + (1 << 32), 7, 2)):
        x, out = torch.ones(37, 1024, device="cuda"), torch.empty(37, 1024, device="cuda")
        bl.bitlogic_dropout(x, out, _counter(seed, step), 0.3, site)
        torch.cuda.synchronize()
        same = ((out != 0).cpu() == want).float().mean()
        assert abs(float(same) - (0.7 ** 2 + 0.3 ** 2)) <= 6 * np.sqrt(0.25 / want.numel())   # independent masks


@pytest.mark.gpu
def test_elements_past_32_bits():
    R, C = 70001, 65536      # 4.6e9 elements
    x = torch.ones(R, C, dtype=torch.bfloat16, device="cuda")
    bl.bitlogic_dropout(x, x, _counter(3, 4), 0.25)
    torch.cuda.synchronize()
    for row in (0, 65535, 65536, R - 1):
        keep = bref.kept_values(row * C, C, 3, 4, 0.25, 0)
        assert np.array_equal((x[row] != 0).cpu().numpy(), keep), row
    y = x.view(-1)[: (R - 1) * C + 5].view(1, -1)     # no multiple of eight: the path for any length
    y.fill_(1.0)
    bl.bitlogic_dropout(y, y, _counter(3, 4), 0.25)
    torch.cuda.synchronize()
    tail = bref.kept_values((R - 2) * C, C + 5, 3, 4, 0.25, 0)
    assert np.array_equal((y[0, (R - 2) * C:] != 0).cpu().numpy(), tail)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_gradient_is_the_same_call_and_agrees_with_differences(dtype):
    x, g = _matrix(50, 200, dtype), _matrix(50, 200, dtype)
    r = _matrix(50, 200, dtype)
    c = _counter(11, 5)
    dx = torch.empty_like(x)
    bl.bitlogic_dropout(g, dx, c, 0.4, 9)
    # L = sum g out is linear in x: L(x + e d) - L(x - e d) = 2 e <dx, d> but for roundings
    d = torch.sign(torch.randn(50, 200, device="cuda")).to(dtype)
    def loss(v):
        out = torch.empty(50, 200, device="cuda")
        bl.bitlogic_dropout(v.float(), out, c, 0.4, 9, residual=r.float())
        return (g.double() * out.double()).sum()
    diff = float(loss(x.float() + d.float()) - loss(x.float() - d.float())) / 2
    want = float((dx.double() * d.double()).sum())
    # dx is rounded to its type, out to fp32
    tol = float((dx.double().abs().sum()) * torch.finfo(dtype).eps / 2 + (g.double().abs() * 20).sum() * 2.0 ** -23)
    assert abs(diff - want) <= tol


@pytest.mark.gpu
def test_a_captured_call_drops_anew_when_the_step_advances():
    x, out = torch.ones(64, 512, device="cuda"), torch.empty(64, 512, device="cuda")
    c = _counter(21, 0)
    g = torch.cuda.CUDAGraph()
    bl.bitlogic_dropout(x, out, c, 0.5)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        bl.bitlogic_dropout(x, out, c, 0.5)
    for step in range(3):
        c[1] = step
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal((out != 0).cpu().numpy().reshape(-1), bref.kept_values(0, x.numel(), 21, step, 0.5, 0))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    bl.bitlogic_dropout(x, out, c, 0.25, stream=st)
    st.synchronize()
    assert np.array_equal((out != 0).cpu().numpy().reshape(-1), bref.kept_values(0, x.numel(), 21, 2, 0.25, 0))


def _small(k=6, classes=4, d=40, B=96):
    wl = synth.Workload("small", B, d, classes, 40.0, (64, 128, 192), (256, 128), k, 4.0)
    conn1, th1, conn2, th2 = synth.network(wl, seed=0)
    x, labels = synth.blob_batch(wl.batch, wl.d, wl.classes, wl.sigma, seed=1)
    return wl, conn1, th1, conn2, th2, x, labels


@pytest.mark.gpu
@pytest.mark.parametrize("k,B,node", [(6, 96, "soft"), (6, 97, "soft"), (2, 96, "soft"), (6, 96, "st"), (2, 50, "soft")])
@pytest.mark.parametrize("captured", [False, True])
def test_the_training_step_drops_layer_1(k, B, node, captured):
    wl, conn1, th1, conn2, th2, x, labels = _small(k, B=B)
    st = TrainStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau, node=node,
                   dropout=0.25, seed=77)
    st.load(x.cuda(), labels.cuda())
    run = st.run
    if captured:
        run = st.capture().replay
    for step in range(2):
        run()
        torch.cuda.synchronize()
        theta1, theta2 = st.net.theta1.cpu().numpy(), st.net.theta2.cpu().numpy()
        bits = oracle.encode_thermometer(x.numpy(), wl.thresholds)
        keep = bref.kept_values(0, wl.widths[0] * B, 77, step, 0.25, 0).reshape(wl.widths[0], B)
        y1 = oracle.lut_forward(bits, conn1, theta1, node) * keep / 0.75
        y2 = oracle.lut_forward(y1, conn2, theta2, node)
        logits, loss, dY = oracle.head_loss(y2, labels.numpy(), wl.classes, wl.tau)
        dth2, dy1 = oracle.lut_backward(y1, conn2, theta2, dY, node=node)
        dth1, _ = oracle.lut_backward(bits, conn1, theta1, dy1 * keep / 0.75, node=node)
        assert abs(float(st.loss) - loss) <= 1e-5 * abs(loss)
        for got, want, tol in ((st.y1, y1, 1e-5), (st.y2, y2, 1e-5), (st.dth2, dth2, 1e-4), (st.dth1, dth1, 1e-4)):
            assert np.abs(got.cpu().numpy() - want).max() <= tol * np.abs(want).max()
        st.update()
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_a_step_without_dropout_keeps_its_route_and_results():
    wl, conn1, th1, conn2, th2, x, labels = _small()
    a = TrainStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau)
    b = TrainStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau, dropout=0.0)
    for st in (a, b):
        st.load(x.cuda(), labels.cuda())
        st.run()
    torch.cuda.synchronize()
    assert a.codes1 and b.codes1 and torch.equal(a.dth1, b.dth1) and torch.equal(a.loss, b.loss)


@pytest.mark.gpu
def test_distillation_with_dropout():
    wl, conn1, th1, conn2, th2, x, labels = _small()
    teacher = TeacherRecord(wl.batch, 3, 2.0)
    teacher.take(torch.randn(wl.batch, wl.classes, device="cuda"))
    st = DistillStep(Network(conn1, th1, conn2, th2, wl.w_in), wl.batch, wl.d, wl.thresholds, wl.classes, wl.tau, teacher,
                     dropout=0.5, seed=5)
    st.load(x.cuda(), labels.cuda())
    st.run()
    torch.cuda.synchronize()
    keep = bref.kept_values(0, wl.widths[0] * wl.batch, 5, 0, 0.5, 0).reshape(wl.widths[0], wl.batch)
    assert (st.y1.cpu().numpy()[~keep] == 0).all() and (st.y1.cpu().numpy()[keep] > 0).mean() > 0.9
    assert float(st.loss) > 0 and st.dth1.abs().sum() > 0


def test_refusals():
    lib, P = bl.load(), __import__("ctypes").c_void_p
    f = P(1 << 12)
    call = lambda X=f, dt=0, R=4, C=8, ldx=8, res=None, ldr=8, out=f, ldo=8, c=f, p=0.5, site=0: \
        lib.bitlogic_dropout(X, dt, R, C, ldx, res, ldr, out, ldo, c, p, site, None)   # noqa: E731
    assert call(dt=3) == -13 and call(dt=9) == -13 and call(dt=-1) == -13
    assert call(R=-1) == -2 and call(C=-1) == -2 and call(ldx=7) == -2 and call(ldo=7) == -2
    assert call(res=f, ldr=7) == -2 and call(R=1 << 21, C=1 << 20, ldx=1 << 20, ldo=1 << 20) == -2
    assert call(ldx=1 << 62) == -2 and call(R=1 << 62, C=1 << 62) == -2
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf"), 1.0 - 2.0 ** -34):
        assert call(p=p) == -11
    assert call(site=-1) == -11
    assert call(X=None) == -1 and call(out=None) == -1 and call(c=None) == -1
    assert call(X=P(4097)) == -4 and call(out=P(4098)) == -4 and call(c=P(4100)) == -4 and call(res=P(4097)) == -4
    assert call(X=P(4097), dt=1) == -4
    assert call(R=0, X=None, out=None, c=None) == 0 and call(C=0, X=None) == 0
    with pytest.raises(TypeError):
        bl.bitlogic_dropout(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2), None, 0.1)
    with pytest.raises(ValueError):
        bl.bitlogic_dropout(torch.zeros(2, 2), torch.zeros(2, 2), None, 0.1)
