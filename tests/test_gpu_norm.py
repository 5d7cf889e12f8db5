"""Norms to 8 bits and their gradient on the GPU against their 64-bit forms."""
import ctypes

import numpy as np
import pytest
import torch

import beside_ref as bref
import paper_2602_07400_gb300 as bl

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
E4M3 = torch.float8_e4m3fn


def _matrix(T, d, dtype, pad=0, shift=0, scale=1.0):
    buf = torch.empty(T * (d + pad) + shift + 16, dtype=dtype, device="cuda")
    x = buf[shift:shift + T * (d + pad)].view(T, d + pad)[:, :d]
    x.copy_(torch.randn(T, d, device="cuda") * scale)
    return x


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _y_error(d):
    """Relative error of y: h (one sum) and its squares to 2^-24 each, a sum of
    squares by runs of 8 to 32 a thread and a tree of 10, the root, the quotient
    and two products; all terms of the sum of one sign."""
    return (32 + 10 + 8) * 2.0 ** -24


def _check(out, scale, y, group, fixed=0.0):
    T, d = y.shape
    most = 127.0 if out.dtype == torch.uint8 else 448.0
    rel = _y_error(d) + 3 * 2.0 ** -24
    got, sc = out.float().double().cpu().numpy() if out.dtype == E4M3 else out.double().cpu().numpy() - 128.0, _np(scale)
    for i, (a, b) in enumerate(bref.groups(d, group)):
        part = y[:, a:b]
        big = np.abs(part).max(1)
        if fixed:
            s = np.full(T, fixed)
        else:
            s = sc[:, i]
            assert (np.abs(s - big / most) <= rel * big / most).all()
        with np.errstate(divide="ignore", invalid="ignore"):
            q = np.where(s[:, None] > 0, part / s[:, None], 0.0)
        q = np.clip(q, -most, most)
        # half a step of a whole number, of e4m3 (2^-4 of the value, 2^-10 of its least), and y's own error
        half = 0.5 if out.dtype == torch.uint8 else np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10)
        assert (np.abs(got[:, a:b] - q) <= half * (1 + 1e-9) + 3 * rel * np.abs(q)).all()


SHAPES = [(1, 1), (2, 7), (3, 8), (5, 16), (4, 100), (1, 255), (33, 256), (7, 1001), (300, 512), (3, 4096), (1, 8192), (2, 8200),
          (2, 16384), (3, 20001), (2, 32768), (0, 64),
          # more rows than run at once: rows come ahead of their turn
          (2500, 200), (2600, 1024), (400, 2048), (330, 8192), (170, 16384), (160, 20008)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", [torch.uint8, E4M3])
def test_norm_against_its_definition(T, d, dtype, form):
    for i, (group, residual, pad, shift, weight) in enumerate([(0, False, 0, 0, None), (128, True, 0, 0, "same"), (16, True, 8, 0, "f32"),
                                                               (256, True, 3, 1, "same"), (0, True, 5, 3, "f32"), (64, False, 16, 8, "same"),
                                                               (32, True, 0, 0, None)]):
        x = _matrix(T, d, dtype, pad, shift)
        r = _matrix(T, d, dtype, pad, shift) if residual else None
        w = None if weight is None else (1 + 0.3 * torch.randn(d, device="cuda")).to(dtype if weight == "same" else torch.float32)
        G = len(bref.groups(d, group))
        total = _matrix(T, d, dtype, pad, shift) if i % 2 else None
        out = torch.empty(T, d + (pad if i == 3 else 0), dtype=torch.uint8, device="cuda").fill_(3).view(form)[:, :d]
        scale = torch.full((T, G), 9.0, device="cuda")
        bl.bitlogic_norm_bytes(x, out, scale, weight=w, residual=r, total=total, group=group, eps=1e-5)
        torch.cuda.synchronize()
        if T == 0:
            continue
        h = _np(x) + (_np(r) if residual else 0.0)
        _check(out, scale, bref.norm(h, _np(w), 1e-5), group)
        if total is not None:
            eps = torch.finfo(dtype).eps / 2
            terms = np.abs(_np(x)) + (np.abs(_np(r)) if residual else 0)
            assert (np.abs(_np(total) - h) <= eps * np.abs(h) + 2.0 ** -24 * terms + torch.finfo(dtype).smallest_normal * eps * 2).all()
        # the sum in the place of either
        for at in (x, r) if residual else (x,):
            keep = at.clone()
            out2, scale2 = torch.empty_like(out), torch.empty_like(scale)
            bl.bitlogic_norm_bytes(x, out2, scale2, weight=w, residual=r, total=at, group=group, eps=1e-5)
            torch.cuda.synchronize()
            assert torch.equal(out2.contiguous().view(torch.uint8), out.contiguous().view(torch.uint8)) and torch.equal(scale2, scale)
            if total is not None:
                assert torch.equal(at, total)
            at.copy_(keep)


@pytest.mark.gpu
@pytest.mark.parametrize("form", [torch.uint8, E4M3])
@pytest.mark.parametrize("fixed", [0.02, 3.0 / 127, 1.0, 1e-3])
def test_a_fixed_scale_clips(form, fixed):
    x = _matrix(50, 300, torch.bfloat16)
    out = torch.empty(50, 300, dtype=form, device="cuda")
    bl.bitlogic_norm_bytes(x, out, fixed_scale=fixed, eps=1e-6)
    torch.cuda.synchronize()
    _check(out, None, bref.norm(_np(x), None, 1e-6), 0, np.float32(fixed))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_size_and_content(dtype):
    d = 1000
    x = _matrix(9, d, dtype)
    x[1] *= 1e30                 # squares past fp32
    x[2] *= 1e-30                # squares below it: eps alone
    x[3] = 0.0
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    x[6] = 3e38
    x[7] = 0.0
    x[7, 999] = 2.0
    for form in (torch.uint8, E4M3):
        for group in (0, 64):
            out, scale = torch.empty(9, d, dtype=form, device="cuda"), torch.empty(9, len(bref.groups(d, group)), device="cuda")
            bl.bitlogic_norm_bytes(x, out, scale, group=group, eps=1e-6)
            torch.cuda.synchronize()
            ok = [0, 1, 2, 3, 6, 7, 8]
            h = _np(x)[ok]
            with np.errstate(over="ignore"):
                _check(out[ok].view(torch.uint8).view(form), scale[ok], bref.norm(h, None, 1e-6), group)
            assert (scale[3] == 0).all() and (out[3].float() == (128 if form == torch.uint8 else 0)).all()
            assert torch.isnan(scale[4]).any() and torch.isnan(scale[5]).any()
            if form == torch.uint8:
                assert (out[4, :1] == 128).all()
            else:
                assert torch.isnan(out[4].float()).any()
            if group:
                assert (scale[7, :-1] == 0).all() and float(scale[7, -1]) > 0


BACK = [(1, 1), (2, 7), (3, 8), (5, 100), (1, 4096), (700, 256), (509, 1001), (33, 8192), (4, 8200), (5, 16384), (3, 20001), (2, 32768),
        (3000, 33), (2500, 200), (2600, 1024), (400, 2048), (700, 8192), (170, 16384), (160, 20008)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", BACK)
@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_against_its_formula(T, d, dtype):
    for res, pad, shift, weight in ((False, 0, 0, None), (True, 0, 0, "same"), (True, 8, 0, "f32"), (True, 3, 1, "same")):
        dy, h = _matrix(T, d, dtype, pad, shift), _matrix(T, d, dtype, pad, shift)
        r = _matrix(T, d, dtype, pad, shift) if res else None
        w = None if weight is None else (1 + 0.3 * torch.randn(d, device="cuda")).to(dtype if weight == "same" else torch.float32)
        dx, dw = _matrix(T, d, dtype, pad, shift), torch.full((d,), 5.0, device="cuda")
        ws = torch.full((bl.bitlogic_norm_backward_workspace(T, d),), 0xA5, dtype=torch.uint8, device="cuda")
        bl.bitlogic_norm_backward(dy, h, dx, weight=w, dweight=dw, residual_grad=r, workspace=ws, eps=1e-5)
        torch.cuda.synchronize()
        a, b = _np(dy), _np(h)
        gx, gw = bref.norm_backward(a, b, _np(w), 1e-5)
        want = gx + (_np(r) if res else 0.0)
        rr = 1.0 / np.sqrt((b * b).mean(1, keepdims=True) + 1e-5)
        g = np.abs(a if w is None else a * _np(w))
        rel = 60 * 2.0 ** -24    # as y, and the sum along h of the magnitudes of its terms
        terms = rr * (g + np.abs(b) * rr * rr * (g * np.abs(b)).mean(1, keepdims=True)) + (np.abs(_np(r)) if res else 0.0)
        eps = torch.finfo(dtype).eps / 2
        assert (np.abs(_np(dx) - want) <= eps * np.abs(want) + rel * terms + torch.finfo(dtype).smallest_normal * eps * 2).all()
        # a column's products: y's error each, and runs of T / 1024 rows and the partials
        depth = T // 304 + min(T, 1024) / 8 + 8
        assert (np.abs(_np(dw) - gw) <= ((60 + depth) * 2.0 ** -24) * np.abs(a * b * rr).sum(0) + 1e-30).all()
        first = dx.clone()
        for at in (dy, h, r) if res else (dy, h):      # in place, the gradient at x alone
            keep = at.clone()
            bl.bitlogic_norm_backward(dy, h, at, weight=w, residual_grad=r, eps=1e-5)
            torch.cuda.synchronize()
            assert torch.equal(at, first)
            at.copy_(keep)


@pytest.mark.gpu
def test_gradient_against_differences():
    # y in float64 by the formula; L = sum c y
    rng = np.random.default_rng(0)
    h, c, w = rng.normal(0, 1, (4, 37)), rng.normal(0, 1, (4, 37)), 1 + 0.2 * rng.normal(0, 1, 37)
    h, c, w = (v.astype(np.float32).astype(np.float64) for v in (h, c, w))
    f = lambda a, b: (c * bref.norm(a, b, 1e-5)).sum()   # noqa: E731
    t = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()   # noqa: E731
    dx, dw = torch.empty(4, 37, device="cuda"), torch.empty(37, device="cuda")
    ws = torch.empty(bl.bitlogic_norm_backward_workspace(4, 37), dtype=torch.uint8, device="cuda")
    bl.bitlogic_norm_backward(t(c), t(h), dx, weight=t(w), dweight=dw, workspace=ws, eps=1e-5)
    torch.cuda.synchronize()
    e = 1e-5    # the third derivative is of order 10: 1e-9, far below fp32
    for i in range(4):
        for j in range(37):
            d = np.zeros_like(h)
            d[i, j] = e
            assert abs((f(h + d, w) - f(h - d, w)) / (2 * e) - float(dx[i, j])) <= 3e-6
    for j in range(37):
        d = np.zeros_like(w)
        d[j] = e
        assert abs((f(h, w + d) - f(h, w - d)) / (2 * e) - float(dw[j])) <= 6e-6


@pytest.mark.gpu
def test_gradient_of_rows_whose_squares_pass_fp32_and_of_none():
    h, dy = torch.randn(3, 500, device="cuda"), torch.randn(3, 500, device="cuda")
    h[1] *= 1e25
    dx, dw = torch.empty_like(h), torch.full((500,), 5.0, device="cuda")
    ws = torch.empty(bl.bitlogic_norm_backward_workspace(3, 500), dtype=torch.uint8, device="cuda")
    bl.bitlogic_norm_backward(dy, h, dx, dweight=dw, workspace=ws)
    torch.cuda.synchronize()
    gx, gw = bref.norm_backward(_np(dy), _np(h), None, 1e-6)
    for i in range(3):
        assert np.abs(_np(dx)[i] - gx[i]).max() <= 1e-5 * np.abs(gx[i]).max()
    assert np.abs(_np(dw) - gw).max() <= 1e-5 * np.abs(gw).max()
    e = torch.empty(0, 500, device="cuda")
    bl.bitlogic_norm_backward(e, e, e.clone(), dweight=dw)
    torch.cuda.synchronize()
    assert (dw == 0).all()


@pytest.mark.gpu
def test_results_are_the_same_from_run_to_run_in_graphs_and_on_streams():
    T, d = 2000, 1000
    dy, h, w = _matrix(T, d, torch.bfloat16), _matrix(T, d, torch.bfloat16), torch.randn(d, device="cuda")
    def make():
        return (torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(d, device="cuda"),
                torch.empty(bl.bitlogic_norm_backward_workspace(T, d), dtype=torch.uint8, device="cuda"))
    def call(o, stream=None):
        bl.bitlogic_norm_backward(dy, h, o[0], weight=w, dweight=o[1], workspace=o[2], stream=stream)
    first, a, b = make(), make(), make()
    call(first)
    graphs = []
    for o in (a, b):
        g = torch.cuda.CUDAGraph()
        call(o)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(o)
        graphs.append(g)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for o in (a, b):
        o[0].zero_()
        o[1].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            graphs[0].replay()
        with torch.cuda.stream(s2):
            graphs[1].replay()
    torch.cuda.synchronize()
    for o in (a, b):
        assert torch.equal(o[0], first[0]) and torch.equal(o[1], first[1])
    c = make()
    s1.wait_stream(torch.cuda.current_stream())
    call(c, s1)
    s1.synchronize()
    assert torch.equal(c[0], first[0]) and torch.equal(c[1], first[1])


def test_refusals():
    lib, P, F = bl.load(), ctypes.c_void_p, ctypes.c_float
    f = P(1 << 12)

    def norm(X=f, dt=0, T=4, d=64, ldx=64, res=None, ldr=64, tot=None, ldt=64, w=None, wd=0, eps=1e-6, form=0, out=f, ldo=64, sc=f,
             group=0, fixed=0.0):
        return lib.bitlogic_norm_bytes(X, dt, T, d, ldx, res, ldr, tot, ldt, w, wd, F(eps), form, out, ldo, sc, group, F(fixed), None)

    assert norm(dt=3) == -13 and norm(form=2) == -13 and norm(form=-1) == -13 and norm(w=f, dt=1, wd=2) == -13
    assert norm(T=-1) == -2 and norm(d=0) == -2 and norm(d=32769, ldx=40000, ldo=40000) == -2 and norm(ldx=63) == -2 and norm(ldo=63) == -2
    assert norm(res=f, ldr=63) == -2 and norm(tot=f, ldt=63) == -2 and norm(ldx=1 << 60) == -2
    for group in (-1, 1, 8, 48, 512):
        assert norm(group=group) == -2
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert norm(eps=eps) == -11
    for fixed in (-1.0, float("nan"), float("inf"), 1e-45):
        assert norm(fixed=fixed) == -11
    assert norm(X=None) == -1 and norm(out=None) == -1 and norm(sc=None) == -1
    assert norm(X=P(4097)) == -4 and norm(sc=P(4097)) == -4 and norm(w=P(4097), dt=1, wd=1) == -4 and norm(tot=P(4097)) == -4
    assert norm(T=0, X=None, out=None, sc=None) == 0

    def back(dY=f, dt=0, T=4, d=64, ldy=64, H=f, ldh=64, w=None, wd=0, res=None, ldr=64, eps=1e-6, dX=f, ldx=64, dw=f, ws=f, n=1 << 20):
        return lib.bitlogic_norm_backward(dY, dt, T, d, ldy, H, ldh, w, wd, res, ldr, F(eps), dX, ldx, dw, ws, n, None)

    need = bl.bitlogic_norm_backward_workspace(4, 64)
    assert need == 4 * 64 * 4 and bl.bitlogic_norm_backward_workspace(1 << 20, 64) == 1024 * 64 * 4
    assert back(dt=3) == -13 and back(w=f, dt=1, wd=2) == -13
    assert back(T=-1) == -2 and back(d=0) == -2 and back(d=32769) == -2 and back(ldy=63) == -2 and back(ldh=63) == -2 and back(ldx=63) == -2
    assert back(res=f, ldr=63) == -2 and back(eps=0.0) == -11
    assert back(dY=None) == -1 and back(H=None) == -1 and back(dX=None) == -1 and back(ws=None) == -1
    assert back(ws=P(4104)) == -4 and back(dw=P(4097)) == -4 and back(H=P(4097)) == -4
    assert back(n=need - 1) == -5
    assert back(T=0, dw=None, ws=None) == 0
    with pytest.raises(TypeError):
        bl.bitlogic_norm_bytes(torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        bl.bitlogic_norm_bytes(torch.zeros(2, 2), torch.zeros(2, 2, dtype=torch.uint8))
