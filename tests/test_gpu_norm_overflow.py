"""The norm's gradient where sums over a row pass fp32 although its terms and the
gradient do not."""
import numpy as np
import pytest
import torch

import beside_ref as bref
import paper_2602_07400_gb300 as bl
from test_gpu_norm import _matrix, _np

pytestmark = pytest.mark.gpu


# rows, columns: by warps and by blocks, with rows ahead and without, off 16 bytes
SHAPES = [(3, 8), (4, 200), (5, 1001), (3, 4096), (2500, 200), (2600, 1024), (400, 2048), (330, 8192), (2, 20001)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h_size,dy_size", [(3e38, 1e20), (1e37, 1.0), (1e30, 1e12), (1e18, 1e25), (1e25, 1e-10), (3e38, 1e-3)])
def test_sums_past_fp32(T, d, dtype, h_size, dy_size):
    for i, (weight, res, pad, shift) in enumerate([(None, False, 0, 0), ("same", True, 8, 0), ("f32", False, 3, 1)]):
        dy, h = _matrix(T, d, dtype, pad, shift), _matrix(T, d, dtype, pad, shift)
        # all of one sign in some rows, so that nothing cancels; ordinary rows between them
        h.copy_((torch.rand(T, d, device="cuda") * 0.5 + 0.5) * h_size * torch.where(torch.rand(T, d, device="cuda") < 0.5, -1.0, 1.0))
        h[::3] = h[::3].abs()
        dy.copy_(torch.randn(T, d, device="cuda") * dy_size)
        dy[::3] = dy[::3].abs()
        h[1::3] = torch.randn_like(h[1::3])
        w = None if weight is None else (1 + 0.3 * torch.randn(d, device="cuda")).to(dtype if weight == "same" else torch.float32)
        r = _matrix(T, d, dtype, pad, shift) if res else None
        if res:
            r.mul_(dy_size / h_size)       # of dX's size
        dx, dw = _matrix(T, d, dtype, pad, shift), torch.full((d,), 5.0, device="cuda")
        ws = torch.full((bl.bitlogic_norm_backward_workspace(T, d),), 0xA5, dtype=torch.uint8, device="cuda")
        bl.bitlogic_norm_backward(dy, h, dx, weight=w, dweight=dw, residual_grad=r, workspace=ws, eps=1e-5)
        torch.cuda.synchronize()
        a, b = _np(dy), _np(h)
        gx, gw = bref.norm_backward(a, b, _np(w), 1e-5)
        want = gx + (_np(r) if res else 0.0)
        rr = 1.0 / np.sqrt((b * b).mean(1, keepdims=True) + 1e-5)
        g = np.abs(a if w is None else a * _np(w))
        # as for rows of any size (60 of 2^-24), and a root below fp32's normal numbers: 2^-149 of 2^-128.2, 2^-22
        # in each of its uses
        rel = (60 + 3 * 8) * 2.0 ** -24
        terms = rr * (g + np.abs(b) * rr * rr * (g * np.abs(b)).mean(1, keepdims=True)) + (np.abs(_np(r)) if res else 0.0)
        eps = torch.finfo(dtype).eps / 2
        assert (np.abs(_np(dx) - want) <= eps * np.abs(want) + rel * terms + torch.finfo(dtype).smallest_normal * eps * 2).all()
        depth = T // 304 + min(T, 1024) / 8 + 8
        assert (np.abs(_np(dw) - gw) <= ((84 + depth) * 2.0 ** -24) * np.abs(a * b * rr).sum(0) + 1e-30).all()
        first = dx.clone()
        for at in (dy, h, r) if res else (dy, h):
            keep = at.clone()
            bl.bitlogic_norm_backward(dy, h, at, weight=w, residual_grad=r, eps=1e-5)
            torch.cuda.synchronize()
            assert torch.equal(at, first)
            at.copy_(keep)


@pytest.mark.parametrize("d", [200, 1001, 8192])
def test_rows_with_nan_or_infinity_stay_their_own(d):
    T = 40
    h, dy = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda")
    h[3, 5], h[9, 7], dy[20, 1], dy[30, 0] = float("nan"), float("inf"), float("nan"), float("inf")
    bad = [3, 9, 20, 30]
    ok = [t for t in range(T) if t not in bad]
    dx = torch.empty_like(h)
    bl.bitlogic_norm_backward(dy, h, dx)
    torch.cuda.synchronize()
    assert torch.isfinite(dx[ok]).all()
    for t in bad:
        assert not torch.isfinite(dx[t]).all()
    gx, _ = bref.norm_backward(_np(dy)[ok], _np(h)[ok], None, 1e-6)
    assert np.abs(_np(dx)[ok] - gx).max() <= 1e-5 * np.abs(gx).max()
