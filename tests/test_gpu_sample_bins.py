"""Cuts by mass where the bins of powers that find them are off the most: many equal
powers, all rounded the same way, with a cut among single classes behind them."""
import numpy as np
import pytest
import torch

import paper_2602_07400_gb300 as bl

pytestmark = pytest.mark.gpu
LOG2E = np.float32(1.4426950408889634)


def _power(z):
    """e of logits about 0 at temperature 1, in the draw's roundings."""
    return torch.exp2(z * float(LOG2E))


def _unlucky(octave, mantissa, dev="cuda"):
    """A logit whose power lies `octave` octaves below 1 with the mantissa (24 bits)
    next to `mantissa`, of those that powers of logits have there."""
    at = np.float32((octave - np.log2(mantissa / 2.0 ** 23)) / float(LOG2E))
    z = torch.from_numpy((at.view(np.int32) + np.arange(-400, 400, dtype=np.int32)).astype(np.int32).view(np.float32)).to(dev).neg()
    off = (_power(z).view(torch.int32) - ((127 - octave) << 23) - (mantissa & 0x7FFFFF)).abs()
    assert int(off.min()) <= 8
    return float(z[off.argmin()])


def _rows(V, octave, mantissa, equal, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.full((V,), -70.0, device="cuda")
    a = _unlucky(octave, mantissa)
    z[0] = 0.0
    z[1:1 + equal] = a
    z[1 + equal:200 + equal] = a - torch.arange(1, 200, device="cuda") / 64.0 * float(np.log(2.0))
    return z[torch.randperm(V, generator=g, device="cuda")]


def _expected(z, p24):
    """floor and last for shares p24 / 2^24 of the whole weights, and the border itself."""
    w = (_power(z - z.max()).double() * 2.0 ** 40).round().long()
    zs, order = torch.sort(z, descending=True, stable=True)
    upto = w[order].cumsum(0)
    total = int(upto[-1])
    at = [int(torch.searchsorted(upto, max(1, (total * p) >> 24))) for p in p24]
    return zs[at], order[at].int()


@pytest.mark.parametrize("V,equal", [(5000, 4000), (40000, 30000), (131072, 60000), (131072, 100000)])
@pytest.mark.parametrize("octave", [3, 5, 8])
@pytest.mark.parametrize("mantissa", [0x800100, 0x8000FF, 0x800300, 0xFFFF00])
@pytest.mark.parametrize("rows", [6, 400])
def test_cuts_behind_many_equal_powers(V, equal, octave, mantissa, rows):
    z = _rows(V, octave, mantissa, equal, V + octave)
    w = (_power(z).double() * 2.0 ** 40).round().long()
    up = w.sort(descending=True).values.cumsum(0)
    total = int(up[-1])
    p24 = []
    for j in (equal + 1, equal + 2, equal + 6, equal + 60):
        border = -(-int(up[j - 1]) * 2 ** 24 // total)
        p24 += [border - 1, border, border + 1]
    p24 = [min(p, 2 ** 24 - 1) for p in p24]
    p24 = (p24 * (rows // len(p24) + 1))[:rows]
    x = z.expand(rows, V).contiguous()
    top_p = torch.tensor([p / 2.0 ** 24 for p in p24], device="cuda", dtype=torch.float32)
    floor, last = torch.empty(rows, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    bl.bitlogic_support_logits(x, floor, last, top_p=top_p)
    f, l = _expected(z, p24)
    torch.cuda.synchronize()
    assert torch.equal(floor, f) and torch.equal(last, l)
    # and the draw among them
    kept = torch.where((x > f[:, None]) | ((x == f[:, None]) & (torch.arange(V, device="cuda") <= l[:, None])), x, float("-inf"))
    a, b = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    for u in (0.0, 0.37, 0.99999994):
        bl.bitlogic_sample_logits(x, torch.full((rows,), u, device="cuda"), a, top_p=top_p)
        bl.bitlogic_sample_logits(kept, torch.full((rows,), u, device="cuda"), b)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
