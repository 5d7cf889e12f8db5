"""Whether a draft is accepted goes by its row and numbers alone, to the last bit
of u: not by how many rows the call has, nor by how a row is split over blocks."""
import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2602_07400_gb300 as bl
from test_gpu_verify import DTYPES

pytestmark = pytest.mark.gpu
N = 400                                    # numbers side by side around the border


def _accepted(target, first, token, u, lp, draft, **settings):
    S, D, V = first.numel() - 1, token.numel(), target.shape[1]
    acc, nxt = torch.full((S,), -7, dtype=torch.int32, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
    n = bl.bitlogic_verify_drafts_workspace(S, D, V)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") if n else None
    bl.bitlogic_verify_drafts(target, first, token, u, torch.zeros(S, device="cuda"), acc, nxt, ws, draft=draft, draft_logprob=lp,
                              **settings)
    torch.cuda.synchronize()
    return acc


def _exact(z, T, token):
    """The share of `token` in whole multiples of 2^-40 about the row's largest."""
    e, w = ref.weights(z, T)
    return e[token] / (sum(int(v) for v in w) * 2.0 ** -40)


@pytest.mark.parametrize("V,dtype,temp", [(5000, "f32", 1.0), (9000, "bf16", 0.7), (20011, "f16", 1.3), (50001, "f32", 1.0),
                                          (131072, "bf16", 1.0), (131072, "f32", 2.0), (600, "f32", 1.0)])
@pytest.mark.parametrize("kind", ["normal", "rising", "cut"])
def test_the_border_does_not_move(V, dtype, temp, kind):
    g = torch.Generator(device="cuda").manual_seed(V)
    for seed in range(3):
        z = torch.randn(V, generator=g, device="cuda") * 2
        if kind == "rising":               # the running largest rises all along the row
            z = z.sort().values
        x = z.to(DTYPES[dtype])
        # one of the likely, so that its p is some percent and u has digits to spare
        token = int(x.float().argmax())
        zh = x.double().cpu().numpy()
        settings = {}
        if kind == "cut":
            keep = torch.full((1,), min(1000, V - 1), dtype=torch.int32, device="cuda")
            f, l = torch.empty(1, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
            bl.bitlogic_support_logits(x[None].contiguous(), f, l, top_k=keep)
            settings = dict(floor=f, last=l)
            fl, la = float(f), int(l)
            zh = np.where((zh > fl) | ((zh == fl) & (np.arange(V) <= la)), zh, -np.inf)
        p = _exact(zh, np.float32(temp), token)
        lp = torch.full((N,), float(np.log(p / 0.75)), device="cuda")
        q = float(torch.exp(lp[0].double()))
        at = int(round(p / q * 2 ** 24)) + np.arange(N) - N // 2
        u = torch.from_numpy((at / 2.0 ** 24).astype(np.float32)).cuda()
        rows = x[None].expand(2 * N, V).contiguous()
        tok = torch.full((N,), token, dtype=torch.int32, device="cuda")
        one = lambda t, n: t.expand(n).contiguous()   # noqa: E731
        T = torch.full((2 * N,), temp, device="cuda")
        many = _accepted(rows, torch.arange(N + 1, dtype=torch.int32, device="cuda"), tok, u, lp, rows[:N], temperature=T,
                         **{k: one(v, 2 * N) for k, v in settings.items()})
        edge = int(many.sum())
        # accepted below the border alone
        assert many[:edge].all() and not many[edge:].any()
        # a step of u is 2^-24 / 0.75 of p: the power is right to 2^-22 (3 steps), q's
        # expf to 2 of its last places (3), the product, the sum and the quotient round
        assert abs(edge - N // 2) <= 16
        for n in (1, 3, 9, 40, 120):       # sequences of one draft, in every split of a row
            for i0 in sorted({max(0, min(N - n, edge - n // 2 + d)) for d in (-9, -3, 0, 2, 7)}):
                few = _accepted(rows[:2 * n], torch.arange(n + 1, dtype=torch.int32, device="cuda"), tok[i0:i0 + n], u[i0:i0 + n],
                                lp[i0:i0 + n], rows[:n], temperature=T[:2 * n], **{k: one(v, 2 * n) for k, v in settings.items()})
                assert torch.equal(few, many[i0:i0 + n]), (n, i0, edge)
        # drafts one after another in one sequence: up to the first past the border
        for i0 in (edge - 5, edge - 2):
            k = 8
            got = _accepted(rows[:k + 1], torch.tensor([0, k], dtype=torch.int32, device="cuda"), tok[:k], u[i0:i0 + k], lp[:k], rows[:k],
                            temperature=T[:k + 1], **{n: one(v, k + 1) for n, v in settings.items()})
            assert int(got) == edge - i0


@pytest.mark.parametrize("V,dtype", [(5000, "f32"), (131072, "bf16"), (30011, "f16")])
@pytest.mark.parametrize("k,others", [(20, 0), (100, 0), (140, 0), (100, 260)])
def test_many_drafts_at_the_border(V, dtype, k, others):
    # drafts of one row, those just accepted and the first just refused in any place:
    # rows in parts, by rounds, and whole rows among those of other sequences
    g = torch.Generator(device="cuda").manual_seed(V + k)
    x = (torch.randn(V, generator=g, device="cuda") * 2).to(DTYPES[dtype])
    token = int(x.float().argmax())
    p = _exact(x.double().cpu().numpy(), np.float32(1.0), token)
    lp = float(np.log(p / 0.75))
    q = float(torch.tensor(lp, dtype=torch.float32).double().exp())
    S, D = 1 + others, k + others
    rows = x[None].expand(S + D, V).contiguous()
    tok, lps = torch.full((D,), token, dtype=torch.int32, device="cuda"), torch.full((D,), lp, device="cuda")
    # the last u that is accepted, by sequences of one draft
    at = int(round(p / q * 2 ** 24)) + np.arange(N) - N // 2
    u = torch.from_numpy((at / 2.0 ** 24).astype(np.float32)).cuda()
    one = _accepted(x[None].expand(2 * N, V).contiguous(), torch.arange(N + 1, dtype=torch.int32, device="cuda"),
                    torch.full((N,), token, dtype=torch.int32, device="cuda"), u, torch.full((N,), lp, device="cuda"),
                    x[None].expand(N, V).contiguous())
    edge = int(one.sum())
    yes, no = float(u[edge - 1]), float(u[edge])
    first = torch.cat([torch.zeros(1), torch.arange(k, D + 1)]).to(torch.int32).cuda()
    for stop in (0, 1, 7, 15, 16, k // 2, k - 1, k):
        v = torch.full((D,), 0.3, device="cuda")
        v[:k:3] = yes
        v[max(0, stop - 2):stop] = yes
        if stop < k:
            v[stop] = no
            v[stop + 1:k:2] = yes
            v[stop + 2:k:4] = 0.999
        got = _accepted(rows, first, tok, v, lps, rows[:D])
        assert int(got[0]) == stop and (got[1:] == 1).all()
