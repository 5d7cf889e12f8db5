"""Draft verification and row supports on the GPU against their 64-bit forms."""
import ctypes

import numpy as np
import pytest
import torch

import beside_ref as bref
import logits_ref as ref
import paper_2602_07400_gb300 as bl

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}


def _logits(rows, V, dtype, rng, pad=0, shift=0):
    """[rows, V] in the type, `pad` values between rows, `shift` values off the
    start of the memory."""
    z = rng.normal(0, 2, (rows, V))
    z[np.arange(rows), rng.integers(0, V, rows)] += 4
    t = torch.from_numpy(np.round(z * 50) + 3200 if dtype == "i32" else z).to(DTYPES[dtype])
    buf = torch.empty(rows * (V + pad) + shift + 8, dtype=DTYPES[dtype], device="cuda")
    x = buf[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
    x.copy_(t.cuda())
    return x


def _unit(dtype):
    return 50.0 if dtype == "i32" else 1.0


def _f32(a):
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def _i32(a):
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


class Batch:
    """Sequences with their drafts, drawn by bitlogic_sample_logits."""

    def __init__(self, counts, V, dtype, draft, seed, pad=0, shift=0, cut=None, spare=0):
        rng = np.random.default_rng(seed)
        self.V, self.S, self.D = V, len(counts), int(sum(counts)) + spare
        S, D = self.S, self.D
        self.first = _i32(np.concatenate([[0], np.cumsum(counts)]))
        self.target = _logits(S + D, V, dtype, rng, pad, shift)
        self.temperature = _f32((0.6 + rng.random(S + D)) * _unit(dtype))
        self.u, self.draw_u = _f32(rng.random(D)), _f32(rng.random(S))
        self.draft = self.lp = self.draft_temperature = None
        self.floor = self.last = self.draft_floor = self.draft_last = None
        used = int(sum(counts))
        at = np.arange(used) + np.repeat(np.arange(S), counts)
        self.token = _i32(rng.integers(0, V, D))
        if cut:
            self.floor, self.last = torch.empty(S + D, device="cuda"), torch.empty(S + D, dtype=torch.int32, device="cuda")
            bl.bitlogic_support_logits(self.target, self.floor, self.last, temperature=self.temperature,
                                       top_k=torch.full((S + D,), cut, dtype=torch.int32, device="cuda"))
        if draft is not None:
            near = ref.values(self.target)[at] / _unit(dtype) - (64.0 if dtype == "i32" else 0.0) if used else np.zeros((0, V))
            zd = np.zeros((D, V))
            zd[:used] = near + rng.normal(0, 0.7, near.shape)
            t = torch.from_numpy(np.round(zd * 50) + 3200 if draft == "i32" else zd).to(DTYPES[draft])
            buf = torch.empty(D, V + pad, dtype=DTYPES[draft], device="cuda")
            self.draft = buf[:, :V]
            self.draft.copy_(t.cuda())
            self.draft_temperature = _f32((0.6 + rng.random(D)) * _unit(draft))
            self.lp = torch.zeros(D, device="cuda")
            k = torch.full((D,), cut or 0, dtype=torch.int32, device="cuda")
            if D:
                bl.bitlogic_sample_logits(self.draft, _f32(rng.random(D)), self.token, self.lp,
                                          temperature=self.draft_temperature, top_k=k)
            if cut:
                self.draft_floor, self.draft_last = torch.empty(D, device="cuda"), torch.empty(D, dtype=torch.int32, device="cuda")
                bl.bitlogic_support_logits(self.draft, self.draft_floor, self.draft_last,
                                           temperature=self.draft_temperature, top_k=k)
        elif used:   # half of them the likeliest
            top = torch.from_numpy(np.nanargmax(ref.values(self.target)[at], 1).astype(np.int32)).cuda()
            pick = torch.from_numpy(rng.random(used) < 0.6).cuda()
            self.token[:used] = torch.where(pick, top, self.token[:used])
        self.accepted = torch.full((S,), -7, dtype=torch.int32, device="cuda")
        self.next = torch.full((S,), -7, dtype=torch.int32, device="cuda")
        self.logprob = torch.full((S,), 7.0, device="cuda")
        n = bl.bitlogic_verify_drafts_workspace(S, D, V)
        self.ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") if n else None

    def run(self, stream=None, ws=None):
        bl.bitlogic_verify_drafts(self.target, self.first, self.token, self.u, self.draw_u, self.accepted, self.next,
                                  ws if ws is not None else self.ws, logprob=self.logprob, draft=self.draft,
                                  draft_logprob=self.lp, temperature=self.temperature, floor=self.floor, last=self.last,
                                  draft_temperature=self.draft_temperature, draft_floor=self.draft_floor,
                                  draft_last=self.draft_last, stream=stream)
        return self

    def check(self, seqs=None):
        torch.cuda.synchronize()
        n = lambda t: None if t is None else t.cpu().numpy()   # noqa: E731
        z, zd = ref.values(self.target), ref.values(self.draft) if self.draft is not None else None
        first, token, T, fl, la = n(self.first), n(self.token), n(self.temperature), n(self.floor), n(self.last)
        lp, Td, fd, ld = n(self.lp), n(self.draft_temperature), n(self.draft_floor), n(self.draft_last)
        u, du, acc, nxt, out_lp = n(self.u), n(self.draw_u), n(self.accepted), n(self.next), n(self.logprob)
        for s in range(self.S) if seqs is None else seqs:
            a, b = int(first[s]), int(first[s + 1])
            rows = [(z[r], T[r], *((fl[r], la[r]) if fl is not None else (-np.inf, -1))) for r in range(a + s, b + s + 1)]
            drafts = None if zd is None else [(zd[j], Td[j], *((fd[j], ld[j]) if fd is not None else (-np.inf, -1))) for j in range(a, b)]
            ok = bref.verdicts(rows, token[a:b], None if lp is None else lp[a:b].astype(float), u[a:b], du[s], drafts)
            got = (int(acc[s]), int(nxt[s]))
            assert got in ok, (s, got, sorted(ok)[:5])
            p = bref.probs(*rows[got[0]])
            if p is None:
                assert got[1] == -1 and out_lp[s] == -np.inf
            else:
                # e by the power unit, to 2^-22; the weight in 2^-40; the sums exact
                want = p[got[1]]
                tol = 1e-6 + 2.0 ** -24 * abs(np.log(want)) + 2.0 ** -41 / (want / p.max())
                # the power's argument is rounded to 2^-24 of itself
                zr = rows[got[0]][0]
                m = zr[bref.kept_set(*rows[got[0]][:1], *rows[got[0]][2:])].max()
                if rows[got[0]][1] > 0 and np.isfinite(m):
                    tol += 2.0 ** -22 * (m - zr[got[1]]) / rows[got[0]][1]
                assert abs(out_lp[s] - np.log(want)) <= tol, (s, out_lp[s], np.log(want))


CASES = [
    # counts of drafts, classes, target, draft
    ([4], 32768, "bf16", "bf16"), ([1], 1, "f32", "f32"), ([0], 5, "f32", None), ([3, 0, 2], 2, "f16", "bf16"),
    ([5] * 9, 33, "bf16", "i32"), ([3] * 40, 100, "f32", "i32"), ([2, 3, 0, 1], 100, "i32", "f32"),
    ([8, 1, 0, 17], 1000, "f32", "f16"), ([2] * 5, 1024, "bf16", None), ([2] * 5, 1025, "bf16", "bf16"),
    ([1, 9, 0, 4, 12], 5000, "f16", "f32"), ([3] * 20, 7777, "f32", "bf16"), ([2, 0, 7], 50001, "f32", "f32"),
    ([3, 1], 131072, "bf16", None), ([1, 2], 300001, "bf16", "f16"), ([0, 0], 40000, "i32", None),
    ([1] * 200, 2049, "bf16", "i32"),
    # rows longer than the blocks of a sequence hold
    ([2], 1 << 20, "f32", "f32"), ([1, 0, 1], 700001, "bf16", "f32"), ([1, 1], 900000, "i32", "bf16"),
]


@pytest.mark.parametrize("counts,V,dtype,draft", CASES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_verify_against_its_definition(counts, V, dtype, draft, pad, shift):
    for seed in range(3):
        Batch(counts, V, dtype, draft, seed, pad, shift).run().check()
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("counts,V,dtype,draft", [([3] * 400, 1100, "bf16", "bf16"), ([0, 7, 1, 12, 3] * 90, 2050, "f32", "i32"),
                                                  ([2] * 700, 1500, "f16", None)])
def test_verify_of_more_rows_than_run_at_once(counts, V, dtype, draft):
    # rows behind a refused draft may be left unread
    b = Batch(counts, V, dtype, draft, 1)
    for _ in range(3):
        b.ws.fill_(0xFF)
        b.run().check(range(0, len(counts), 7))
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V", [60, 3000, 33000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_draft_with_nan_and_a_refusal_that_leaves_nothing(V, dtype):
    b = Batch([1] * 40, V, dtype, dtype, 31)
    b.u.fill_(0.99)                      # refuse where q is not far below p
    b.draft[::2, 1::3] = float("nan")    # NaN is never drawn: q is 0 there
    b.run().check()
    # q as p, but for a draw's logarithm that claims more: what is left of p - q is
    # nothing, and the next class is drawn from p
    b = Batch([1] * 40, V, dtype, dtype, 32)
    at = 2 * torch.arange(40, device="cuda")
    b.draft = b.target[at].contiguous()
    b.draft_temperature = b.temperature[at].contiguous()
    b.lp.fill_(5.0)
    b.u.fill_(0.999)
    b.run()
    token, lp = torch.empty(40, dtype=torch.int32, device="cuda"), torch.empty(40, device="cuda")
    bl.bitlogic_sample_logits(b.draft, b.draw_u, token, lp, temperature=b.draft_temperature)
    torch.cuda.synchronize()
    assert (b.accepted == 0).all() and torch.equal(b.next, token) and torch.equal(b.logprob, lp)


@pytest.mark.parametrize("counts,V,dtype,draft", [([3, 0, 2, 5], 33, "bf16", "bf16"), ([4] * 12, 500, "f32", "i32"),
                                                  ([3, 7, 1], 5000, "bf16", "bf16"), ([2, 3], 50001, "f32", None),
                                                  ([2] * 30, 4099, "f16", "f32"), ([1, 1], 600000, "f32", "f32")])
@pytest.mark.parametrize("cut", [1, 5, 40])
def test_verify_among_the_classes_kept(counts, V, dtype, draft, cut):
    # bf16 and counts have many equal logits at the cut
    Batch(counts, V, dtype, draft, 11, 8, 0, cut=min(cut, V - 1)).run().check()
    Batch(counts, V, dtype, draft, 12, 3, 1, cut=min(cut, V - 1)).run().check()


@pytest.mark.parametrize("V,dtype", [(10, "f32"), (100, "i32"), (1000, "bf16"), (3000, "f16"), (50001, "f32"), (131072, "bf16")])
@pytest.mark.parametrize("cut", [None, 20])
def test_without_drafts_the_next_class_is_a_draw(V, dtype, cut):
    b = Batch([0] * 37, V, dtype, None, 5, cut=cut if cut is None else min(cut, V - 1)).run()
    token, lp = torch.empty(37, dtype=torch.int32, device="cuda"), torch.empty(37, device="cuda")
    k = torch.full((37,), min(cut, V - 1), dtype=torch.int32, device="cuda") if cut else None
    bl.bitlogic_sample_logits(b.target, b.draw_u, token, lp, temperature=b.temperature, top_k=k)
    torch.cuda.synchronize()
    assert torch.equal(b.accepted, torch.zeros_like(b.accepted))
    assert torch.equal(b.next, token)
    assert torch.equal(b.logprob, lp)


def test_the_draw_does_not_depend_on_the_batch():
    big = Batch([3] * 200, 9000, "bf16", "bf16", 3).run()
    torch.cuda.synchronize()
    for s in (0, 17, 199):
        rows, drafts = slice(4 * s, 4 * s + 4), slice(3 * s, 3 * s + 3)
        acc, nxt = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(bl.bitlogic_verify_drafts_workspace(1, 3, 9000), dtype=torch.uint8, device="cuda")
        bl.bitlogic_verify_drafts(big.target[rows], _i32([0, 3]), big.token[drafts], big.u[drafts], big.draw_u[s:s + 1], acc,
                                  nxt, ws, draft=big.draft[drafts], draft_logprob=big.lp[drafts],
                                  temperature=big.temperature[rows], draft_temperature=big.draft_temperature[drafts])
        torch.cuda.synchronize()
        assert int(acc) == int(big.accepted[s]) and int(nxt) == int(big.next[s])


@pytest.mark.parametrize("V", [8, 1500])
def test_what_goes_out_is_distributed_as_the_target(V):
    # the first class out of each of N sequences of one draft
    N = 20000
    rng = np.random.default_rng(0)
    z, zd = rng.normal(0, 1, V), rng.normal(0, 1, V)
    if V > 8:
        z[8:] -= 9
        zd[8:] -= 9
    target, draft = _f32(np.tile(z, (2 * N, 1))), _f32(np.tile(zd, (N, 1)))
    token, lp = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")
    bl.bitlogic_sample_logits(draft, torch.rand(N, device="cuda"), token, lp)
    acc, nxt = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
    n = bl.bitlogic_verify_drafts_workspace(N, N, V)
    bl.bitlogic_verify_drafts(target, torch.arange(N + 1, dtype=torch.int32, device="cuda"), token, torch.rand(N, device="cuda"),
                              torch.rand(N, device="cuda"), acc, nxt, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None,
                              draft=draft, draft_logprob=lp)
    out = torch.where(acc > 0, token, nxt).cpu().numpy()
    p = bref.probs(np.float32(z).astype(float))
    got = np.bincount(out, minlength=V) / N
    sd = np.sqrt(p * (1 - p) / N)
    assert (np.abs(got - p) <= 5.5 * sd + 1.0 / N).all()      # 5.5 deviations: 4e-8 a class
    # and so many are accepted as the two have in common
    share = np.minimum(p, bref.probs(np.float32(zd).astype(float))).sum()
    assert abs(float(acc.float().mean()) - share) <= 5.5 * np.sqrt(share * (1 - share) / N)


@pytest.mark.parametrize("V", [50, 6000])
def test_drafts_of_the_target_itself_are_accepted(V):
    b = Batch([4] * 50, V, "f32", "f32", 2)
    at = torch.arange(200, device="cuda") + torch.arange(50, device="cuda").repeat_interleave(4)
    b.draft = b.target[at].contiguous()
    b.draft_temperature = b.temperature[at].contiguous()
    bl.bitlogic_sample_logits(b.draft, b.u, b.token, b.lp, temperature=b.draft_temperature)
    b.u = torch.rand(200, device="cuda") * 0.99999    # u q < p as p and q agree to 1e-6
    b.run()
    torch.cuda.synchronize()
    assert (b.accepted == 4).all()


@pytest.mark.parametrize("V", [6, 200, 3001, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_that_are_masked_infinite_or_greedy(V, dtype):
    b = Batch([2] * 12, V, dtype, dtype, 4)
    low = torch.finfo(DTYPES[dtype]).min
    inf = float("inf")
    t, d = b.target, b.draft
    t[0] = -inf                          # nothing is left: the draft is refused, no class
    t[3, V // 2:] = low                  # the type's lowest is a logit like any
    t[6] = low
    t[9, ::2] = float("nan")             # NaN is never drawn
    t[12, V - 1] = inf                   # the first of +inf takes it all
    t[12, V // 3] = inf
    b.temperature[15] = 0.0              # greedy, with ties
    t[15] = 0.0
    b.temperature[18] = -1.0
    d[12] = -inf                         # a draft row of nothing (with a token all the same)
    b.temperature[21:24] = 1e30          # all but equal
    b.draft_temperature[14] = 0.0        # q all on its token
    d[16, V // 2] = inf                  # likewise
    t[30, : V - 1] = -inf                # one class is left
    b.lp[18] = -inf                      # a draft that its draft does not draw
    b.u[20] = float("nan")
    b.u[21] = 1.0
    b.draw_u[9] = 1.0
    b.draw_u[10] = float("nan")
    b.u = torch.nan_to_num(b.u, nan=0.0).clamp(max=0.99999994)
    b.run()
    b.draw_u = torch.nan_to_num(b.draw_u, nan=0.0).clamp(max=0.99999994)
    b.check()
    assert bl.bitlogic_device_error() == 0
    assert int(b.accepted[0]) == 0 and int(b.next[0]) == -1


@pytest.mark.parametrize("V", [40, 1200, 20011, 60000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_nan_wherever_it_stands(V, dtype, shift):
    # at the ends of rows, in runs as long as what a thread takes at a time, alone
    nan = float("nan")
    b = Batch([1] * 16, V, dtype, dtype, 77, 3 * shift, shift)
    b.u.fill_(0.97)                      # refused mostly: the draw goes over both rows
    for x, rows in ((b.target, 2), (b.draft, 1)):
        for s in range(16):
            r = rows * s
            if s % 8 == 0:
                x[r, 0] = nan
            elif s % 8 == 1:
                x[r, V - 1] = nan
            elif s % 8 == 2:
                x[r, V // 4: 3 * V // 4] = nan
            elif s % 8 == 3:
                x[r, : V // 2] = nan
                x[r, V // 2: V // 2 + 5] = -float("inf")
            elif s % 8 == 4:
                x[r, V // 3] = nan
            elif s % 8 == 5:
                x[r, 3:] = nan
            elif s % 8 == 6:
                x[r, V // 2:] = nan
    # tokens that may be drawn
    ok = b.draft.float()
    b.token = torch.where(torch.isnan(ok), torch.full_like(ok, -1e30), ok).argmax(1).to(torch.int32)
    b.lp.fill_(-0.1)
    b.run().check()
    assert bl.bitlogic_device_error() == 0


def test_u_and_draw_u_outside_their_range_are_clamped():
    for V in (40, 4000):
        b = Batch([1] * 8, V, "f32", "f32", 6)
        b.u[:] = torch.tensor([float("nan"), -3.0, 0.0, 1.0, 2.0, float("inf"), 0.5, 0.99999994], device="cuda")
        b.draw_u[:] = b.u.flip(0)
        b.run()
        torch.cuda.synchronize()
        got = b.accepted.clone(), b.next.clone()
        b.u = torch.nan_to_num(b.u, nan=0.0).clamp(0.0, 0.99999994)
        b.draw_u = torch.nan_to_num(b.draw_u, nan=0.0).clamp(0.0, 0.99999994)
        b.run().check()
        assert torch.equal(got[0], b.accepted) and torch.equal(got[1], b.next)


@pytest.mark.parametrize("V", [77, 2500])
def test_rows_behind_the_last_sequence_are_not_read(V):
    b = Batch([2, 0, 3], V, "bf16", "bf16", 8, spare=5)
    used = 5
    b.target[used + 3:] = float("nan")
    b.draft[used:] = float("nan")
    b.token[used:] = 1 << 30
    b.run().check()
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V", [77, 2500])
def test_bad_places_and_tokens_raise_the_flag(V):
    b = Batch([2, 2, 2], V, "f32", "f32", 9)
    for bad in ([0, 2, 1, 6], [-1, 2, 4, 6], [0, 2, 9, 6], [0, 2, 4, 7]):
        b.first = _i32(bad)
        b.run()
        torch.cuda.synchronize()
        assert bl.bitlogic_device_error() == -8
        hurt = [s for s in range(3) if not (0 <= bad[s] <= bad[s + 1] <= min(6, bad[3]))]
        for s in hurt:
            assert int(b.accepted[s]) == 0 and int(b.next[s]) == -1 and float(b.logprob[s]) == -np.inf
    b.first = _i32([0, 2, 4, 6])
    for bad in (-1, V, -(1 << 31)):
        b.token[2] = bad
        b.run().check()                  # refused, the next class from p
        assert int(b.accepted[1]) == 0
        assert bl.bitlogic_device_error() == -8
    b.token[2] = 0
    b.run().check()
    assert bl.bitlogic_device_error() == 0


def test_no_sequences_and_no_drafts():
    e = lambda n, t=torch.float32: torch.empty(n, dtype=t, device="cuda")   # noqa: E731
    bl.bitlogic_verify_drafts(e((0, 50)), torch.zeros(1, dtype=torch.int32, device="cuda"), e(0, torch.int32), e(0), e(0),
                              e(0, torch.int32), e(0, torch.int32))
    Batch([0, 0, 0], 5000, "bf16", "bf16", 1).run().check()
    assert bl.bitlogic_device_error() == 0


@pytest.mark.parametrize("V", [77, 2500])
def test_settings_of_drafts_that_are_none_are_not_read(V):
    """A caller of the C entry keeps its buffers' addresses when a step has no drafts."""
    b = Batch([0, 0, 0], V, "f32", None, 3)
    b.run().check()
    want = b.next.clone()
    b.next.fill_(-9)
    ws = torch.empty(bl.bitlogic_verify_drafts_workspace(3, 0, V) or 16, dtype=torch.uint8, device="cuda")
    kept, last = _f32(np.zeros(4)), _i32(np.zeros(4))
    p = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())   # noqa: E731
    st = bl.load().bitlogic_verify_drafts(p(b.target), 0, 3, 0, V, b.target.stride(0), p(b.temperature), None, None, p(b.first), None, None,
                                          p(b.draw_u), None, 0, V, p(kept), p(kept), p(kept), p(last), p(b.accepted), p(b.next), None,
                                          p(ws), ws.numel(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(b.next, want) and b.accepted.tolist() == [0, 0, 0]


def test_graphs_streams_and_workspaces():
    a, b = Batch([3] * 20, 4000, "bf16", "bf16", 20), Batch([2] * 30, 7000, "bf16", "i32", 21)
    for x in (a, b):
        x.run().check()
    want = [(x.accepted.clone(), x.next.clone()) for x in (a, b)]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for x in (a, b):
        x.accepted.fill_(-9)
        x.next.fill_(-9)
    torch.cuda.synchronize()
    for _ in range(5):                   # both at once
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for x, (acc, nxt) in zip((a, b), want):
        assert torch.equal(x.accepted, acc) and torch.equal(x.next, nxt)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    a.u.copy_(torch.rand_like(a.u))
    st.wait_stream(torch.cuda.current_stream())
    a.run(stream=st)
    st.synchronize()
    a.check()


# ---------------------------------------------------------------- supports --

def _support(x, **settings):
    T = x.shape[0]
    floor, last = torch.full((T,), 7.0, device="cuda"), torch.full((T,), -7, dtype=torch.int32, device="cuda")
    bl.bitlogic_support_logits(x, floor, last, **settings)
    torch.cuda.synchronize()
    return floor, last


def _settings(rng, T, unit, V):
    return dict(temperature=_f32(np.where(rng.random(T) < 0.1, 0.0, 0.5 + rng.random(T)) * unit),
                top_k=_i32(rng.choice([0, 0, 1, 3, 50, V - 1, V, V + 5], T)),
                top_p=_f32(rng.choice([1.0, 1.0, 0.3, 0.9, 0.99, 0.0], T)), min_p=_f32(rng.choice([0.0, 0.0, 0.05, 1.0], T)))


SUPPORTS = [(200, 1, "f32"), (200, 7, "bf16"), (60, 100, "i32"), (60, 300, "f16"), (40, 1000, "bf16"), (30, 1025, "f32"),
            (30, 5000, "bf16"), (8, 50001, "f32"), (300, 3001, "f16"), (4, 131072, "bf16"), (160, 40000, "bf16")]


@pytest.mark.parametrize("T,V,dtype", SUPPORTS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 3)])
def test_support_against_its_definition(T, V, dtype, pad, shift):
    rng = np.random.default_rng(V + pad)
    x = _logits(T, V, dtype, rng, pad, shift)
    s = _settings(rng, T, _unit(dtype), V)
    floor, last = _support(x, **s)
    z, skipped, by_mass = ref.values(x), 0, 0
    h = {n: t.cpu().numpy() for n, t in s.items()}
    for t in range(0, T, max(1, T // 30)):
        f, l, near = bref.support(z[t], h["temperature"][t], int(h["top_k"][t]), h["top_p"][t], h["min_p"][t])
        by_mass += 0 < h["top_p"][t] < 1
        if near:
            skipped += 1
            continue
        assert (float(floor[t]), int(last[t])) == (f, l), (t, float(floor[t]), int(last[t]), f, l, {n: v[t] for n, v in h.items()})
    assert skipped <= by_mass    # a mass cut among many small weights lies near one of them


@pytest.mark.parametrize("T,V,dtype", SUPPORTS)
def test_draws_lie_in_the_support_and_need_no_more(T, V, dtype):
    # a draw under the settings is the draw without them of the kept logits
    rng = np.random.default_rng(V)
    x = _logits(T, V, dtype, rng)
    s = _settings(rng, T, _unit(dtype), V)
    floor, last = _support(x, **s)
    v = torch.arange(V, device="cuda")[None, :]
    xf = x.float()
    keep = (xf > floor[:, None]) | ((xf == floor[:, None]) & (v <= last[:, None]))
    masked = torch.where(keep, xf, float("-inf"))
    a, b = (torch.empty(T, dtype=torch.int32, device="cuda") for _ in range(2))
    for seed in range(4):
        u = _f32(np.random.default_rng(seed).random(T))
        bl.bitlogic_sample_logits(x, u, a, **s)
        bl.bitlogic_sample_logits(masked, u, b, temperature=s["temperature"])
        torch.cuda.synchronize()
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", [5, 900, 4000, 60000])
@pytest.mark.parametrize("T", [6, 400])
def test_supports_of_masked_equal_and_infinite_rows(T, V):
    x = torch.zeros(T, V, device="cuda")
    inf = float("inf")
    x[0] = -inf
    x[1, V // 2:] = -inf
    x[2] = float("nan")
    x[3, V - 1] = inf
    x[3, V // 2] = inf
    x[4] = torch.finfo(torch.float32).min
    x[5, ::2] = float("nan")
    z = ref.values(x)
    for s in (dict(top_k=3), dict(top_k=V), dict(top_p=0.5), dict(min_p=0.2), dict(top_k=max(2, V // 2 + 1), min_p=0.5), dict(),
              dict(top_p=0.9, min_p=1.0), dict(top_k=min(2000, V - 1), top_p=0.7)):
        dev = {n: (_i32 if n == "top_k" else _f32)([v] * T) for n, v in s.items()}
        floor, last = _support(x, **dev)
        for t in range(6):
            f, l, near = bref.support(z[t], 1.0, s.get("top_k", 0), np.float32(s.get("top_p", 1.0)), np.float32(s.get("min_p", 0.0)))
            # equal logits: sums are whole multiples of one weight, a border is exact
            assert (float(floor[t]), int(last[t])) == (f, l), (s, t, float(floor[t]), int(last[t]), f, l)
    floor, last = _support(x, temperature=torch.zeros(T, device="cuda"))
    assert [int(v) for v in last[:6]] == [-1, 0, -1, V // 2, 0, 1 if V > 1 else -1]
    assert float(floor[3]) == inf
