"""The operators on rows of logits called from two host threads at once, on
streams of their own, with rows that need different amounts of shared memory."""
import ctypes
import threading

import pytest
import torch

import paper_2602_07400_gb300 as bl

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Rows:
    """Rows of an operator of their own, called as bare C calls (which do not
    hold the interpreter's lock)."""

    def __init__(self, op, T, V):
        g = torch.Generator(device=DEV).manual_seed(V)
        self.stream = torch.cuda.Stream()
        x = torch.randn(T, V, generator=g, device=DEV)
        u, p = torch.rand(T, generator=g, device=DEV), torch.full((T,), 0.9, device=DEV)
        val, idx, lse = torch.zeros(T, 20, device=DEV), torch.zeros(T, 20, dtype=torch.int32, device=DEV), torch.zeros(T, device=DEV)
        bl.bitlogic_top_logits(x, val, idx, lse)
        row, loss, grad = torch.zeros(T, device=DEV), torch.zeros(1, device=DEV), torch.zeros_like(x)
        token = torch.zeros(T, dtype=torch.int32, device=DEV)
        self.outputs = dict(top=(val, idx, lse), distill=(row, loss, grad), sample=(token,))[op]
        self.keep = (x, u, p, val, idx, lse, row, loss, grad, token)
        lib, P = bl.load(), lambda t: ctypes.c_void_p(t.data_ptr())   # noqa: E731
        s = ctypes.c_void_p(self.stream.cuda_stream)
        self.call, self.args = {
            "top": (lib.bitlogic_top_logits, (P(x), 0, T, V, V, 20, 1.0, P(val), P(idx), P(lse), s)),
            "distill": (lib.bitlogic_distill_loss, (P(x), 0, T, V, V, P(val), P(idx), 20, P(lse), None, None, 1.0, 1.0, 0.0,
                                                    P(row), P(loss), P(grad), V, 1, 1.0, s)),
            "sample": (lib.bitlogic_sample_logits, (P(x), 0, T, V, V, P(u), None, None, P(p), None, P(token), None, s)),
        }[op]
        torch.cuda.synchronize()

    def loop(self, calls, start, failed):
        start.wait()
        for i in range(calls):
            st = self.call(*self.args)
            if st:
                failed.append(st)
            if i % 64 == 63:
                self.stream.synchronize()


# a kernel's rows in a warp, a block or a cluster each, of two lengths
@pytest.mark.parametrize("op,T,short,long,calls", [("distill", 400, 12000, 50000, 10000), ("distill", 4, 30000, 200000, 10000),
                                                   ("distill", 64, 600, 1000, 10000), ("top", 4, 30000, 131072, 10000),
                                                   ("sample", 4, 30000, 131072, 4000), ("sample", 200, 100000, 1000000, 100)])
def test_short_and_long_rows_at_once(op, T, short, long, calls):
    work = [Rows(op, T, V) for V in (short, long)]
    for w in work:
        assert w.call(*w.args) == 0
    torch.cuda.synchronize()
    want = [[t.clone() for t in w.outputs] for w in work]
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(2)
    threads = [threading.Thread(target=w.loop, args=(calls, start, failed)) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, f"{len(failed)} of {2 * calls} calls refused: {set(failed)}"
    for w, out in zip(work, want):
        assert all(torch.equal(a, b) for a, b in zip(w.outputs, out))
