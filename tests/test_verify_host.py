"""Draft verification and supports without a GPU: calls refused on the host."""
import ctypes

import pytest
import torch

import paper_2602_07400_gb300 as bl


def test_refusals():
    lib, P = bl.load(), ctypes.c_void_p
    f, g = P(1 << 12), P(1 << 13)

    def verify(t=f, dt=0, S=2, D=3, V=5000, ld=5000, temp=None, fl=None, la=None, first=f, tok=f, u=f, du=f, q=None, qt=0, qld=5000,
               lp=None, qtemp=None, qfl=None, qla=None, acc=f, nxt=f, out=None, ws=f, n=1 << 20):
        return lib.bitlogic_verify_drafts(t, dt, S, D, V, ld, temp, fl, la, first, tok, u, du, q, qt, qld, lp, qtemp, qfl, qla, acc, nxt,
                                          out, ws, n, None)

    need = bl.bitlogic_verify_drafts_workspace(2, 3, 5000)
    assert need > 0 and bl.bitlogic_verify_drafts_workspace(2, 3, 1024) == 0
    assert verify(S=-1) == -2 and verify(D=-1) == -2 and verify(S=0) == -2 and verify(V=0) == -2 and verify(ld=4999) == -2
    assert verify(V=(1 << 20) + 1, ld=1 << 21) == -2 and verify(S=(1 << 24) + 1) == -2
    assert verify(dt=4) == -13 and verify(dt=-1) == -13 and verify(q=f, lp=f, qt=4) == -13
    assert verify(q=f, lp=f, qld=4999) == -2 and verify(t=P(4097)) == -4 and verify(q=P(4097), lp=f) == -4
    for missing in ("t", "first", "tok", "u", "du", "acc", "nxt", "ws"):
        assert verify(**{missing: None}) == -1, missing
    assert verify(fl=f) == -1 and verify(la=f) == -1 and verify(q=f) == -1 and verify(lp=f) == -1
    assert verify(q=f, lp=f, qfl=f) == -1 and verify(qtemp=f) == -1 and verify(qfl=f, qla=f) == -1
    assert verify(ws=P((1 << 12) + 8)) == -4 and verify(n=need - 1) == -5
    assert verify(S=0, D=0, t=None, ws=None) == 0
    sup = lambda X=f, dt=0, T=2, V=50, ld=50, fl=f, la=g: lib.bitlogic_support_logits(X, dt, T, V, ld, None, None, None, None, fl, la, None)   # noqa: E731
    assert sup(fl=None) == -1 and sup(la=None) == -1 and sup(X=None) == -1 and sup(V=0) == -2 and sup(ld=49) == -2 and sup(dt=4) == -13
    assert sup(T=0, fl=None) == 0
    with pytest.raises(ValueError):
        bl.bitlogic_verify_drafts(torch.zeros(2, 5), None, torch.zeros(3, dtype=torch.int32), None, None, None, None)
