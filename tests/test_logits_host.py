"""Refusals of the operators on rows of logits: argument checks of the C calls
and of the binding, which come before any CUDA work."""
import ctypes

import pytest
import torch

import paper_2602_07400_gb300 as bl

P = ctypes.c_void_p
FAKE = P(64)
INF, NAN = float("inf"), float("nan")


def top(X=FAKE, dtype=0, T=4, V=10, ld=10, K=3, tau=1.0, val=FAKE, idx=FAKE, lse=None):
    return bl.load().bitlogic_top_logits(X, dtype, T, V, ld, K, tau, val, idx, lse, None)


def distill(Z=FAKE, dtype=0, T=4, V=10, ld=10, val=FAKE, idx=FAKE, K=3, tau=1.0, kd=1.0, ce=0.0, row=FAKE, loss=FAKE,
            dZ=FAKE, ldg=10, incg=1, scale=1.0):
    return bl.load().bitlogic_distill_loss(Z, dtype, T, V, ld, val, idx, K, None, None, None, tau, kd, ce, row, loss,
                                           dZ, ldg, incg, scale, None)


def sample(X=FAKE, dtype=0, T=4, V=10, ld=10, u=FAKE, token=FAKE):
    return bl.load().bitlogic_sample_logits(X, dtype, T, V, ld, u, None, None, None, None, token, None, None)


@pytest.mark.parametrize("call,matrix", [(top, "X"), (distill, "Z"), (sample, "X")])
def test_matrix_of_logits(call, matrix):
    assert call(**{matrix: None}) == -1
    assert call(dtype=4) == -13 and call(dtype=-1) == -13
    assert call(T=-1) == -2
    assert call(V=0) == -2 and call(V=-5) == -2
    assert call(V=(1 << 20) + 1, ld=1 << 21) == -2
    assert call(ld=9) == -2
    assert call(**{matrix: P(66)}) == -4
    assert call(**{matrix: P(65), "dtype": 1}) == -4


def test_top_arguments():
    assert top(K=0) == -2 and top(K=11) == -2 and top(V=1000, ld=1000, K=257) == -2
    assert top(tau=0.0) == -11 and top(tau=-1.0) == -11 and top(tau=NAN) == -11 and top(tau=INF) == -11
    assert top(val=None) == -1 and top(idx=None) == -1
    assert top(T=0) == 0 and top(T=0, X=None, val=None, idx=None) == 0


def test_distill_arguments():
    assert distill(dtype=3) == -13
    assert distill(K=0) == -2 and distill(K=257) == -2
    for bad in (0.0, -1.0, NAN, INF):
        assert distill(tau=bad) == -11
    for bad in (NAN, INF, -INF):
        assert distill(kd=bad) == -11 and distill(ce=bad) == -11 and distill(scale=bad) == -11
    assert distill(val=None) == -1 and distill(idx=None) == -1 and distill(row=None) == -1 and distill(loss=None) == -1
    # gradient rows that overlap, or strides that are none
    assert distill(ldg=9) == -2 and distill(ldg=0) == -2 and distill(incg=0) == -2 and distill(ldg=3, incg=1) == -2
    assert distill(ldg=1, incg=3) == -2
    assert distill(dZ=P(66)) == -4


def test_sample_arguments():
    assert sample(u=None) == -1 and sample(token=None) == -1
    assert sample(T=0) == 0 and sample(T=0, X=None, u=None, token=None) == 0


def test_status_text():
    assert bl.bitlogic_status_string(-13) != "unknown status"


def test_binding_refuses_what_is_no_matrix_of_logits():
    x = torch.zeros(3, 8)
    out = torch.zeros(3, 2)
    for bad, error in [([1.0], TypeError), (x.double(), TypeError), (x.to(torch.uint8), TypeError), (x, ValueError)]:
        with pytest.raises(error):
            bl.bitlogic_top_logits(bad, out, out.int())
        with pytest.raises(error):
            bl.bitlogic_distill_loss(bad, out, out.int(), out[:, 0], out[0, :1])
        with pytest.raises(error):
            bl.bitlogic_sample_logits(bad, out[:, 0], out.int()[:, 0])


@pytest.mark.gpu
def test_binding_refusals_on_the_gpu():
    x = torch.zeros(4, 10, device="cuda")
    val, idx = torch.zeros(4, 3, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    row, loss, tok = torch.zeros(4, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="adjacent"):
        bl.bitlogic_top_logits(x.t(), val, idx)
    with pytest.raises(ValueError, match="dimensions"):
        bl.bitlogic_sample_logits(x[0], row, tok)
    with pytest.raises(TypeError):
        bl.bitlogic_top_logits(x, val, idx.long())
    with pytest.raises(ValueError):
        bl.bitlogic_top_logits(x, val, idx[:, :2])
    with pytest.raises(bl.BitLogicError):
        bl.bitlogic_top_logits(x, val[:, :0].contiguous(), idx[:, :0].contiguous())
    with pytest.raises(TypeError):
        bl.bitlogic_distill_loss(x, val, idx, row, loss, torch.zeros(4, 10, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        bl.bitlogic_distill_loss(x, val, idx, row, loss, torch.zeros(4, 11, device="cuda"))
    with pytest.raises(bl.BitLogicError) as e:   # rows of the gradient over one another
        bl.bitlogic_distill_loss(x, val, idx, row, loss, torch.zeros(10, device="cuda").expand(4, 10))
    assert e.value.code == -2
    with pytest.raises(bl.BitLogicError) as e:
        bl.bitlogic_distill_loss(x.to(torch.int32), val, idx, row, loss)
    assert e.value.code == -13
    with pytest.raises(ValueError):
        bl.bitlogic_distill_loss(x, val, idx, row, loss, labels=tok[:3])
    with pytest.raises(TypeError):
        bl.bitlogic_sample_logits(x, row, tok, top_k=row)
    with pytest.raises(ValueError):
        bl.bitlogic_sample_logits(x, row[:3], tok)
