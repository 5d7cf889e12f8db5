"""Refusals at the ends of the arguments' ranges: the argument checks of the C
calls, which come before any CUDA work."""
import pytest

from test_logits_host import distill, top


@pytest.mark.parametrize("T,V,ldg,incg", [((1 << 28) - 1, 1 << 20, 1 << 36, 1 << 40), ((1 << 28) - 1, 1 << 20, 1 << 40, 1 << 40),
                                          (1 << 24, 1 << 20, 1 << 39, 1 << 40)])
def test_gradient_strides_whose_extent_passes_64_bits(T, V, ldg, incg):
    assert distill(T=T, V=V, ld=V, ldg=ldg, incg=incg) == -2


def test_temperatures_that_fp32_does_not_hold():
    for tau in (1e-45, 1e-42, 4.2e-39):   # log2(e) / tau is not finite
        assert top(tau=tau) == -11 and distill(tau=tau) == -11
    assert top(T=0, tau=4.4e-39) == 0
    # kd_weight tau^2 is not finite, or 0 though the weight is not
    assert distill(tau=1e20) == -11 and distill(tau=1e15, kd=1e10) == -11
    assert distill(tau=1e-25) == -11 and distill(tau=1e-10, kd=1e-30) == -11
