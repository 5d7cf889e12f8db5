"""Refusals at the ends of the arguments' ranges: the argument checks of the C
calls, which come before any CUDA work."""
import pytest

from test_logits_host import distill


@pytest.mark.parametrize("T,V,ldg,incg", [((1 << 28) - 1, 1 << 20, 1 << 36, 1 << 40), ((1 << 28) - 1, 1 << 20, 1 << 40, 1 << 40),
                                          (1 << 24, 1 << 20, 1 << 39, 1 << 40)])
def test_gradient_strides_whose_extent_passes_64_bits(T, V, ldg, incg):
    assert distill(T=T, V=V, ld=V, ldg=ldg, incg=incg) == -2
