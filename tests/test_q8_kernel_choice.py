"""Which kernel decodes over the 8-bit cache (no GPU): the rule's borders, and that the cases of the GPU tests that are made for
one kernel are its."""
import pytest

import q8_kernels
import q8_rule
from paper_2607_08186_gb300 import inputs


@pytest.mark.parametrize("c", q8_kernels.CHANGE + q8_kernels.WAVE)
def test_cases_for_the_tensor_cores(c):
    B, n, Hq, Hkv, Dh, P, T, L = c
    for mode, w in ((inputs.CROSS, 0), (inputs.WITHIN, 0)) + (((inputs.LOCAL, 150),) if n * Hq // Hkv > 16 else ()):
        assert q8_rule.tensor_cores(B, n, Hq, Hkv, Dh, P, L, mode, w)


@pytest.mark.parametrize("c", q8_kernels.SIZES)
def test_cases_of_sizes(c):
    kernel, n, Hq, Hkv, Dh, P, T, L = c
    assert q8_rule.tensor_cores(1, n, Hq, Hkv, Dh, P, L) == kernel


@pytest.mark.parametrize("c", q8_kernels.GIVEN_UP)
def test_cases_of_given_up_pages(c):
    kernel, n, Hq, Hkv, Dh, P, T, L, w = c
    assert q8_rule.tensor_cores(3, n, Hq, Hkv, Dh, P, L, inputs.LOCAL, w) == kernel


def test_borders():
    tc = q8_rule.tensor_cores
    # pieces that TMA cannot bring are never for the tensor cores
    for Dh in (64, 128, 256):
        assert not tc(4, 4, 96, 8, Dh, 1, 8192) and not tc(4, 1, 96, 1, Dh, 131, 8192) and tc(4, 4, 96, 8, Dh, 2, 8192)
    assert not tc(4, 1, 96, 1, 64, 9, 8192) and tc(4, 1, 96, 1, 128, 9, 8192)  # odd pieces of 64 bytes a row
    # up to 16 query rows leave it the long ranges, by the window where there is one
    assert tc(1, 4, 32, 8, 128, 16, 17) and not tc(1, 4, 32, 8, 128, 16, 16)
    assert tc(1, 1, 24, 2, 256, 16, 513) and not tc(1, 1, 24, 2, 256, 16, 512)
    assert tc(33, 3, 16, 4, 64, 20, 2648) and not tc(33, 3, 16, 4, 64, 20, 2647)
    assert not tc(1, 4, 32, 8, 128, 16, 8192, inputs.LOCAL, 61) and tc(1, 4, 32, 8, 128, 16, 8192, inputs.LOCAL, 62)
    assert tc(1, 1, 17, 1, 64, 16, 1) and tc(1, 4, 24, 2, 256, 16, 1)  # more than 16 rows: all of them
