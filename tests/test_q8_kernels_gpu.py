"""Decoding over the 8-bit cache: cases made for one of its two kernels (q8_kernels says which; test_q8_kernel_choice holds the rule
to it), against the oracle on the codes' values.  Tolerance: test_q8_decode_gpu's."""
import pytest
import torch

import q8
import q8_kernels
import test_q8_decode_gpu as decode
from paper_2607_08186_gb300 import binding, build, inputs
from test_q8_decode_gpu import _assert_rows, _case, _decode, _i32

pytestmark = pytest.mark.gpu

CROSS, WITHIN, LOCAL = inputs.CROSS, inputs.WITHIN, inputs.LOCAL
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.mark.parametrize("shape", ["climb", "fall", "jump"])
@pytest.mark.parametrize("c", q8_kernels.CHANGE)
def test_scores_that_change(shape, c):
    decode.test_scores_that_change(shape, *c)


@pytest.mark.parametrize("c", q8_kernels.WAVE)
def test_a_wave_shared_by_uneven_sequences(c):
    decode.test_a_wave_shared_by_uneven_sequences(*c)
