"""Paged decoding, each kernel where it is taken: the cases say by the rule itself (tests/paged_rule.py) which kernel
they reach.  Tolerances and oracle of test_paged_gpu."""
import pytest
import torch

import guards
import oracle
import paged_rule
import paging
from paper_2607_08186_gb300 import binding, build, inputs
from test_paged_gpu import NAN, _assert_empty, _assert_rows, _case, _check, _decode, _i32

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


# large pages that come in small pieces: prime and odd numbers of tokens.  From 4 and 5 rows a piece on they are the
# tensor cores', below the other kernel's
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 900)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P,tc", [(4, 96, 8, 128, 131, False), (4, 24, 1, 128, 131, True), (5, 10, 1, 128, 131, True),
                                              (6, 12, 2, 128, 137, True), (1, 48, 1, 128, 131, False), (2, 24, 2, 256, 131, False),
                                              (4, 32, 2, 256, 131, False), (4, 24, 1, 256, 131, True), (7, 14, 2, 256, 131, True),
                                              (5, 20, 2, 256, 149, True)])
def test_large_pages_of_small_pieces(mode, w, n, Hq, Hkv, Dh, P, tc):
    L = 700
    assert paged_rule.tensor_cores(2, n, Hq, Hkv, Dh, P, L, w) == tc
    q, kc, vc = _case(2, L, n, Hq, Hkv, Dh, 70 + n + Hq)
    _check(q, kc, vc, _i32([L, 401]), n, mode, w, P, seed=3)
