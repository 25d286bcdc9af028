"""The rule that picks the paged decoding kernel, compiled for the host: it goes by the rows of a page that come in
one piece, not by the page's rows (no GPU)."""
import pytest

import paged_rule
from paged_rule import NONE, ONLY_256, WITH_128

LONG = 1 << 17  # positions, above every limit of the rule


@pytest.fixture(scope="module")
def rule():
    return paged_rule.lib()


def test_pieces(rule):
    for most in (32, 64, 128):
        for prow in list(range(1, 700)) + [2**30, 2**30 - 35, 999983]:
            want = max(d for d in range(1, most + 1) if prow % d == 0)
            assert rule.piece(prow, most) == want


def test_a_page_is_what_its_pieces_are(rule):
    for B, n, Hq, Hkv, Dh in ((4, 4, 96, 8, 128), (16, 3, 96, 8, 128), (4, 4, 24, 2, 256), (2, 2, 24, 2, 256), (1, 8, 64, 8, 256)):
        for piece, primes in ((1, (131, 137, 257, 509)), (2, (131, 149)), (4, (131, 151)), (8, (17, 131))):
            small = rule.kernel(B, n, Hq, Hkv, Dh, piece, LONG)
            for p in primes:
                if rule.piece(piece * p, 128) == piece:
                    assert rule.kernel(B, n, Hq, Hkv, Dh, piece * p, LONG) == small, (n, Hq, Dh, piece, p)
    # one row at a time is never for the tensor cores, whole pieces are
    assert rule.kernel(4, 4, 96, 8, 128, 131, LONG) == rule.kernel(4, 4, 24, 2, 256, 257, LONG) == NONE
    assert rule.kernel(4, 4, 96, 8, 128, 64, LONG) == rule.kernel(4, 4, 96, 8, 128, 131 * 64, LONG) == WITH_128
    assert rule.kernel(2, 2, 24, 2, 256, 64, LONG) == ONLY_256
