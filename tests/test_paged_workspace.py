"""The workspace of a paged decoding step: what is enough for a capacity is enough for every step within it, so
that a server may allocate once and pass each step's longest length as max_tokens (no GPU)."""
import random

import pytest

from paper_2607_08186_gb300 import binding, build, inputs

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


HEADS = [(32, 8, 128), (96, 8, 128), (24, 2, 256), (8, 1, 256), (16, 4, 64), (4, 4, 64), (12, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("B", [1, 2, 7, 16, 33, 500])
@pytest.mark.parametrize("n", [1, 4, 7])
def test_enough_for_every_shorter_step(heads, B, n):
    need = lambda T, mode=CROSS, w=0: binding.sfa_decode_paged_workspace_bytes(B, T, n, *heads, mode, w)  # noqa: E731
    last = 0
    for T in list(range(1, 700)) + list(range(700, 20000, 16)) + [1 << e for e in range(15, 27)]:
        now = need(T)
        assert now >= last > -1, T
        last = now
    r = random.Random(n)
    for _ in range(300):
        T, w = r.randint(1, 40000), r.randint(1, 200000)
        assert need(T, LOCAL, w) <= need(r.randint(T, 40000), LOCAL, r.randint(w, 2**31 - 1))
        assert need(T, LOCAL, w) <= need(T, WITHIN)
