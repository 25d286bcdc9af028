"""Packed prompts with several entries of the list for every CTA (or pair of CTAs), at all head dims: what a CTA carries
from one entry to the next, and rows settled over several entries.  Each case asserts that there are more places than
two rounds of CTAs take.  Reference and tolerances of test_packed_gpu."""
import pytest
import torch

from paper_2607_08186_gb300 import build, inputs
from test_packed_gpu import INF, NAN, _case, _check, _near, _reference, _run

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
SMS, SHORT_ROWS = 152, 48


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _places(lens, n, Hq, Hkv, mode):
    """Places of the list at least: the entries (short sequences counted as if they filled their shared tiles) for
    every head slot and stream."""
    mult, streams = (1, n) if mode == WITHIN else (n, 1)
    pairs = (Hq // Hkv) % 2 == 0
    tile, slots = (128, Hq // 2) if pairs else (256, Hq)
    rows = [x * mult for x in lens]
    entries = sum(-(-r // tile) for r in rows if r > SHORT_ROWS) + -(-sum(r for r in rows if r <= SHORT_ROWS) // tile)
    return entries * slots * streams


def _lens(count, most, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(1, most + 1, (count,), generator=g).tolist()
    lens[3], lens[count // 2], lens[-1] = 0, most, 1
    return lens


# (streams, heads, sequences, longest): an average sequence of more than 64 rows and of fewer (the head-dim-64 kernel
# without and with shared tiles), pairs of heads and two tiles of a head, whose second tile is often empty
CASES = [(3, 16, 4, 64, 24, 400), (3, 16, 4, 64, 90, 60), (3, 18, 6, 64, 24, 500), (2, 15, 5, 64, 60, 90), (1, 32, 8, 64, 40, 300),
         (3, 16, 4, 128, 24, 300), (2, 15, 5, 128, 40, 200), (2, 24, 4, 256, 20, 200), (3, 6, 2, 256, 40, 150)]


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 70), (LOCAL, 333)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,B,most", CASES)
def test_many_entries(mode, w, n, Hq, Hkv, Dh, B, most):
    lens = _lens(B, most, B + n)
    assert _places(lens, n, Hq, Hkv, mode) > 2 * (SMS if Dh < 256 else SMS // 2)
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 7 + n + Hq, before=1, behind=2)
    _check(q, k, v, off, n, mode, w)


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 70)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,B,most", [c for c in CASES if c[0] != 1])
def test_hidden_values_in_many_entries(mode, w, n, Hq, Hkv, Dh, B, most, bad):
    # in every second sequence one token's first stream is not finite: rows that do not see it are as if it were
    lens = _lens(B, most, B + n)
    assert _places(lens, n, Hq, Hkv, mode) > 2 * (SMS if Dh < 256 else SMS // 2)
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 17 + n + Hq)
    kb, vb = k.clone(), v.clone()
    at = {i: (37 * i) % x for i, x in enumerate(lens) if i % 2 == 0 and x > 0}
    for i, t in at.items():
        vb[(off[i] + t) * n, :, 1] = bad
        kb[(off[i] + t) * n, :, 2] = bad
    o, lse, st = _run(q, kb, vb, off, n, mode, w)
    assert st == 0
    for i, x in enumerate(lens):
        if x == 0:
            continue
        r = slice(off[i] * n, off[i + 1] * n)
        o_r, A, lse_r = _reference(q, k, v, r, n, mode, w)
        p = torch.arange(x * n)
        sees = torch.zeros_like(p, dtype=torch.bool)
        if i in at:
            sees = p >= at[i] * n
            if mode == WITHIN:
                sees &= p % n == 0
            if mode == LOCAL:
                sees &= p - w < at[i] * n
        if not bool(sees.all()):
            _near(o[r], o_r, A, lse[:, r], lse_r, ~sees)
        if bad != bad and bool(sees.any()):
            assert bool(o[r][sees].isnan().all()) and bool(lse[:, r][:, sees].isnan().all())


@pytest.mark.parametrize("n,Hq,Hkv,Dh,B,most", [CASES[0], CASES[2], CASES[5], CASES[7]])
def test_repeats_give_the_same_bits(n, Hq, Hkv, Dh, B, most):
    lens = _lens(B, most, B + n)
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 27)
    want = _run(q, k, v, off, n, CROSS)
    for _ in range(3):
        got = _run(q, k, v, off, n, CROSS)
        assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[1], want[1])
    # a sequence of more than 48 rows has the bits that it has alone
    i = max(range(B), key=lens.__getitem__)
    r = slice(off[i] * n, off[i + 1] * n)
    alone = _run(*(x[r].contiguous() for x in (q, k, v)), [0, lens[i]], n, CROSS)
    assert torch.equal(want[0][r].view(torch.int16), alone[0].view(torch.int16)) and torch.equal(want[1][:, r], alone[1])
