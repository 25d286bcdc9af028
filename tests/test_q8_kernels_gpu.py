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


@pytest.mark.parametrize("size", [1e-16, 1e-10, 1e-4, 30.0, 3e4, 1e12])
@pytest.mark.parametrize("c", q8_kernels.SIZES)
def test_sizes_of_queries_and_keys(c, size):
    """Queries far from 1 with keys as far on the other side, so that scores stay of order 1; a row of zeros, one of very
    different magnitudes."""
    _, n, Hq, Hkv, Dh, P, T, L = c
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 6)
    q, kc = (q.float() * size).to(BF), (kc.float() / size).to(BF)
    q[0, 0, 0] = 0.0
    q[0, n - 1, 3, ::2] *= 2.0**-9
    lens = _i32([L])
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, 0)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, 0)
    o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, CROSS)
    assert st == 0
    _assert_rows(o, lse, q, kv, vv, L, 0, n, CROSS, 0)


@pytest.mark.parametrize("scale", [1e-3, 0.02, 0.3])
@pytest.mark.parametrize("c", q8_kernels.SIZES)
def test_explicit_scales(c, scale):
    _, n, Hq, Hkv, Dh, P, T, L = c
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 7)
    lens = _i32([L])
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, 0)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, 0)
    for with_lse in (True, False):
        o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, CROSS, scale=scale, with_lse=with_lse)
        assert st == 0
        _assert_rows(o, lse, q, kv, vv, L, 0, n, CROSS, 0, scale=scale)


@pytest.mark.parametrize("c", q8_kernels.GIVEN_UP)
def test_pages_given_up_behind_a_window(c):
    """A sequence whose pages before its window are given back (entries -1, or pages of other sequences) has the rows that
    it would have with them."""
    _, n, Hq, Hkv, Dh, P, T, L, w = c
    q, kc, vc = _case(3, L, n, Hq, Hkv, Dh, 11)
    lens = [L, L - 37, L // 2 + 1]
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, 1)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, 1)
    given = 0
    for b, x in enumerate(lens):
        first = max(0, (x - 1) * n - w + 1)  # the first position that a row sees
        keep = first // n // P
        table[b, :keep] = _i32([-1, -7, kq.shape[0], 2**31 - 1])[torch.arange(keep) % 4]
        given += keep
    assert given > 0
    o, lse, st = _decode(q, kq, vq, ks, vs, table, _i32(lens), n, LOCAL, window=w)
    assert st == 0
    for b, x in enumerate(lens):
        _assert_rows(o, lse, q, kv, vv, x, b, n, LOCAL, w)
    # one entry more, which a row sees, empties the sequence
    last = max(0, (lens[0] - 1) * n - w + 1) // n // P
    table[0, last] = -1
    o, lse, st = _decode(q, kq, vq, ks, vs, table, _i32(lens), n, LOCAL, window=w)
    assert st == binding.HD_DEVBIT_INDEX and torch.count_nonzero(o[0]) == 0
    _assert_rows(o, lse, q, kv, vv, lens[1], 1, n, LOCAL, w)
