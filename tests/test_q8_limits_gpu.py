"""Decoding over the 8-bit paged cache where values lie far apart: V's scales, a row's weights, the queries' values.
Against the 64-bit oracle on the values that the codes stand for.

Caches here are a few kinds of pages, which a table names over and over, so that many positions stay small.  Tolerance:
test_q8_decode_gpu's."""
import pytest
import torch

import oracle
import q8
from paper_2607_08186_gb300 import binding, build, inputs
from test_q8_decode_gpu import _assert_rows, _decode, _i32

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
F8, BF = torch.float8_e4m3fn, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _codes(x):
    """Values to the nearest codes, as values."""
    return q8.nearest(x.clamp(-448, 448))


def _cache(kinds, order, n, P):
    """Pages of the kinds [(K codes' values [Hkv][P*n][Dh], its exponent, V's, its exponent)], a scale a page, and the
    table row that names them in this order: (k, v, ks, vs, table [1][pages], K's values, V's)."""
    table = torch.tensor([order], dtype=torch.int32)
    out = []
    for i in (0, 2):
        codes = torch.stack([_codes(k[i]) for k in kinds])
        scales = torch.tensor([k[i + 1] + q8.BIAS for k in kinds], dtype=torch.uint8)[:, None, None]
        scales = scales.expand(-1, codes.shape[1], 1).contiguous()
        codes = codes.float().to(F8)
        pages, Hkv, _, Dh = codes.shape
        values = q8.Cache(pages, P, n, Hkv, Dh, P, codes, scales).rows(order, len(order) * P).to(BF)[None]
        out.append((codes, scales, values))
    return out[0][0], out[1][0], out[0][1], out[1][1], table, out[0][2], out[1][2]


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _order(where, one, other, pages):
    """Page kind `one` once among `pages` of `other`: first, last or in the middle."""
    order = [other] * pages
    order[{"first": 0, "last": -1, "middle": pages // 2}[where]] = one
    return order


def _signs(Dh):
    return torch.where(_normal(1, Dh) > 0, 1.0, -1.0).double()


def _key(rows, d):
    """K of a page whose first key scores d binary orders above zero against a query of signs (codes of exponent -6); its
    others 0.  Some columns have the code below what every one should have, the others the code above it."""
    Dh = rows[2]
    grid = q8.nearest(torch.arange(16, 449).double()).unique()
    total = d / 1.4426950408889634 * Dh**0.5 * 64
    i = int((grid <= total / Dh).sum()) - 1
    many = round((total - Dh * float(grid[i])) / float(grid[i + 1] - grid[i]))
    k = torch.zeros(rows, dtype=torch.float64)
    k[:, 0] = _signs(Dh) * torch.where(torch.arange(Dh) < many, grid[i + 1], grid[i])
    return k


# The largest V first, last or among many keys of far smaller ones whose scores lie d binary orders lower and which
# together weigh about as much as it does.  B = 1: many splits; some: shared by one wave; many: a CTA each.  Pages of 4
# rows: the mma.sync kernel, of 16 positions or more the tcgen05 one.
@pytest.mark.parametrize("where", ["first", "last", "middle"])
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,pages,d", [
    (1, 4, 4, 1, 128, 16, 512, 18), (400, 4, 4, 2, 128, 16, 512, 18), (24, 4, 4, 1, 128, 16, 512, 18), (40, 4, 12, 1, 256, 16, 256, 18),
    (24, 4, 8, 1, 64, 16, 512, 18), (1, 1, 4, 1, 128, 4, 4096, 14), (200, 1, 4, 1, 64, 4, 4096, 14), (120, 2, 4, 1, 256, 2, 4096, 13)])
def test_sums_over_scales_far_apart(where, B, n, Hq, Hkv, Dh, P, pages, d):
    rows = (Hkv, P * n, Dh)
    q = _signs(Dh).to(BF).expand(B, n, Hq, Dh).contiguous()
    lens = _i32([pages * P] * B)
    big = (_key(rows, d), -6, _normal(2, *rows) * 100, q8.E_MAX)
    for ev in (q8.E_MIN, q8.E_MIN + 9):
        small = (_normal(3, *rows) * 32, -12, _normal(4, *rows) * 100 * (ev > q8.E_MIN), ev)
        k, v, ks, vs, table, kv, vv = _cache([big, small], _order(where, 0, 1, pages), n, P)
        for mode in (CROSS, WITHIN):
            o, lse, st = _decode(q, k, v, ks, vs, table.expand(B, -1).contiguous(), lens, n, mode)
            assert st == 0
            for b in {0, B - 1}:
                _assert_rows(o[b:b + 1], lse[b:b + 1], q[:1], kv, vv, pages * P, 0, n, mode, 0)


def test_sums_of_many_light_keys():
    """The same on the mma.sync kernel where the largest V comes first, and a CTA has a sequence and head whole: 27
    orders lower, a key's weight times its V's scale is below fp32's smallest beside that one's.  (Pages of a prime
    number of rows, which TMA would bring one at a time.)"""
    n, Hq, Hkv, Dh, P, pages, d, B = 1, 2, 1, 64, 131, 6400, 27.2, 960
    rows = (Hkv, P * n, Dh)
    big = (_key(rows, d), -6, _normal(2, *rows) * 100, q8.E_MAX)
    small = (_normal(3, *rows) * 4, -12, torch.zeros(rows, dtype=torch.float64), q8.E_MIN)
    k, v, ks, vs, table, kv, vv = _cache([big, small], _order("first", 0, 1, pages), n, P)
    q = _signs(Dh).to(BF).expand(B, n, Hq, Dh).contiguous()
    o, lse, st = _decode(q, k, v, ks, vs, table.expand(B, -1).contiguous(), _i32([pages * P] + [P] * (B - 1)), n, CROSS)
    assert st == 0
    _assert_rows(o[:1], lse[:1], q[:1], kv, vv, pages * P, 0, n, CROSS, 0)


def _assert_columns(o, q, kv, vv, T, n, mode, window):
    """One sequence's rows, whose weights may lose 2^-7 of them all beside what test_q8_decode_gpu allows: column by
    column, against the column's largest visible V."""
    a = (q, kv, vv, _i32([T]), n, mode)
    o_r, _, bad = oracle.decode(*a, window=window)
    A, _, _ = oracle.decode(q, kv, vv.abs(), *a[3:], window=window)
    assert bad == 0
    n_, Hq, Hkv = q.shape[1], q.shape[2], kv.shape[2]
    most = vv[0].double().abs().amax(0).repeat_interleave(Hq // Hkv, 0)  # [Hq][Dh]
    err = (o[0].double() - o_r[0]).abs()
    lim = (2.0**-8 + 1e-3) * o_r[0].abs() + (2.0**-9 + 2.0**-11 + 1e-3) * A[0] + 2.0**-7 * most
    assert bool((err <= lim).all()), float((err / lim).max())


# V of one page is far larger than all others, and only in one column; the others' columns hold what they would without it.
@pytest.mark.parametrize("apart", [8, 14, 20, 24, 31, 48, 70])
@pytest.mark.parametrize("where", ["first", "last", "middle"])
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,pages,window", [
    (1, 4, 4, 1, 128, 16, 64, 0), (400, 4, 4, 2, 128, 16, 64, 0), (24, 4, 16, 1, 128, 16, 128, 0), (40, 4, 12, 1, 256, 16, 64, 3000),
    (24, 4, 8, 1, 64, 16, 128, 0), (1, 1, 4, 1, 128, 4, 512, 0), (200, 1, 4, 1, 64, 4, 512, 1500), (120, 2, 4, 1, 256, 2, 512, 0)])
def test_columns_beside_a_far_larger_block(where, apart, B, n, Hq, Hkv, Dh, P, pages, window):
    rows = (Hkv, P * n, Dh)
    huge = _normal(2, *rows) * 100
    huge[..., 1:] = 0.0
    large = (_normal(5, *rows) * 100, -6, huge, -30 + apart)
    usual = (_normal(3, *rows) * 100, -6, _normal(4, *rows) * 100, -30)
    k, v, ks, vs, table, kv, vv = _cache([large, usual], _order(where, 0, 1, pages), n, P)
    q = _normal(6, 1, n, Hq, Dh).to(BF)
    L = pages * P
    for mode in (LOCAL,) if window else (CROSS, WITHIN):
        o, lse, st = _decode(q.expand(B, -1, -1, -1).contiguous(), k, v, ks, vs, table.expand(B, -1).contiguous(), _i32([L] * B), n,
                             mode, window)
        assert st == 0
        _, lse_r, _ = oracle.decode(q, kv, vv, _i32([L]), n, mode, window=window)
        for b in {0, B - 1}:
            _assert_columns(o[b:b + 1], q, kv, vv, L, n, mode, window)
            assert float((lse[b].double() - lse_r[0]).abs().max()) <= 1e-3


# Queries whose largest value meets zeros of K, and whose others, 2^small times as large, make the scores; every other head
# has ordinary queries beside a smaller K.  The second shape's K is small in one half of the sequence.
@pytest.mark.parametrize("small", [-8, -12, -16, -22, -28, -36, -48])
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,pages", [
    (1, 4, 4, 1, 128, 16, 64), (24, 4, 16, 1, 128, 16, 64), (400, 1, 24, 2, 128, 16, 64), (40, 4, 12, 1, 256, 16, 32),
    (3, 1, 16, 2, 256, 64, 32), (6, 4, 8, 1, 256, 16, 32), (2, 4, 16, 1, 256, 16, 32), (24, 4, 8, 1, 64, 16, 64), (1, 1, 4, 1, 128, 4, 256), (200, 1, 4, 1, 64, 4, 256), (12, 4, 24, 2, 256, 1, 256)])
def test_small_values_of_queries(small, B, n, Hq, Hkv, Dh, P, pages):
    rows = (Hkv, P * n, Dh)
    k_large, k_small = _normal(2, *rows) * 100, _normal(3, *rows) * 100
    k_large[..., 0] = 0.0
    large = (k_large, -7 - small, _normal(4, *rows) * 100, -6)
    little = (k_small, -9, _normal(5, *rows) * 100, -6)
    k, v, ks, vs, table, kv, vv = _cache([large, little], [0] * (pages // 2) + [1] * (pages - pages // 2), n, P)
    q = _normal(6, 1, n, Hq, Dh)
    q[..., 1:] *= 2.0**small
    q[:, :, ::2, 0] = 1.5
    q = q.to(BF)
    L = pages * P
    for mode in (CROSS, WITHIN):
        o, lse, st = _decode(q.expand(B, -1, -1, -1).contiguous(), k, v, ks, vs, table.expand(B, -1).contiguous(), _i32([L] * B), n, mode)
        assert st == 0
        for b in {0, B - 1}:
            _assert_rows(o[b:b + 1], lse[b:b + 1], q, kv, vv, L, 0, n, mode, 0)


# Queries near bf16's largest values over K's smallest scale: scores of 2^60 and more, whose products in codes pass fp32's
# range before the scale brings them back.  The largest score takes the row; LSE relative to it.
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,pages", [(1, 4, 4, 1, 128, 16, 8), (5, 4, 12, 1, 256, 16, 6), (3, 4, 8, 1, 64, 16, 8), (2, 1, 4, 1, 128, 4, 16)])
def test_large_queries_over_small_keys(B, n, Hq, Hkv, Dh, P, pages):
    rows = (Hkv, P * n, Dh)
    page = (_normal(2, *rows) * 100, q8.E_MIN, _normal(4, *rows) * 100, -6)
    k, v, ks, vs, table, kv, vv = _cache([page], [0] * pages, n, P)
    q = (_normal(6, 1, n, Hq, Dh) * 2.0**124).to(BF)
    L = P  # (pages past the first would repeat its scores)
    o, lse, st = _decode(q.expand(B, -1, -1, -1).contiguous(), k, v, ks, vs, table.expand(B, -1).contiguous(), _i32([L] * B), n, CROSS)
    assert st == 0
    o_r, lse_r, _ = oracle.decode(q, kv, vv, _i32([L]), n, CROSS)
    for b in {0, B - 1}:
        assert float((lse[b].double() / lse_r[0] - 1).abs().max()) <= 1e-3
        assert float((o[b].double() - o_r[0]).abs().max()) <= 2.0**-8 * float(o_r.abs().max())


# Batches in which some sequences have a page far larger, or queries far apart over large K, and the others do not, of uneven
# lengths, some empty or on bad pages: CTAs that go on from one to another keep their bounds apart.
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,pages", [(24, 4, 16, 1, 128, 16, 96), (40, 4, 12, 1, 256, 16, 48), (128, 2, 16, 1, 64, 16, 60), (33, 4, 96, 4, 128, 16, 40),
                                                   (60, 1, 4, 1, 128, 4, 200), (4, 4, 4, 1, 128, 16, 96)])
def test_sequences_far_apart_beside_ordinary_ones(B, n, Hq, Hkv, Dh, P, pages):
    rows = (Hkv, P * n, Dh)
    huge = _normal(2, *rows) * 100
    huge[..., 1:] = 0.0
    k_large = _normal(3, *rows) * 100
    k_large[..., 0] = 0.0
    usual = (_normal(4, *rows) * 100, -6, _normal(5, *rows) * 100, -30)
    kinds = [usual, (_normal(6, *rows) * 100, -6, huge, 10), (k_large, 13, _normal(7, *rows) * 100, -30), (_normal(8, *rows) * 100, -6, _normal(9, *rows), q8.E_MAX)]
    orders = [[0] * pages, [0] * pages, [2] * pages, [0] * pages]
    orders[1][pages // 3], orders[3][1] = 1, 3
    caches = [_cache(kinds, o, n, P) for o in orders]
    k, v, ks, vs = caches[0][:4]
    which = [(b * 7 // 3) % 4 for b in range(B)]
    lens = [pages * P - (b * 53) % (pages * P - P) for b in range(B)]
    lens[1] = 0
    table = torch.cat([caches[w][4] for w in which]).clone()
    table[2, 0] = -1
    small = _normal(10, 1, n, Hq, Dh)
    apart = small.clone()
    apart[..., 1:] *= 2.0**-20
    apart[..., 0] = 1.5
    q = torch.cat([apart if w == 2 else small for w in which]).to(BF)
    for mode, window in ((CROSS, 0), (LOCAL, 30 * n), (WITHIN, 0)):
        o, lse, st = _decode(q, k, v, ks, vs, table, _i32(lens), n, mode, window)
        assert st == (binding.HD_DEVBIT_INDEX if mode != LOCAL else st)
        for b in (1, 2) if mode != LOCAL else (1,):
            assert torch.count_nonzero(o[b]) == 0 and bool((lse[b] == -float("inf")).all())
        for b in ({0, B - 1} | set(range(3, min(B, 12)))) - {1, 2}:
            kv, vv = caches[which[b]][5:]
            _assert_columns(o[b:b + 1], q[b:b + 1], kv, vv, lens[b], n, mode, window)
            _, lse_r, _ = oracle.decode(q[b:b + 1], kv, vv, _i32([lens[b]]), n, mode, window=window)
            assert float((lse[b].double() - lse_r[0]).abs().max()) <= 1e-3
