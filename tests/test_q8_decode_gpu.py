"""Decoding over the 8-bit paged cache on the GPU, against the 64-bit oracle on the values that the codes stand for.

Tolerance of O, element by element.  The tcgen05 kernel rounds P to f16 (off by at most half a step, 2^-11 relative) and
then to three codes of three bits, nine bits (2^-9), or below those codes' range by 2^-28 of the row's largest P; the
mma.sync kernel to f16 alone.  O is rounded to bf16 (2^-8).  1e-3 (A + |O|), A = sum P |V|, covers the fp32 sums of up to
2^17 terms and exp2 of scores that are off by Dh * 2^-24 * sum |q k| * scale (1.6e-4 at Dh = 256 and N(0, 1) operands; a
query's two codes leave at most 2^-22 of the row's largest value beside that).  LSE: 1e-3, the same scores' error with a
margin of 5."""
import pytest
import torch

import guards
import oracle
import q8
from paper_2607_08186_gb300 import binding, build, inputs

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
I32, F8, BF = torch.int32, torch.float8_e4m3fn, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=I32)


def _case(B, Lcap, n, Hq, Hkv, Dh, seed):
    return (inputs.normal_bf16((B, n, Hq, Dh), seed), inputs.normal_bf16((B, Lcap * n, Hkv, Dh), seed + 1),
            inputs.normal_bf16((B, Lcap * n, Hkv, Dh), seed + 2))


def _decode(q, kc, vc, ks, vs, table, lens, n, mode, window=0, max_tokens=None, scale=0.0, with_lse=True):
    """(o, lse, status) of one call, on the host."""
    B, _, Hq, Dh = q.shape
    T = max_tokens or table.shape[1] * (kc.shape[2] // n)
    ws = guards.empty((binding.sfa_decode_paged_q8_workspace_bytes(B, T, n, Hq, kc.shape[1], Dh, mode, window),), torch.uint8,
                      0xFF, what="workspace")
    o = guards.empty(q.shape, BF, 7.0)
    lse = guards.empty((B, Hq, n), torch.float32, 7.0) if with_lse else None
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.sfa_decode_paged_q8(q.cuda(), kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(), table.cuda(), lens.cuda(), o, n, mode,
                                ws, max_tokens=T, lse=lse, softmax_scale=scale, window=window, dev_status=st)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu() if with_lse else None, int(st.item())


def _assert_rows(o, lse, q, kv, vv, T, b, n, mode, window, scale=0.0):
    """Sequence b's rows against the oracle on the values."""
    a = (q[b:b + 1], kv[b:b + 1], vv[b:b + 1], _i32([T]), n, mode)
    o_r, lse_r, bad = oracle.decode(*a, window=window, scale=scale)
    A, _, _ = oracle.decode(a[0], a[1], a[2].abs(), *a[3:], window=window, scale=scale)
    assert bad == 0
    err = (o[b].double() - o_r[0]).abs()
    lim = 2.0**-8 * o_r[0].abs() + (2.0**-9 + 2.0**-11 + 1e-3) * A[0] + 1e-3 * o_r[0].abs()
    assert bool((err <= lim).all()), float((err / lim).max())
    if lse is not None:
        assert float((lse[b].double() - lse_r[0]).abs().max()) <= 1e-3


def _assert_empty(o, lse, b):
    assert torch.count_nonzero(o[b]) == 0 and bool((lse[b] == -float("inf")).all())


def _check(q, kc, vc, lens, n, mode, window, P, T, seed=0, max_tokens=None, width=None):
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, seed, width=width)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, seed, width=width, scale_fill=0)
    o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, mode, window, max_tokens)
    assert st == 0
    for b, L in enumerate(lens.tolist()):
        _assert_empty(o, lse, b) if L == 0 else _assert_rows(o, lse, q, kv, vv, L, b, n, mode, window)


MASKS = [(WITHIN, 0), (CROSS, 0), (LOCAL, 1), (LOCAL, 100), (LOCAL, 2**31 - 1)]


# query rows per K/V head: 1 to 64 in one to four row tiles, 96 and 140 in groups; pages of every size against tiles of 128
# positions (64 at head dim 256): smaller, equal, larger, odd, prime, one token with more streams than a tile holds, rows
# that TMA cannot place (odd pieces at head dim 64); blocks of a token, of some, of the page
@pytest.mark.parametrize("mode,w", MASKS)
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P,T", [
    (4, 32, 8, 128, 16, 16), (4, 32, 8, 128, 16, 1), (8, 32, 8, 128, 3, 3), (8, 64, 8, 128, 1, 1), (1, 8, 8, 128, 64, 8),
    (3, 6, 2, 128, 7, 7), (2, 4, 4, 64, 8, 2), (3, 16, 4, 64, 50, 10), (4, 8, 2, 64, 5, 1), (1, 8, 2, 128, 131, 131),
    (4, 8, 2, 128, 43, 43), (4, 32, 8, 128, 2, 1), (70, 2, 1, 64, 1, 1), (140, 1, 1, 64, 1, 1), (5, 10, 2, 64, 9, 3),
    (1, 4, 4, 64, 9, 3), (4, 96, 8, 128, 16, 16), (8, 32, 2, 128, 3, 1), (3, 96, 8, 128, 1, 1), (4, 12, 1, 128, 43, 43),
    (8, 96, 8, 128, 16, 4), (4, 16, 2, 64, 32, 32), (4, 96, 8, 64, 16, 16)])
def test_ragged(mode, w, n, Hq, Hkv, Dh, P, T):
    q, kc, vc = _case(4, 150, n, Hq, Hkv, Dh, n + Hq + P)
    _check(q, kc, vc, _i32([150, 1, 0, 129]), n, mode, w, P, T)


@pytest.mark.parametrize("mode,w", MASKS)
@pytest.mark.parametrize("n,Hq,Hkv,P,T", [(4, 24, 2, 16, 16), (1, 4, 1, 3, 3), (3, 6, 2, 5, 1), (8, 32, 2, 4, 2), (4, 24, 2, 64, 16),
                                          (2, 12, 2, 1, 1), (8, 64, 2, 6, 6), (1, 12, 1, 131, 1), (4, 8, 2, 16, 8), (2, 16, 1, 20, 5)])
def test_ragged_head_dim_256(mode, w, n, Hq, Hkv, P, T):
    q, kc, vc = _case(4, 150, n, Hq, Hkv, 256, 40 + n + Hq + P)
    _check(q, kc, vc, _i32([150, 1, 0, 129]), n, mode, w, P, T)


@pytest.mark.parametrize("n,Hq,Hkv,Dh,mode,P,T", [(4, 32, 8, 128, WITHIN, 16, 16), (4, 32, 8, 128, CROSS, 37, 1),
                                                  (4, 24, 2, 256, WITHIN, 16, 4), (4, 24, 2, 256, CROSS, 3, 3),
                                                  (4, 96, 8, 128, CROSS, 32, 32), (3, 16, 4, 64, WITHIN, 20, 20)])
def test_long(n, Hq, Hkv, Dh, mode, P, T):
    q, kc, vc = _case(2, 6000, n, Hq, Hkv, Dh, 8)
    _check(q, kc, vc, _i32([6000, 3001]), n, mode, 0, P, T)


@pytest.mark.parametrize("B,Hq,Hkv,Dh,P,T", [(33, 4, 1, 128, 7, 7), (70, 2, 2, 64, 16, 4), (40, 8, 1, 256, 20, 20)])
def test_many_sequences(B, Hq, Hkv, Dh, P, T):
    n, L = 4, 500
    lens = [max(0, int(L * (0.618 * b % 1.0)) - 60) for b in range(B)]
    lens[0] = L
    q, kc, vc = _case(B, L, n, Hq, Hkv, Dh, B)
    _check(q, kc, vc, _i32(lens), n, CROSS, 0, P, T)


# scores that climb, fall or jump along the sequence: references that go up at every tile, never, or late; rows of one
# split with many tiles, and of several; more query rows than a CTA takes; scales that change inside a tile or rarely
@pytest.mark.parametrize("shape", ["climb", "fall", "jump"])
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,T,L", [(2, 4, 8, 2, 128, 16, 16, 700), (1, 4, 24, 2, 256, 16, 4, 500), (160, 1, 4, 4, 64, 32, 1, 900),
                                                 (90, 2, 16, 8, 128, 8, 2, 600), (1, 8, 96, 8, 128, 8, 8, 200), (3, 3, 16, 4, 64, 32, 8, 1100)])
def test_scores_that_change(shape, B, n, Hq, Hkv, Dh, P, T, L):
    q, kc, vc = _case(B, L, n, Hq, Hkv, Dh, 11)
    at = torch.arange(L * n) / (L * n)
    size = {"climb": 8 * at, "fall": 8 * (1 - at), "jump": torch.where(at > 0.7, 8.0, 0.1)}[shape]
    # keys along the queries of their group, so that all rows' scores follow `size` (up to about 8 * Dh / sqrt(Dh))
    along = q.float().view(B, n, Hkv, Hq // Hkv, Dh)[:, 0, :, 0] / 4
    kc = (along[:, None] * size[None, :, None, None] + 0.1 * kc.float()).to(BF)
    lens = [L - 3 * b % (L // 2) for b in range(B)]
    few = [0, B // 2, B - 1] if B > 3 else range(B)
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, 1)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, 1)
    for mode, w in ((CROSS, 0), (WITHIN, 0), (LOCAL, 150)):
        o, lse, st = _decode(q, kq, vq, ks, vs, table, _i32(lens), n, mode, w)
        assert st == 0
        for b in few:
            _assert_rows(o, lse, q, kv, vv, lens[b], b, n, mode, w)


# sequences whose tables name the same few pages, so that long ones in numbers stay small here: splits of one CTA and of many
# tiles, shared out by length or not; blocks of one token, whose scales a split's first positions share with nobody, over
# and over; pieces that leave positions of a tile over; scales whose bytes end inside a word
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,T", [(132, 1, 8, 4, 64, 48, 1), (132, 1, 8, 4, 64, 16, 16), (100, 4, 12, 3, 128, 12, 1),
                                               (60, 1, 9, 9, 128, 24, 1), (12, 4, 32, 8, 128, 16, 16), (24, 2, 48, 8, 128, 15, 1),
                                               (128, 1, 12, 3, 256, 9, 9), (20, 4, 48, 1, 256, 10, 5), (9, 8, 72, 3, 128, 11, 11),
                                               (20, 8, 8, 4, 64, 6, 1), (100, 8, 8, 4, 64, 6, 1),
                                               (132, 8, 4, 2, 64, 2, 2)])
def test_long_sequences_in_numbers(B, n, Hq, Hkv, Dh, P, T):
    L = 1500
    q, kc, vc = _case(2, L, n, Hq, Hkv, Dh, B + P)
    kq, ks, table, kv = q8.quantised(kc, [L, L], P, T, n, 3)
    vq, vs, _, vv = q8.quantised(vc, [L, L], P, T, n, 3)
    which = [b % 2 for b in range(B)]
    lens = [1 + (b * 977) % L for b in range(B)]
    lens[0], lens[1], lens[2], lens[3], lens[-1] = L, 0, -5, L + 1, L
    q = torch.cat([q, inputs.normal_bf16((B - 2, n, Hq, Dh), 77)])
    for mode, w in ((CROSS, 0), (WITHIN, 0), (LOCAL, 700 * n + 1)):
        o, lse, st = _decode(q, kq, vq, ks, vs, table[which], _i32(lens), n, mode, w, max_tokens=L)
        assert st == binding.HD_DEVBIT_INDEX
        for b in (1, 2, 3):
            _assert_empty(o, lse, b)
        for b in (0, 4, 5, B // 2, B - 1):
            i = which[b]
            _assert_rows(o[b:b + 1], lse[b:b + 1], q[b:b + 1], kv[i:i + 1], vv[i:i + 1], lens[b], 0, n, mode, w)


# batches whose tiles one wave of CTAs shares, with lengths from nothing to everything: a sequence in more parts than are
# merged, in one, in none; parts of many sequences; the lengths of a captured call replaced between its replays
@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,T,L", [(2, 4, 4, 1, 64, 32, 8, 16000), (2, 4, 4, 1, 128, 16, 16, 16000), (6, 4, 48, 4, 128, 16, 16, 2500),
                                                 (128, 2, 16, 2, 256, 20, 5, 1200), (128, 4, 48, 2, 64, 16, 1, 900), (33, 4, 24, 1, 128, 9, 3, 1000)])
def test_a_wave_shared_by_uneven_sequences(B, n, Hq, Hkv, Dh, P, T, L):
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, B + P)
    kq, ks, table, kv = q8.quantised(kc, [L], P, T, n, 3)
    vq, vs, _, vv = q8.quantised(vc, [L], P, T, n, 3)
    q = inputs.normal_bf16((B, n, Hq, Dh), 78)
    many = [b * 37 % 90 for b in range(B)]
    batches = [[L] + [0] * (B - 1), [0] * (B - 1) + [L], [1] * B, [0] * B, many[:-1] + [L], [L - b % 7 for b in range(B)]]
    dev = [x.cuda() for x in (q, kq, vq, ks, vs, table.expand(B, -1).contiguous())]
    lens = torch.zeros(B, dtype=I32, device="cuda")
    ws = guards.empty((binding.sfa_decode_paged_q8_workspace_bytes(B, L, n, Hq, Hkv, Dh, CROSS),), torch.uint8, 0xFF, what="workspace")
    o, lse = guards.empty(q.shape, BF, 7.0), guards.empty((B, Hq, n), torch.float32, 7.0)
    st = torch.zeros(1, dtype=I32, device="cuda")
    call = lambda: binding.sfa_decode_paged_q8(*dev, lens, o, n, CROSS, ws, max_tokens=L, lse=lse, dev_status=st)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for batch in batches:
        lens.copy_(_i32(batch))
        g.replay()
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        oc, lc = o.cpu(), lse.cpu()
        for b in {0, 1, B // 2, B - 1}:
            if batch[b]:
                _assert_rows(oc[b:b + 1], lc[b:b + 1], q[b:b + 1], kv, vv, batch[b], 0, n, CROSS, 0)
            else:
                _assert_empty(oc, lc, b)
        ob = o.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), ob.view(torch.int16))


@pytest.mark.parametrize("B,n,Hq,Hkv,Dh,P,L", [(40, 2, 8, 2, 128, 16, 900), (70, 2, 48, 2, 64, 32, 1000), (40, 3, 36, 2, 256, 12, 700)])
def test_a_shared_wave_keeps_bad_pages_and_hidden_nan_to_their_sequences(B, n, Hq, Hkv, Dh, P, L):
    q, kc, vc = _case(2, L, n, Hq, Hkv, Dh, 21)
    vc[1, (L - 300) * n, 0, 3] = float("nan")  # of stream 0: hidden from the other streams' rows
    kq, ks, table, kv = q8.quantised(kc, [L, L], P, P, n, 3)
    vq, vs, _, vv = q8.quantised(vc, [L, L], P, P, n, 3)
    q = inputs.normal_bf16((B, n, Hq, Dh), 79)
    which = [1 if b % 5 == 2 else 0 for b in range(B)]
    tables = table[which].clone()
    wrong = {3: kq.shape[0], 4: -1, B // 2: 2**31 - 1, B - 1: -5}
    for b, page in wrong.items():
        tables[b, (b * 7) % (L // P)] = page
    lens = [L - 2 * (b % 9) for b in range(B)]
    vv[1, (L - 300) * n, 0, 3] = 0.0
    o, lse, st = _decode(q, kq, vq, ks, vs, tables, _i32(lens), n, WITHIN, max_tokens=L)
    assert st == binding.HD_DEVBIT_INDEX
    for b in range(B):
        if b in wrong:
            _assert_empty(o, lse, b)
        elif which[b] == 0:
            if b % 3 == 0 or b < 9:
                _assert_rows(o[b:b + 1], lse[b:b + 1], q[b:b + 1], kv[:1], vv[:1], lens[b], 0, n, WITHIN, 0)
        else:  # stream 0's rows of the first K/V head are NaN in that column, and nothing else is
            assert bool(torch.isnan(o[b, 0, :Hq // Hkv, 3]).all()) and int(torch.isnan(o[b]).sum()) == Hq // Hkv
            ob = o[b:b + 1].clone()
            keep = torch.ones(n, Hq, Dh, dtype=torch.bool)
            keep[0, :Hq // Hkv, 3] = False
            o_r, lse_r, _ = oracle.decode(q[b:b + 1], kv[1:], vv[1:], _i32([lens[b]]), n, WITHIN)
            A, _, _ = oracle.decode(q[b:b + 1], kv[1:], vv[1:].abs(), _i32([lens[b]]), n, WITHIN)
            lim = 2.0**-8 * o_r.abs() + (2.0**-9 + 2.0**-11 + 1e-3) * A + 1e-3 * o_r.abs()
            assert bool(((ob.double() - o_r).abs() <= lim)[0][keep].all())
            assert float((lse[b].double() - lse_r[0]).abs().max()) <= 1e-3


@pytest.mark.parametrize("Dh,P", [(64, 16), (128, 16), (256, 16), (128, 3)])
def test_wrong_lengths_and_pages_empty_their_sequence_alone(Dh, P):
    n, Hq, Hkv, L = 2, 8, 2, 90
    q, kc, vc = _case(5, L, n, Hq, Hkv, Dh, 3)
    lens = _i32([L, 70, 60, 50, 40])
    kq, ks, table, kv = q8.quantised(kc, lens, P, P, n, 1)
    vq, vs, _, vv = q8.quantised(vc, lens, P, P, n, 1)
    table[1, 1], table[2, 0] = kq.shape[0], -7  # no pages of the pool
    lens[3], lens[4] = L + 1, -1
    for T in (L, L * 40):  # one split, and several
        wide = torch.cat([table, torch.full((5, T // P + 1), -1, dtype=I32)], 1)
        o, lse, st = _decode(q, kq, vq, ks, vs, wide, torch.where(lens > L, T + 1, lens).int(), n, CROSS, max_tokens=T)
        assert st == binding.HD_DEVBIT_INDEX
        _assert_rows(o, lse, q, kv, vv, L, 0, n, CROSS, 0)
        for b in (1, 2, 3, 4):
            _assert_empty(o, lse, b)
    # pages before the window are not looked at (the first position seen is (P + 1) n - n + 1, in the second page)
    table[1, 0] = -1
    table[1, 1:] = torch.where(table[1, 1:] == kq.shape[0], table[0, 1], table[1, 1:])
    o, lse, st = _decode(q, kq, vq, ks, vs, table, _i32([L, P + 2, 0, 0, 0]), n, LOCAL, window=n)
    assert st == 0


@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", [(4, 32, 8, 128, 16), (4, 24, 2, 256, 16), (2, 8, 4, 64, 8), (4, 96, 8, 128, 3)])
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (LOCAL, 30)])
def test_hidden_nan_has_no_effect(n, Hq, Hkv, Dh, P, mode, w):
    """NaN in K and V rows that some query rows see and others do not: the rows that see one are NaN, the others right."""
    L = 70
    q, kc, vc = _case(2, L, n, Hq, Hkv, Dh, 9)
    at = (L - 20) * n + 1  # stream 1
    lens = _i32([L, L])
    for where, x in (("v", vc), ("k", kc)):
        x[0, at, 0, 3] = float("nan")
        kq, ks, table, kv = q8.quantised(kc, lens, P, 1, n, 0)
        vq, vs, _, vv = q8.quantised(vc, lens, P, 1, n, 0)
        o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, mode, w)
        assert st == 0
        _assert_rows(o, lse, q, kv, vv, L, 1, n, mode, w)
        x[0, at, 0, 3] = 0.0
        kv[0, at, 0, 3] = vv[0, at, 0, 3] = 0.0
        o_r, lse_r, _ = oracle.decode(q[:1], kv[:1], vv[:1], _i32([L]), n, mode, window=w)
        for s in range(n):
            pq = (L - 1) * n + s
            sees = at % n == s if mode == WITHIN else at > pq - w
            for h in range(Hq):
                if h < Hq // Hkv and sees:
                    got = o[0, s, h] if where == "k" else o[0, s, h, 3:4]
                    assert bool(torch.isnan(got).all()), (s, h)
                else:
                    assert float((o[0, s, h].double() - o_r[0, s, h]).abs().max()) <= 2e-2
                    assert abs(float(lse[0, h, s]) - float(lse_r[0, h, s])) <= 1e-3


@pytest.mark.parametrize("Dh", [64, 128, 256])
def test_scales_far_apart(Dh):
    """V's blocks over the whole range of scales; the largest rules O, and the softmax's sum counts them all alike."""
    n, Hq, Hkv, L, P = 2, 4, 2, 115, 4
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 5)
    vc = (vc.float() * torch.exp2((torch.arange(L * n) // n - 64.0).clamp(-60, 49))[None, :, None, None]).to(BF)
    lens = _i32([L])
    kq, ks, table, kv = q8.quantised(kc, lens, P, 1, n, 0)
    vq, vs, _, vv = q8.quantised(vc, lens, P, 1, n, 0)
    assert int(vs[vs != 255].min()) < 70 and int(vs[vs != 255].max()) > 165
    for mode, w in ((CROSS, 0), (WITHIN, 0), (LOCAL, 9)):
        o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, mode, w)
        assert st == 0
        _assert_rows(o, lse, q, kv, vv, L, 0, n, mode, w)


@pytest.mark.parametrize("size", [1e-30, 1e-4, 30.0, 3e4])
def test_sizes_of_queries_and_keys(size):
    """Queries far from 1 with keys as far on the other side, one row of zeros, one of very different magnitudes."""
    n, Hq, Hkv, Dh, L, P, T = 2, 8, 2, 128, 80, 8, 2
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 6)
    q = (q.float() * size).to(BF)
    kc = (kc.float() / max(size, 1e-15)).to(BF)
    q[0, 0, 0] = 0.0
    q[0, 1, 3, ::2] *= 2.0**-9
    lens = _i32([L])
    kq, ks, table, kv = q8.quantised(kc, lens, P, T, n, 0)
    vq, vs, _, vv = q8.quantised(vc, lens, P, T, n, 0)
    o, lse, st = _decode(q, kq, vq, ks, vs, table, lens, n, CROSS)
    assert st == 0
    _assert_rows(o, lse, q, kv, vv, L, 0, n, CROSS, 0)


def test_scale_and_no_lse():
    n, Hq, Hkv, Dh, L, P = 2, 8, 2, 128, 200, 16
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 6)
    lens = _i32([L])
    kq, ks, table, kv = q8.quantised(kc, lens, P, P, n, 0)
    vq, vs, _, vv = q8.quantised(vc, lens, P, P, n, 0)
    for scale in (0.02, 0.3):
        o, _, st = _decode(q, kq, vq, ks, vs, table, lens, n, CROSS, scale=scale, with_lse=False)
        assert st == 0
        _assert_rows(o, None, q, kv, vv, L, 0, n, CROSS, 0, scale=scale)


def test_scale_bytes_outside_their_range():
    """Bytes below 63 and above 177 are read as the nearest of these."""
    n, Hq, Hkv, Dh, L, P = 1, 2, 1, 64, 16, 4
    q, kc, vc = _case(1, L, n, Hq, Hkv, Dh, 6)
    lens = _i32([L])
    kq, ks, table, _ = q8.quantised(kc, lens, P, P, n, 0)
    vq, vs, _, _ = q8.quantised(vc, lens, P, P, n, 0)
    ks[table[0, 0].long()], vs[table[0, 1].long()], vs[table[0, 2].long()] = 0, 255, 20
    near = _decode(q, kq, vq, ks.clamp(63, 177), vs.clamp(63, 177), table, lens, n, CROSS)
    got = _decode(q, kq, vq, ks, vs, table, lens, n, CROSS)
    assert torch.equal(got[0], near[0]) and torch.equal(got[1], near[1])


def _serve(n, Hq, Hkv, Dh, P, T, steps, graph):
    """Prompts, their cache in 8 bits, a fork, single tokens: the outputs of each step and of the model."""
    B, width, pages = 3, 12, 30
    i32 = dict(dtype=I32, device="cuda")
    refs, lens, table = torch.zeros(pages, **i32), torch.zeros(B, **i32), torch.full((B, width), -1, **i32)
    st, served = torch.zeros(1, **i32), torch.zeros(B, **i32)
    k = torch.full((pages, Hkv, P * n, Dh), 0x7F, dtype=torch.uint8, device="cuda").view(F8)
    v = k.clone()
    ks, vs = (torch.full((pages, Hkv, P // T), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    wsp = torch.empty(binding.hd_pages_workspace_bytes(B, pages), dtype=torch.uint8, device="cuda")
    wsd = torch.empty(binding.sfa_decode_paged_q8_workspace_bytes(B, P * width, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8,
                      device="cuda")
    new = [29, 13, 0]
    kn, vn = inputs.normal_bf16((42 * n, Hkv, Dh), 1), inputs.normal_bf16((42 * n, Hkv, Dh), 2)
    binding.hd_pages_grow(refs, table, lens, torch.tensor(new, **i32), P, wsp, served=served, dev_status=st)
    binding.sfa_kv_append_paged_q8(kn.cuda(), vn.cuda(), k, v, ks, vs, table, lens, n, offsets=torch.tensor([0, 29, 42, 42], **i32),
                                   served=served, dev_status=st)
    copies = torch.empty(1, 2, **i32)
    binding.hd_pages_fork(refs, table, lens, torch.tensor([0], **i32), torch.tensor([2], **i32), torch.tensor([22], **i32), copies,
                          P, wsp, dev_status=st)
    binding.hd_pages_copy_q8(k, v, ks, vs, copies, dev_status=st)
    qs, kt, vt = (inputs.normal_bf16((steps, B, n, h, Dh), 5 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    q1, k1, v1 = qs[0].cuda(), kt[0].cuda(), vt[0].cuda()
    o, lse = torch.empty_like(q1), torch.empty(B, Hq, n, dtype=torch.float32, device="cuda")
    one = torch.ones(B, **i32)

    def step():
        binding.hd_pages_grow(refs, table, lens, one, P, wsp, served=served, dev_status=st)
        binding.sfa_kv_append_paged_q8(k1, v1, k, v, ks, vs, table, lens, n, served=served, dev_status=st)
        binding.sfa_decode_paged_q8(q1, k, v, ks, vs, table, lens, o, n, CROSS, wsd, lse=lse, dev_status=st)

    if graph:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    got = []
    for i in range(steps):
        q1.copy_(qs[i]), k1.copy_(kt[i]), v1.copy_(vt[i])
        g.replay() if graph else step()
        torch.cuda.synchronize()
        got.append((o.cpu(), lse.cpu()))
    assert int(st.item()) == 0
    # the same in the model, on pages of its own
    own = torch.arange(B * width).view(B, width)
    mk, mv = (q8.Cache(B * width, P, n, Hkv, Dh, T) for _ in range(2))
    for m, x in ((mk, kn), (mv, vn)):
        x = x.view(42, n, Hkv, Dh)
        m.append(x[:29], own[0], 0)
        m.append(x[29:], own[1], 0)
        m.codes[own[2]], m.e[own[2]] = m.codes[own[0]], m.e[own[0]]
    have = [29, 13, 22]
    for i in range(steps):
        for b in range(B):
            for m, x in ((mk, kt), (mv, vt)):
                m.append(x[i, b:b + 1], own[b], have[b] + i)
            L = have[b] + i + 1
            kv, vv = (m.rows(own[b], L).to(BF)[None] for m in (mk, mv))
            _assert_rows(got[i][0][b:b + 1], got[i][1][b:b + 1], qs[i, b:b + 1], kv, vv, L, 0, n, CROSS, 0)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P,T", [(4, 32, 8, 128, 8, 8), (2, 8, 2, 256, 8, 2), (3, 4, 4, 64, 5, 1), (4, 24, 2, 128, 16, 16)])
def test_a_serving_run(n, Hq, Hkv, Dh, P, T, graph):
    _serve(n, Hq, Hkv, Dh, P, T, 9, graph)


def test_two_calls_at_once_and_the_same_bits():
    """Two steps on two streams, each with its workspace; every run the same bits."""
    n, Hq, Hkv, Dh, L, P, T = 4, 32, 8, 128, 3000, 16, 16
    lens = _i32([L, 1100])
    runs = []
    for seed in (1, 2):
        q, kc, vc = _case(2, L, n, Hq, Hkv, Dh, seed)
        kq, ks, table, _ = q8.quantised(kc, lens, P, T, n, seed)
        vq, vs, _, _ = q8.quantised(vc, lens, P, T, n, seed)
        ws = torch.empty(binding.sfa_decode_paged_q8_workspace_bytes(2, L, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8, device="cuda")
        t = [x.cuda() for x in (q, kq, vq, ks, vs, table, lens)]
        runs.append((t, torch.empty_like(t[0]), ws, torch.cuda.Stream()))
    want = []
    for (t, o, ws, _) in runs:
        binding.sfa_decode_paged_q8(*t, o, n, CROSS, ws, max_tokens=L)
        torch.cuda.synchronize()
        want.append(o.clone())
    for _ in range(20):
        for (t, o, ws, s) in runs:
            o.zero_()
            s.wait_stream(torch.cuda.current_stream())
            binding.sfa_decode_paged_q8(*t, o, n, CROSS, ws, max_tokens=L, stream=s)
        torch.cuda.synchronize()
        for (t, o, _, _), w in zip(runs, want):
            assert torch.equal(o, w)


@pytest.mark.parametrize("Hq,Hkv,Dh,P,T", [(32, 8, 128, 16, 16), (16, 4, 64, 3, 1), (24, 2, 256, 20, 5)])
def test_pools_beyond_32_bits(Hq, Hkv, Dh, P, T):
    """Pages whose codes lie more than 2^32 bytes into the pool: prompt, token, read, copy and step give the bits that they
    give in a small pool."""
    n, L = 4, 100
    far = 2**32 // (P * n * Hkv * Dh) + 2
    held = -(-L // P)
    q, kn, vn = (inputs.normal_bf16((1, n, h, Dh), 1 + i).cuda() for i, h in enumerate((Hq, Hkv, Hkv)))
    kr, vr = (inputs.normal_bf16(((L - 1) * n, Hkv, Dh), 5 + i).cuda() for i in range(2))
    runs = []
    for base in (0, far):
        pages = base + held + 1
        kc, vc = (torch.empty(pages, Hkv, P * n, Dh, dtype=F8, device="cuda") for _ in range(2))
        ks, vs = (torch.empty(pages, Hkv, P // T, dtype=torch.uint8, device="cuda") for _ in range(2))
        table = (base + 1 + torch.arange(held, dtype=I32)).flip(0).view(1, held).cuda()
        lens, st = _i32([L - 1]).cuda(), torch.zeros(1, dtype=I32, device="cuda")
        binding.sfa_kv_append_paged_q8(kr, vr, kc, vc, ks, vs, table, lens, n, offsets=_i32([0, L - 1]).cuda(), dev_status=st)
        lens += 1
        binding.sfa_kv_append_paged_q8(kn, vn, kc, vc, ks, vs, table, lens, n, dev_status=st)
        binding.hd_pages_copy_q8(kc, vc, ks, vs, torch.stack([table[0, -1:], table[0, -1:] - 1], 1).contiguous(), dev_status=st)
        table[0, -1] -= 1  # the copy
        k, v = (torch.empty(L * n, Hkv, Dh, dtype=BF, device="cuda") for _ in range(2))
        binding.sfa_kv_read_paged_q8(kc, vc, ks, vs, table, lens, _i32([0, L]).cuda(), k, v, n, dev_status=st)
        ws = torch.empty(binding.sfa_decode_paged_q8_workspace_bytes(1, held * P, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8,
                         device="cuda")
        o, lse = torch.empty_like(q), torch.empty(1, Hq, n, device="cuda")
        binding.sfa_decode_paged_q8(q, kc, vc, ks, vs, table, lens, o, n, CROSS, ws, lse=lse, dev_status=st)
        assert int(st.item()) == 0
        runs.append([x.cpu() for x in (k, v, o, lse)])
    for a, b in zip(*runs):
        assert torch.equal(a.view(torch.int16 if a.dtype == BF else I32), b.view(torch.int16 if b.dtype == BF else I32))
    _assert_rows(runs[1][2], runs[1][3], q.cpu(), runs[1][0][None], runs[1][1][None], L, 0, n, CROSS, 0)
