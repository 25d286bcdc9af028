"""Attention over packed prompts on the GPU against the 64-bit oracle, sequence by sequence, and what the
header says of rows outside the sequences, bad offsets and values that a mask hides.

Tolerances as derived in test_paged_gpu.py: |dO| <= (2^-8 + 1e-3) (A + |O|) with A = sum P |V|, LSE 1e-3."""
import pytest
import torch

import guards
import oracle
from paper_2607_08186_gb300 import binding, build, inputs

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
NAN, INF = float("nan"), float("inf")
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _case(lens, n, Hq, Hkv, Dh, seed, before=0, behind=0):
    """q, k, v of the packed sequences with NaN rows around them, and the offsets."""
    off = [before]
    for x in lens:
        off.append(off[-1] + x)
    N = off[-1] + behind
    q, k, v = (inputs.normal_bf16((N * n, h, Dh), seed + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    for x in (q, k, v):
        x[:before * n] = NAN
        x[off[-1] * n:] = NAN
    return q, k, v, off


def _run(q, k, v, off, n, mode, window=0, stream=None):
    """(o, lse, status) on the host; o and lse start as 7."""
    rows, Hq, Dh = q.shape
    B, N = len(off) - 1, rows // n
    ws = guards.empty((binding.sfa_fwd_packed_workspace_bytes(B, N, n, Hq, k.shape[1], Dh, mode),), torch.uint8, 0xFF)
    o, lse = guards.empty(q.shape, torch.bfloat16, 7.0), guards.empty((Hq, rows), torch.float32, 7.0)
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.sfa_fwd_packed(q.cuda(), k.cuda(), v.cuda(), o, lse, torch.tensor(off, dtype=I32, device="cuda"), n, mode, ws,
                           window=window, dev_status=st)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu(), int(st.item())


def _near(o, o_r, A, lse, lse_r, rows=slice(None)):
    err, scale = (o.double() - o_r).abs()[rows], (A + o_r.abs())[rows]
    assert bool((err <= (2.0**-8 + 1e-3) * scale).all()), float((err / scale).max())
    assert float((lse.double() - lse_r).abs()[:, rows].max()) <= 1e-3


def _reference(q, k, v, r, n, mode, window):
    a = [x[r][None] for x in (q, k, v)]
    o_r, lse_r = oracle.sfa_fwd(*a, n, mode, window=window)
    A, _ = oracle.sfa_fwd(a[0], a[1], a[2].abs(), n, mode, window=window)
    return o_r[0], A[0], lse_r[0]


def _check(q, k, v, off, n, mode, window):
    o, lse, st = _run(q, k, v, off, n, mode, window)
    assert st == 0
    for a, z in zip(off, off[1:]):
        if a < z:
            r = slice(a * n, z * n)
            o_r, A, lse_r = _reference(q, k, v, r, n, mode, window)
            _near(o[r], o_r, A, lse[:, r], lse_r)
    for r in (slice(0, off[0] * n), slice(off[-1] * n, None)):
        assert bool((o[r] == 7.0).all()) and bool((lse[:, r] == 7.0).all())


MASKS = [(WITHIN, 0), (CROSS, 0), (LOCAL, 1), (LOCAL, 150), (LOCAL, 2**31 - 1)]


# an even group of heads (a CTA's two tiles are two heads') and odd ones (two tiles of a head); lengths of no,
# one and few tokens, and around the tiles
@pytest.mark.parametrize("mode,w", MASKS)
@pytest.mark.parametrize("n,Hq,Hkv,Dh", [(4, 8, 2, 128), (3, 3, 1, 128), (1, 6, 6, 128), (2, 4, 4, 64), (3, 8, 2, 64),
                                         (4, 4, 2, 256), (2, 3, 1, 256), (1, 2, 2, 256)])
def test_ragged(mode, w, n, Hq, Hkv, Dh):
    q, k, v, off = _case([70, 0, 1, 129, 32, 0, 128, 33, 3, 127], n, Hq, Hkv, Dh, n + Hq, before=2, behind=5)
    _check(q, k, v, off, n, mode, w)


@pytest.mark.parametrize("n,Hq,Hkv,Dh", [(1, 4, 2, 64), (2, 3, 1, 128), (1, 2, 1, 256)])
def test_many_short_sequences(n, Hq, Hkv, Dh):
    # more sequences than the list's one CTA has threads
    lens = [(7 * i) % 5 for i in range(1300)]
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 3)
    _check(q, k, v, off, n, CROSS, 0)


# Short neighbours share a tile: pairs of heads, and two tiles of a head; at most 32 sequences of a tile, empty ones
# among them, lengths around the longest that shares one (48 rows), and others that interrupt
SHORT = [(1, 4, 2, 64), (3, 3, 1, 64), (4, 8, 2, 128), (1, 3, 1, 128), (2, 4, 2, 256), (4, 3, 3, 256), (1, 1, 1, 256)]


@pytest.mark.parametrize("mode,w", MASKS[:2] + [(LOCAL, 1), (LOCAL, 7), (LOCAL, 2**31 - 1)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", SHORT)
def test_short_neighbours(mode, w, n, Hq, Hkv, Dh):
    lens = [3, 0, 0, 7, 12, 11, 24, 48, 1, 49, 5, 16, 0, 47, 47, 200, 2, 9] + [1] * 70 + [0] * 40 + [2, 30, 17, 0]
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 60 + n + Hq, before=1, behind=2)
    _check(q, k, v, off, n, mode, w)


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 5)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", SHORT)
def test_short_neighbours_that_are_not_finite(mode, w, n, Hq, Hkv, Dh, bad):
    # all of one sequence, behind and before the others, and the last token of another one's K and V
    lens = [6, 9, 3, 11, 0, 8]
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 90 + n + Hq, behind=2)
    kb, vb = k.clone(), v.clone()
    r = slice(off[1] * n, off[2] * n)
    kb[r], vb[r] = bad, bad
    last = slice((off[4] - 1) * n, off[4] * n)
    kb[last], vb[last] = bad, bad
    o, lse, st = _run(q, kb, vb, off, n, mode, w)
    assert st == 0
    for i, rows in ((0, lens[0]), (2, lens[2]), (3, lens[3] - 1), (5, lens[5])):
        r, keep = slice(off[i] * n, off[i + 1] * n), slice(0, rows * n)
        o_r, A, lse_r = _reference(q, k, v, r, n, mode, w)
        _near(o[r], o_r, A, lse[:, r], lse_r, keep)


@pytest.mark.parametrize("B", [1, 3])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", [(2, 4, 2, 128), (2, 1, 1, 64), (4, 2, 1, 256)])
def test_nothing_but_empty_sequences(B, n, Hq, Hkv, Dh):
    q, k, v, off = _case([0] * B, n, Hq, Hkv, Dh, 4, before=3, behind=4)
    _check(q, k, v, off, n, CROSS, 0)


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 500)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", [(4, 8, 2, 128), (3, 4, 4, 64), (4, 6, 2, 256), (2, 4, 1, 256)])
def test_long_and_the_same_bits_as_alone(mode, w, n, Hq, Hkv, Dh):
    # a sequence's rows do not depend, to the bit, on what is packed around it
    q, k, v, off = _case([900, 333], n, Hq, Hkv, Dh, 17, behind=1)
    _check(q, k, v, off, n, mode, w)
    o, lse, _ = _run(q, k, v, off, n, mode, w)
    for a, z in zip(off, off[1:]):
        r = slice(a * n, z * n)
        o2, lse2, _ = _run(*(x[r].contiguous() for x in (q, k, v)), [0, z - a], n, mode, w)
        assert torch.equal(o[r].view(torch.int16), o2.view(torch.int16)) and torch.equal(lse[:, r], lse2)


@pytest.mark.parametrize("mode", [WITHIN, CROSS])
@pytest.mark.parametrize("Hq,Hkv,Dh", [(32, 8, 128), (24, 2, 256)])
def test_full_size_heads(mode, Hq, Hkv, Dh):
    # 8B- and 80B-class heads, sampled rows (tile edges and ends among them)
    n, lens = 4, [1500, 77, 1021]
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 23)
    o, lse, st = _run(q, k, v, off, n, mode)
    assert st == 0
    from parity import sample_rows
    for i, (a, z) in enumerate(zip(off, off[1:])):
        r = slice(a * n, z * n)
        rows = sample_rows(1, Hq, (z - a) * n, 60, i, extra_p=(0, 127, 128, 511, 512, (z - a) * n - 1))
        x = [t[r][None] for t in (q, k, v)]
        o_r, lse_r = oracle.sfa_fwd_rows(*x, n, mode, rows)
        A, _ = oracle.sfa_fwd_rows(x[0], x[1], x[2].abs(), n, mode, rows)
        got = o[r][rows[:, 2], rows[:, 1]]
        err = (got.double() - o_r).abs()
        assert bool((err <= (2.0**-8 + 1e-3) * (A + o_r.abs())).all())
        assert float((lse[:, r][rows[:, 1], rows[:, 2]].double() - lse_r).abs().max()) <= 1e-3


@pytest.mark.parametrize("off", [[0, 30, 20, 40], [-1, 10, 20, 30], [0, 10, 20, 41], [5, 4, 3, 2], [2**31 - 1] * 4,
                                 [-2**31, 0, 2**31 - 1, 40]])
@pytest.mark.parametrize("Dh", [64, 128, 256])
def test_bad_offsets_write_nothing(off, Dh):
    q, k, v, _ = _case([40], 2, 4, 2, Dh, 5)
    o, lse, st = _run(q, k, v, off, 2, CROSS)
    assert st == binding.HD_DEVBIT_INDEX and bool((o == 7.0).all()) and bool((lse == 7.0).all())


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 90)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", [(2, 4, 2, 128), (2, 1, 1, 128), (2, 4, 2, 64), (2, 4, 2, 256), (2, 1, 1, 256)])
def test_what_a_mask_hides_has_no_effect(mode, w, n, Hq, Hkv, Dh, bad):
    # one sequence's K and V rows are not finite (all of them), and in its neighbour those of one token in the
    # middle of a tile: rows before that token, rows whose window has passed it, rows of its other stream and
    # the other sequences are as if they were finite
    lens, t = [100, 40, 230, 64], 150  # token 150 of sequence 2
    q, k, v, off = _case(lens, n, Hq, Hkv, Dh, 9, behind=3)
    kb, vb = k.clone(), v.clone()
    r1 = slice(off[1] * n, off[2] * n)
    kb[r1], vb[r1] = bad, bad
    at = (off[2] + t) * n
    vb[at, :, 1] = bad
    kb[at, :, 2] = bad
    o, lse, st = _run(q, kb, vb, off, n, mode, w)
    assert st == 0
    for i in (0, 2, 3):
        r = slice(off[i] * n, off[i + 1] * n)
        o_r, A, lse_r = _reference(q, k, v, r, n, mode, w)
        p = torch.arange(lens[i] * n)
        sees = torch.zeros_like(p, dtype=torch.bool)
        if i == 2:
            sees = p >= t * n
            if mode == WITHIN:
                sees &= p % n == 0
            if mode == LOCAL:
                sees &= p - w < t * n
        _near(o[r], o_r, A, lse[:, r], lse_r, ~sees)
        if i == 2 and bad != bad:
            assert bool(o[r][sees].isnan().all()) and bool(lse[:, r][:, sees].isnan().all())


@pytest.mark.parametrize("Hq,Hkv,Dh", [(4, 2, 128), (4, 2, 256)])
def test_repeats_graphs_and_streams_give_the_same_bits(Hq, Hkv, Dh):
    n = 4
    q, k, v, off = _case([300, 0, 77, 140], n, Hq, Hkv, Dh, 41, behind=2)
    want = _run(q, k, v, off, n, CROSS)
    for _ in range(3):
        got = _run(q, k, v, off, n, CROSS)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    dev = [x.cuda() for x in (q, k, v)]
    offs = torch.tensor(off, dtype=I32, device="cuda")
    N = q.shape[0] // n
    ws = torch.empty(binding.sfa_fwd_packed_workspace_bytes(4, N, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8, device="cuda")
    o, lse = torch.full_like(dev[0], 7.0), torch.full((Hq, N * n), 7.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.sfa_fwd_packed(*dev, o, lse, offs, n, CROSS, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.sfa_fwd_packed(*dev, o, lse, offs, n, CROSS, ws)
    # the captured call follows its offsets
    for cut in (off, [0, 10, 10, 200, off[-1]], [5, 505, 506, 507, off[-1]]):
        offs.copy_(torch.tensor(cut, dtype=I32))
        dev[0][off[-1] * n:].zero_()
        o.fill_(7.0), lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want = _run(dev[0].cpu(), k, v, cut, n, CROSS)
        assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


def test_serving_run():
    # prompts prefilled and put into pages, one forked (its last page is copied), every sequence decoded
    # for some steps with pages taken as they are needed, one freed and the pool drawn together on the way:
    # each step's rows against the oracle on the plain caches
    import paging
    n, Hq, Hkv, Dh, P, pages, B, width = 4, 8, 2, 128, 8, 60, 4, 16
    cu = lambda x: torch.tensor(x, dtype=I32, device="cuda")  # noqa: E731
    st = cu([0])
    refs, lens, table = cu([0] * pages), cu([0] * B), torch.full((B, width), -1, dtype=I32, device="cuda")
    book = paging.Book(B, width, pages, P)
    kp, vp = (torch.full((pages, P * n, Hkv, Dh), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pws = torch.empty(binding.hd_pages_workspace_bytes(B, pages), dtype=torch.uint8, device="cuda")
    prompt = [61, 20, 0, 33]
    q, k, v, off = _case(prompt, n, Hq, Hkv, Dh, 77)
    o, lse, fst = _run(q, k, v, off, n, CROSS)
    assert fst == 0
    _check(q, k, v, off, n, CROSS, 0)
    binding.hd_pages_grow(refs, table, lens, cu(prompt), P, pws, dev_status=st)
    binding.sfa_kv_append_paged(k.cuda(), v.cuda(), kp, vp, table, lens, n, offsets=cu(off), dev_status=st)
    book.grow(prompt)
    plain = [[x[a * n:z * n].clone() for a, z in zip(off, off[1:])] for x in (k, v)]
    copies = torch.empty(1, 2, dtype=I32, device="cuda")
    binding.hd_pages_fork(refs, table, lens, cu([0]), cu([2]), cu([45]), copies, P, pws, dev_status=st)
    binding.hd_pages_copy(kp, vp, copies, dev_status=st)
    book.fork([0], [2], [45])
    for c in plain:
        c[2] = c[0][:45 * n].clone()
    ws = torch.empty(binding.sfa_decode_paged_workspace_bytes(B, width * P, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8,
                     device="cuda")
    moves = torch.empty(pages // 2, 2, dtype=I32, device="cuda")
    for step in range(12):
        if step == 5:
            binding.hd_pages_free(refs, table, lens, cu([1]), P, dev_status=st)
            binding.hd_pages_compact(refs, table, lens, refs, table, moves, P, pws, dev_status=st)
            binding.hd_pages_copy(kp, vp, moves, dev_status=st)
            book.free([1]), book.compact()
            plain[0][1], plain[1][1] = plain[0][1][:0], plain[1][1][:0]
        add = [int(T > 0) for T in book.lens]
        binding.hd_pages_grow(refs, table, lens, cu(add), P, pws, dev_status=st)
        book.grow(add)
        qn, kn, vn = (inputs.normal_bf16((B, n, h, Dh), 100 + 3 * step + i) for i, h in enumerate((Hq, Hkv, Hkv)))
        on, ln = torch.empty(B, n, Hq, Dh, dtype=torch.bfloat16, device="cuda"), torch.empty(B, Hq, n, device="cuda")
        binding.sfa_kv_append_paged(kn.cuda(), vn.cuda(), kp, vp, table, lens, n, dev_status=st)
        binding.sfa_decode_paged(qn.cuda(), kp, vp, table, lens, on, n, CROSS, ws, lse=ln, dev_status=st)
        assert table.tolist() == book.table and refs.tolist() == book.refs and lens.tolist() == book.lens
        for b, T in enumerate(book.lens):
            if T == 0:
                assert torch.count_nonzero(on[b]) == 0
                continue
            for c, new in zip(plain, (kn, vn)):
                c[b] = torch.cat([c[b], new[b]])
            a = (qn[b:b + 1], plain[0][b][None], plain[1][b][None], torch.tensor([T], dtype=I32), n, CROSS)
            o_r, lse_r, _ = oracle.decode(*a)
            A, _, _ = oracle.decode(a[0], a[1], a[2].abs(), *a[3:])
            err = (on[b].cpu().double() - o_r[0]).abs()
            assert bool((err <= (2.0**-8 + 1e-3) * (A[0] + o_r[0].abs())).all())
            assert float((ln[b].cpu().double() - lse_r[0]).abs().max()) <= 1e-3
    assert int(st.item()) == 0
