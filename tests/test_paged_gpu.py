"""Paged cache on the GPU: decoding over pages and appends into them, against the 64-bit oracle on the
contiguous cache, and the calls that the header refuses or leaves out.

Tolerance of O, element by element: P is rounded to bf16 for its product (off by at most half a step,
2^-8 relative), and so is O, so |dO| <= 2^-8 (A + |O|), A = sum P |V|; 1e-3 (A + |O|) on top covers the
fp32 sums of up to 2^17 terms and exp2 of scores that are off by Dh * 2^-24 * sum |q k| * scale (1.6e-4
at Dh = 256 and N(0, 1) operands, so P is off by as much, relative).  LSE: 1e-3, the same scores' error
with a margin of 5.  Appends are bit copies."""
import pytest
import torch

import guards
import oracle
import paging
from paper_2607_08186_gb300 import binding, build, inputs

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
NAN = float("nan")
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=I32)


def _case(B, Lcap, n, Hq, Hkv, Dh, seed):
    return (inputs.normal_bf16((B, n, Hq, Dh), seed), inputs.normal_bf16((B, Lcap * n, Hkv, Dh), seed + 1),
            inputs.normal_bf16((B, Lcap * n, Hkv, Dh), seed + 2))


def _decode(q, kp, vp, table, lens, n, mode, window=0, max_tokens=None):
    """(o, lse, status) of one call, on the host."""
    B, _, Hq, Dh = q.shape
    T = max_tokens or table.shape[1] * (kp.shape[1] // n)
    ws = guards.empty((binding.sfa_decode_paged_workspace_bytes(B, T, n, Hq, kp.shape[2], Dh, mode, window),), torch.uint8,
                      0xFF, what="workspace")
    o, lse = guards.empty(q.shape, torch.bfloat16, 7.0), guards.empty((B, Hq, n), torch.float32, 7.0)
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.sfa_decode_paged(q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), lens.cuda(), o, n, mode, ws, max_tokens=T,
                             lse=lse, window=window, dev_status=st)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu(), int(st.item())


def _assert_rows(o, lse, q, kc, vc, T, b, n, mode, window):
    """Sequence b's rows against the oracle on its contiguous cache."""
    a = (q[b:b + 1], kc[b:b + 1], vc[b:b + 1], _i32([T]), n, mode)
    o_r, lse_r, bad = oracle.decode(*a, window=window)
    A, _, _ = oracle.decode(a[0], a[1], a[2].abs(), *a[3:], window=window)
    assert bad == 0
    err = (o[b].double() - o_r[0]).abs()
    assert bool((err <= (2.0**-8 + 1e-3) * (A[0] + o_r[0].abs())).all()), float((err / (A[0] + o_r[0].abs())).max())
    assert float((lse[b].double() - lse_r[0]).abs().max()) <= 1e-3


def _assert_empty(o, lse, b):
    assert torch.count_nonzero(o[b]) == 0 and bool((lse[b] == -float("inf")).all())


def _check(q, kc, vc, lens, n, mode, window, P, seed=0, max_tokens=None, width=None):
    kp, table = paging.to_pages(kc, lens, P, n, seed, width=width)
    vp, _ = paging.to_pages(vc, lens, P, n, seed, width=width)
    o, lse, st = _decode(q, kp, vp, table, lens, n, mode, window, max_tokens)
    assert st == 0
    for b, T in enumerate(lens.tolist()):
        _assert_empty(o, lse, b) if T == 0 else _assert_rows(o, lse, q, kc, vc, T, b, n, mode, window)


MASKS = [(WITHIN, 0), (CROSS, 0), (LOCAL, 1), (LOCAL, 100), (LOCAL, 2**31 - 1)]


# rows per K/V head: 16 and 32 (one and two m16 tiles), 9, 48, 64 and 128 (on the tensor-core kernel from
# pages of eight rows on, else two row groups); pages of every
# size against tiles of 64 rows: smaller, equal, larger, odd, prime, one token with more streams than a tile holds
@pytest.mark.parametrize("mode,w", MASKS)
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", [(4, 32, 8, 128, 16), (8, 32, 8, 128, 3), (8, 64, 8, 128, 1), (1, 8, 8, 128, 64),
                                           (3, 6, 2, 128, 7), (2, 4, 4, 64, 8), (3, 16, 4, 64, 50), (4, 8, 2, 64, 5),
                                           (1, 8, 2, 128, 131), (4, 8, 2, 128, 43), (4, 32, 8, 128, 2), (70, 2, 1, 64, 1), (5, 10, 2, 64, 9),
                                           (4, 96, 8, 128, 16), (8, 32, 2, 128, 3), (3, 96, 8, 128, 1), (4, 12, 1, 128, 43)])
def test_ragged(mode, w, n, Hq, Hkv, Dh, P):
    q, kc, vc = _case(4, 150, n, Hq, Hkv, Dh, n + Hq + P)
    _check(q, kc, vc, _i32([150, 1, 0, 129]), n, mode, w, P)


# head dim 256: 24 to 128 query rows on the tensor-core kernel where pages are not too small, up to 16 and 256
# of them on the other one, by TMA and by cp.async
@pytest.mark.parametrize("mode,w", MASKS)
@pytest.mark.parametrize("n,Hq,Hkv,P", [(4, 24, 2, 16), (1, 4, 1, 3), (3, 6, 2, 5), (8, 32, 2, 4), (4, 24, 2, 32),
                                        (4, 24, 2, 64), (2, 12, 2, 1), (8, 64, 2, 6), (8, 64, 2, 1), (3, 24, 2, 43), (4, 24, 2, 43), (1, 12, 1, 131), (1, 4, 1, 1),
                                        (4, 16, 2, 3), (3, 16, 2, 4), (4, 16, 2, 2), (1, 24, 1, 16), (4, 8, 2, 16), (3, 10, 2, 11)])
def test_ragged_head_dim_256(mode, w, n, Hq, Hkv, P):
    q, kc, vc = _case(4, 150, n, Hq, Hkv, 256, 40 + n + Hq + P)
    _check(q, kc, vc, _i32([150, 1, 0, 129]), n, mode, w, P)


@pytest.mark.parametrize("n,Hq,Hkv,Dh,mode,P", [(4, 32, 8, 128, WITHIN, 16), (4, 32, 8, 128, CROSS, 37),
                                                (4, 24, 2, 256, WITHIN, 16), (4, 24, 2, 256, CROSS, 24),
                                                (4, 96, 8, 128, CROSS, 32), (4, 16, 2, 256, CROSS, 3),
                                                (3, 16, 2, 256, WITHIN, 5), (4, 16, 2, 256, WITHIN, 2)])
def test_long(n, Hq, Hkv, Dh, mode, P):
    q, kc, vc = _case(2, 8192, n, Hq, Hkv, Dh, 8)
    _check(q, kc, vc, _i32([8192, 3001]), n, mode, 0, P)


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 2000)])
@pytest.mark.parametrize("B,Hq,Hkv,Dh,P", [(3, 8, 2, 128, 16), (33, 4, 1, 128, 7), (70, 2, 2, 64, 16), (7, 24, 2, 256, 16),
                                           (40, 2, 1, 256, 20), (40, 8, 1, 256, 20), (9, 12, 1, 128, 16)])
def test_splits_shared_out_by_length(mode, w, B, Hq, Hkv, Dh, P):
    # long splits of sequences of very different lengths, empty ones, one beyond max_tokens and one below
    # zero among them (these three alone are empty); more sequences than a warp has lanes
    n, L = 4, 1500
    lens = [max(0, int(L * (0.618 * b % 1.0)) - 60) for b in range(B)]
    lens[0] = L
    if B > 10:
        lens[5], lens[B - 1] = -7, L + 1
    q, kc, vc = _case(B, L, n, Hq, Hkv, Dh, B)
    held = [x if 0 <= x <= L else 0 for x in lens]
    kp, table = paging.to_pages(kc, held, P, n, 1, width=-(-L // P))
    vp, _ = paging.to_pages(vc, held, P, n, 1, width=-(-L // P))
    o, lse, st = _decode(q, kp, vp, table, _i32(lens), n, mode, w, max_tokens=L)
    assert st == (binding.HD_DEVBIT_INDEX if B > 10 else 0)
    for b, T in enumerate(held):
        _assert_empty(o, lse, b) if T == 0 else _assert_rows(o, lse, q, kc, vc, T, b, n, mode, w)


@pytest.mark.parametrize("Dh", [64, 128, 256])
def test_max_tokens_and_wide_tables(Dh):
    # a table with more entries than the longest sequence needs, and a bound above it
    q, kc, vc = _case(2, 90, 4, 8, 2, Dh, 5)
    _check(q, kc, vc, _i32([90, 77]), 4, CROSS, 0, 8, max_tokens=100, width=40)


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 70)])
@pytest.mark.parametrize("Hq,Hkv,Dh,P", [(32, 8, 128, 16), (4, 4, 64, 5), (24, 2, 256, 20)])
def test_where_pages_lie_changes_no_bit(mode, w, Hq, Hkv, Dh, P):
    n = 4
    q, kc, vc = _case(3, 200, n, Hq, Hkv, Dh, 3)
    lens = _i32([200, 33, 121])
    runs = []
    for seed in (1, 2):
        kp, table = paging.to_pages(kc, lens, P, n, seed)
        vp, _ = paging.to_pages(vc, lens, P, n, seed)
        runs.append(_decode(q, kp, vp, table, lens, n, mode, w))
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1]) and runs[0][2] == 0


@pytest.mark.parametrize("Hq,Hkv,Dh", [(8, 2, 128), (24, 2, 256), (8, 2, 256)])
@pytest.mark.parametrize("entry", [-1, -2**31, 2**31 - 1, None])  # None: one past the pool
def test_bad_pages_empty_the_sequence_alone(Hq, Hkv, Dh, entry):
    n, P = 4, 16
    q, kc, vc = _case(3, 700, n, Hq, Hkv, Dh, 11)
    lens = _i32([700, 500, 700])
    kp, table = paging.to_pages(kc, lens, P, n, 1, width=60)
    vp, _ = paging.to_pages(vc, lens, P, n, 1, width=60)
    bad = kp.shape[0] if entry is None else entry
    table[1, 32:] = bad  # behind the sequence's pages: not looked at
    table[2, 20] = bad
    o, lse, st = _decode(q, kp, vp, table, lens, n, CROSS)
    assert st == binding.HD_DEVBIT_INDEX
    _assert_empty(o, lse, 2)
    for b in (0, 1):
        _assert_rows(o, lse, q, kc, vc, int(lens[b]), b, n, CROSS, 0)


def test_bad_lengths_empty_the_sequence_alone():
    q, kc, vc = _case(4, 48, 2, 4, 2, 128, 6)
    kp, table = paging.to_pages(kc, _i32([48] * 4), 8, 2, 2)
    vp, _ = paging.to_pages(vc, _i32([48] * 4), 8, 2, 2)
    o, lse, st = _decode(q, kp, vp, table, _i32([-1, 48, 49, 0]), 2, CROSS)
    assert st == binding.HD_DEVBIT_INDEX
    for b in (0, 2, 3):
        _assert_empty(o, lse, b)
    _assert_rows(o, lse, q, kc, vc, 48, 1, 2, CROSS, 0)


@pytest.mark.parametrize("Hq,Hkv,Dh,P", [(8, 2, 128, 16), (24, 2, 128, 16), (24, 2, 256, 16), (24, 2, 256, 5), (8, 2, 256, 16),
                                           (4, 2, 64, 1)])
@pytest.mark.parametrize("w", [150, 500])  # a range for the mma.sync kernel, and for the tensor cores
def test_local_needs_only_the_windows_pages(Hq, Hkv, Dh, P, w):
    n, T = 4, 333
    first = ((T - 1) * n - w + 1) // n  # the token at which the first row's window begins
    q, kc, vc = _case(1, T, n, Hq, Hkv, Dh, 21)
    kp, table = paging.to_pages(kc, _i32([T]), P, n, 3)
    vp, _ = paging.to_pages(vc, _i32([T]), P, n, 3)
    table[0, :first // P] = -1
    o, lse, st = _decode(q, kp, vp, table, _i32([T]), n, LOCAL, w)
    assert st == 0
    _assert_rows(o, lse, q, kc, vc, T, 0, n, LOCAL, w)


@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf"), 3.38e38])
@pytest.mark.parametrize("Hq,Hkv,Dh", [(8, 2, 128), (24, 2, 128), (24, 2, 256), (8, 2, 256), (4, 2, 64)])
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 90), (LOCAL, 600)])
def test_what_the_mask_hides_has_no_effect(mode, w, Hq, Hkv, Dh, bad):
    # cached rows that stream 0's new position does not see hold infinities, NaN or huge values: those of
    # another stream (WITHIN), the new token's later positions (CROSS), what lies before the window (LOCAL)
    n, T = 4, 300
    q, kc, vc = _case(1, T, n, Hq, Hkv, Dh, 31)
    hidden = {WITHIN: [5 * n + 1, 290 * n + 1, (T - 1) * n + 1], CROSS: [(T - 1) * n + 1, (T - 1) * n + 3],
              LOCAL: [0, (T - 1) * n - w, (T - 1) * n - w - 30]}[mode]
    kb, vb = kc.clone(), vc.clone()
    kb[0, hidden, :, 3] = bad
    vb[0, hidden, :, 5] = bad
    kp, table = paging.to_pages(kb, _i32([T]), 16, n, 4)
    vp, _ = paging.to_pages(vb, _i32([T]), 16, n, 4)
    o, lse, st = _decode(q, kp, vp, table, _i32([T]), n, mode, w)
    assert st == 0
    o_r, lse_r, _ = oracle.decode(q, kc, vc, _i32([T]), n, mode, window=w)
    A, _, _ = oracle.decode(q, kc, vc.abs(), _i32([T]), n, mode, window=w)
    rows = [0] if mode != LOCAL else range(n)
    for s in rows:
        err = (o[0, s].double() - o_r[0, s]).abs()
        assert bool((err <= (2.0**-8 + 1e-3) * (A[0, s] + o_r[0, s].abs())).all())
        assert float((lse[0, :, s].double() - lse_r[0, :, s]).abs().max()) <= 1e-3
    if mode == WITHIN and bad != bad:  # and those that see it are not finite
        assert not bool(torch.isfinite(o[0, 1, :, 5].float()).any())


@pytest.mark.parametrize("Hq,Hkv,Dh", [(8, 2, 128), (24, 2, 256), (8, 2, 256)])
def test_nan_query_is_its_own(Hq, Hkv, Dh):
    q, kc, vc = _case(1, 400, 4, Hq, Hkv, Dh, 33)
    qn = q.clone()
    qn[0, 2, 1, 7] = NAN
    kp, table = paging.to_pages(kc, _i32([400]), 16, 4, 4)
    vp, _ = paging.to_pages(vc, _i32([400]), 16, 4, 4)
    o, lse, _ = _decode(qn, kp, vp, table, _i32([400]), 4, CROSS)
    assert bool(o[0, 2, 1].isnan().all()) and bool(lse[0, 1, 2].isnan())
    o2, lse2, _ = _decode(q, kp, vp, table, _i32([400]), 4, CROSS)
    keep = torch.ones(4, Hq, dtype=torch.bool)
    keep[2, 1] = False
    assert torch.equal(o[0][keep], o2[0][keep]) and torch.equal(lse[0].t()[keep], lse2[0].t()[keep])


@pytest.mark.parametrize("Hq,Hkv,Dh", [(16, 8, 128), (8, 4, 256), (24, 4, 256)])
def test_pools_beyond_32_bits(Hq, Hkv, Dh):
    # pages whose rows start more than 2^32 elements into the pool (8.6 GB each)
    n, P, T = 4, 16, 100
    row = Hkv * Dh
    pages = 2**32 // (P * n * row) + 8
    q, kc, vc = _case(1, T, n, Hq, Hkv, Dh, 51)
    kp, vp = (torch.empty(pages, P * n, Hkv, Dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(pages - 7, pages, dtype=I32).flip(0).view(1, 7)
    ks, vs = inputs.normal_bf16((1, n, Hkv, Dh), 1), inputs.normal_bf16((1, n, Hkv, Dh), 2)
    kc[0, -n:], vc[0, -n:] = ks[0], vs[0]
    for pool, c in ((kp, kc), (vp, vc)):
        for i in range(7):
            part = c[0, i * P * n:min((i + 1) * P, T - 1) * n]
            pool[int(table[0, i]), :part.shape[0]] = part.cuda()
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.sfa_kv_append_paged(ks.cuda(), vs.cuda(), kp, vp, table.cuda(), _i32([T]).cuda(), n, dev_status=st)
    ws = torch.empty(binding.sfa_decode_paged_workspace_bytes(1, 112, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q, device="cuda"), torch.empty(1, Hq, n, device="cuda")
    binding.sfa_decode_paged(q.cuda(), kp, vp, table.cuda(), _i32([T]).cuda(), o, n, CROSS, ws, lse=lse, dev_status=st)
    assert int(st.item()) == 0
    _assert_rows(o.cpu(), lse.cpu(), q, kc, vc, T, 0, n, CROSS, 0)


@pytest.mark.parametrize("Hq,Hkv,Dh", [(32, 8, 128), (24, 2, 256)])
def test_graph_and_other_stream_give_the_same_bits(Hq, Hkv, Dh):
    n, P = 4, 16
    q, kc, vc = _case(3, 500, n, Hq, Hkv, Dh, 61)
    lens = _i32([500, 0, 311])
    kp, table = paging.to_pages(kc, lens, P, n, 5)
    vp, _ = paging.to_pages(vc, lens, P, n, 5)
    want = _decode(q, kp, vp, table, lens, n, CROSS)
    dev = [x.cuda() for x in (q, kp, vp, table, lens)]
    ws = torch.empty(binding.sfa_decode_paged_workspace_bytes(3, table.shape[1] * P, n, Hq, Hkv, Dh, CROSS), dtype=torch.uint8,
                     device="cuda")
    o, lse = torch.empty_like(dev[0]), torch.empty(3, Hq, n, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.sfa_decode_paged(*dev, o, n, CROSS, ws, lse=lse, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.sfa_decode_paged(*dev, o, n, CROSS, ws, lse=lse)
    # the captured step follows its buffers: other lengths, other queries
    lens2 = _i32([17, 256, 500])
    kp2, table2 = paging.to_pages(kc, lens2, P, n, 6, spare=kp.shape[0] - sum(-(-int(x) // P) for x in lens2), width=table.shape[1])
    vp2, _ = paging.to_pages(vc, lens2, P, n, 6, spare=kp.shape[0] - sum(-(-int(x) // P) for x in lens2), width=table.shape[1])
    for x, y in zip(dev, (q.flip(0), kp2, vp2, table2, lens2)):
        x.copy_(y)
    for _ in range(3):
        o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        want = _decode(q.flip(0).contiguous(), kp2, vp2, table2, lens2, n, CROSS)
        assert torch.equal(o.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


# ------------------------------------------------------------------ append

def _append(kn, vn, kp, vp, table, lens, n, offsets=None):
    k, v = guards.like(kp.cuda()), guards.like(vp.cuda())
    k.copy_(kp), v.copy_(vp)
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.sfa_kv_append_paged(kn.cuda(), vn.cuda(), k, v, table.cuda(), lens.cuda(), n,
                                offsets=None if offsets is None else offsets.cuda(), dev_status=st)
    torch.cuda.synchronize()
    return k.cpu(), v.cpu(), int(st.item())


def _bits(x):
    return x.contiguous().view(torch.int16)


def _put(pool, rows, table, b, t, n):
    P = pool.shape[1] // n
    pool[int(table[b, t // P]), t % P * n:(t % P + 1) * n] = rows


@pytest.mark.parametrize("n,Hkv,Dh,P", [(4, 8, 128, 16), (1, 1, 8, 1), (3, 2, 64, 7), (2, 2, 256, 3), (8, 8, 128, 2)])
def test_append_one_token_each(n, Hkv, Dh, P):
    lens = [1, 0, 40, P, P + 1, 33]
    B = len(lens)
    kp, table = paging.to_pages(torch.zeros(B, 40 * n, Hkv, Dh, dtype=torch.bfloat16), lens, P, n, 7)
    vp = kp.clone()
    kn, vn = inputs.normal_bf16((B, n, Hkv, Dh), 1), inputs.normal_bf16((B, n, Hkv, Dh), 2)
    k, v, st = _append(kn, vn, kp, vp, table, _i32(lens), n)
    for b, T in enumerate(lens):
        if T:
            _put(kp, kn[b], table, b, T - 1, n)
            _put(vp, vn[b], table, b, T - 1, n)
    assert st == 0 and torch.equal(_bits(k), _bits(kp)) and torch.equal(_bits(v), _bits(vp))


@pytest.mark.parametrize("n,Hkv,Dh,P,B", [(4, 8, 128, 16, 7), (3, 2, 64, 7, 33), (1, 4, 256, 5, 70), (2, 1, 64, 1, 1100)])
def test_append_packed_prompts(n, Hkv, Dh, P, B):
    # sequences with no, one, some and only new tokens; rows before the first and behind the last one
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 60, (B,), generator=g).tolist()
    lens[0] = 60
    new = [0 if b % 5 == 3 else x if b % 2 == 0 else min(1, x) if b % 3 == 0 else x // 2 for b, x in enumerate(lens)]
    off = [2]
    for x in new:
        off.append(off[-1] + x)
    N = off[-1] + 3
    kp, table = paging.to_pages(torch.zeros(B, 60 * n, Hkv, Dh, dtype=torch.bfloat16), lens, P, n, 8)
    vp = kp.clone()
    kn, vn = inputs.normal_bf16((N * n, Hkv, Dh), 1), inputs.normal_bf16((N * n, Hkv, Dh), 2)
    k, v, st = _append(kn, vn, kp, vp, table, _i32(lens), n, _i32(off))
    for b, T in enumerate(lens):
        for i in range(new[b]):
            _put(kp, kn[(off[b] + i) * n:(off[b] + i + 1) * n], table, b, T - new[b] + i, n)
            _put(vp, vn[(off[b] + i) * n:(off[b] + i + 1) * n], table, b, T - new[b] + i, n)
    assert st == 0 and torch.equal(_bits(k), _bits(kp)) and torch.equal(_bits(v), _bits(vp))


def test_append_leaves_out_what_it_cannot_place():
    n, Hkv, Dh, P = 2, 2, 64, 4
    kp, table = paging.to_pages(torch.zeros(4, 16 * n, Hkv, Dh, dtype=torch.bfloat16), [16] * 4, P, n, 9, fill=1.0)
    table[1, 3], table[2, 3] = -1, kp.shape[0]
    kn = inputs.normal_bf16((4, n, Hkv, Dh), 1)
    k, _, st = _append(kn, kn, kp, kp, table, _i32([16, 16, 14, 17]), n)  # 17: beyond the table
    want = kp.clone()
    _put(want, kn[0], table, 0, 15, n)
    assert st == binding.HD_DEVBIT_INDEX and torch.equal(_bits(k), _bits(want))
    # packed: a page that is not there takes its own rows only
    rows = inputs.normal_bf16((6 * n, Hkv, Dh), 3)
    k, _, st = _append(rows, rows, kp, kp, table, _i32([2, 16, 2, 2]), n, _i32([0, 0, 6, 6, 6]))
    want = kp.clone()
    for i in (0, 1):
        _put(want, rows[i * n:(i + 1) * n], table, 1, 10 + i, n)
    assert st == binding.HD_DEVBIT_INDEX and torch.equal(_bits(k), _bits(want))


@pytest.mark.parametrize("off", [[0, 4, 2, 6, 8], [-3, 2, 4, 6, 8], [0, 2, 4, 6, 99], [0, 8, 8, 8, 8], [5, 4, 3, 2, 1],
                                 [2**31 - 1] * 5, [-2**31, 0, 0, 2**31 - 1, 8]])
def test_append_bad_offsets_are_reported(off):
    # the rows of a sequence whose offsets make no sense stay unwritten; no row of the pool beyond the
    # sequences' own pages changes
    n, Hkv, Dh, P = 2, 2, 64, 4
    lens = [3, 7, 7, 7]
    kp, table = paging.to_pages(torch.zeros(4, 8 * n, Hkv, Dh, dtype=torch.bfloat16), lens, P, n, 9, fill=1.0)
    rows = inputs.normal_bf16((8 * n, Hkv, Dh), 3)
    k, _, st = _append(rows, rows, kp, kp, table, _i32(lens), n, _i32(off))
    assert st == binding.HD_DEVBIT_INDEX
    held = set(table[table >= 0].tolist())
    for p in range(kp.shape[0]):
        if p not in held:
            assert torch.equal(_bits(k[p]), _bits(kp[p]))
