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


# query rows per K/V head and ranges of the tensor cores, which smaller cases miss: head dim 128 from 33 rows on, 256 with
# 17 to 32 rows from 1200 positions on
TC = [(4, 24, 2, 128, 16), (4, 48, 4, 128, 7), (4, 12, 2, 256, 16), (3, 8, 1, 256, 20), (4, 8, 1, 256, 5)]


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 1500), (LOCAL, 2**31 - 1)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", TC)
def test_tensor_cores_ragged(mode, w, n, Hq, Hkv, Dh, P):
    L = 700
    assert paged_rule.tensor_cores(5, n, Hq, Hkv, Dh, P, L, min(w, L * n))
    q, kc, vc = _case(5, L, n, Hq, Hkv, Dh, 80 + n + Hq)
    _check(q, kc, vc, _i32([L, 1, 0, 401, 33]), n, mode, w, P, seed=4)


@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", TC)
@pytest.mark.parametrize("entry", [-1, 2**31 - 1, None])  # None: one past the pool
def test_tensor_cores_bad_pages(n, Hq, Hkv, Dh, P, entry):
    L = 700
    width = -(-L // P)
    assert paged_rule.tensor_cores(3, n, Hq, Hkv, Dh, P, L)
    q, kc, vc = _case(3, L, n, Hq, Hkv, Dh, 11)
    lens = _i32([L, 500, L])
    kp, table = paging.to_pages(kc, lens, P, n, 1, width=width)
    vp, _ = paging.to_pages(vc, lens, P, n, 1, width=width)
    bad = kp.shape[0] if entry is None else entry
    table[1, -(-500 // P):] = bad  # behind the sequence's pages: not looked at
    table[2, width // 2] = bad
    o, lse, st = _decode(q, kp, vp, table, lens, n, CROSS, max_tokens=L)
    assert st == binding.HD_DEVBIT_INDEX
    _assert_empty(o, lse, 2)
    for b in (0, 1):
        _assert_rows(o, lse, q, kc, vc, int(lens[b]), b, n, CROSS, 0)


@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", TC)
def test_tensor_cores_need_only_the_windows_pages(n, Hq, Hkv, Dh, P):
    T, w = 700, 1501
    assert paged_rule.tensor_cores(1, n, Hq, Hkv, Dh, P, T, w)
    first = ((T - 1) * n - w + 1) // n  # the token at which the first row's window begins
    q, kc, vc = _case(1, T, n, Hq, Hkv, Dh, 21)
    kp, table = paging.to_pages(kc, _i32([T]), P, n, 3)
    vp, _ = paging.to_pages(vc, _i32([T]), P, n, 3)
    table[0, :first // P] = -1
    o, lse, st = _decode(q, kp, vp, table, _i32([T]), n, LOCAL, w, max_tokens=T)
    assert st == 0
    _assert_rows(o, lse, q, kc, vc, T, 0, n, LOCAL, w)


@pytest.mark.parametrize("bad", [NAN, float("inf"), 3.38e38])
@pytest.mark.parametrize("n,Hq,Hkv,Dh,P", TC)
@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 1400)])
def test_tensor_cores_hidden_values(mode, w, n, Hq, Hkv, Dh, P, bad):
    # cached rows that stream 0's new position does not see, as in test_paged_gpu, over a range for the tensor cores
    T = 600
    assert paged_rule.tensor_cores(1, n, Hq, Hkv, Dh, P, T, w)
    q, kc, vc = _case(1, T, n, Hq, Hkv, Dh, 31)
    hidden = {WITHIN: [5 * n + 1, 590 * n + 1, (T - 1) * n + 1], CROSS: [(T - 1) * n + 1, (T - 1) * n + 2],
              LOCAL: [0, (T - 1) * n - w, (T - 1) * n - w - 30]}[mode]
    kb, vb = kc.clone(), vc.clone()
    kb[0, hidden, :, 3] = bad
    vb[0, hidden, :, 5] = bad
    kp, table = paging.to_pages(kb, _i32([T]), P, n, 4)
    vp, _ = paging.to_pages(vb, _i32([T]), P, n, 4)
    o, lse, st = _decode(q, kp, vp, table, _i32([T]), n, mode, w, max_tokens=T)
    assert st == 0
    o_r, lse_r, _ = oracle.decode(q, kc, vc, _i32([T]), n, mode, window=w)
    A, _, _ = oracle.decode(q, kc, vc.abs(), _i32([T]), n, mode, window=w)
    for s in [0] if mode != LOCAL else range(n):
        err = (o[0, s].double() - o_r[0, s]).abs()
        assert bool((err <= (2.0**-8 + 1e-3) * (A[0, s] + o_r[0, s].abs())).all())
        assert float((lse[0, :, s].double() - lse_r[0, :, s]).abs().max()) <= 1e-3


# one and several splits of both kernels, every head dim
FORMS = [(4, 32, 8, 128, 16, 60), (4, 32, 8, 128, 16, 700), (8, 32, 8, 128, 2, 300), (4, 24, 2, 128, 16, 700), (2, 4, 4, 64, 8, 500),
         (4, 24, 2, 256, 16, 700), (1, 4, 1, 256, 3, 40)]


@pytest.mark.parametrize("n,Hq,Hkv,Dh,P,T", FORMS)
def test_scales_and_no_lse(n, Hq, Hkv, Dh, P, T):
    # a scale of up to twice the usual one: scores are off by at most twice as much as derived, 3.2e-4 of the 1e-3
    q, kc, vc = _case(2, T, n, Hq, Hkv, Dh, 91)
    lens = _i32([T, T // 2 + 1])
    kp, table = paging.to_pages(kc, lens, P, n, 4)
    vp, _ = paging.to_pages(vc, lens, P, n, 4)
    dev = [x.cuda() for x in (q, kp, vp, table, lens)]
    ws = guards.empty((binding.sfa_decode_paged_workspace_bytes(2, T, n, Hq, Hkv, Dh, CROSS),), torch.uint8, 0xFF)
    for scale in (0.3 * Dh**-0.5, 1.9 * Dh**-0.5):
        o, lse = guards.empty(q.shape, torch.bfloat16, 7.0), guards.empty((2, Hq, n), torch.float32, 7.0)
        binding.sfa_decode_paged(*dev, o, n, CROSS, ws, max_tokens=T, lse=lse, softmax_scale=scale)
        o_r, lse_r, _ = oracle.decode(q, kc, vc, lens, n, CROSS, scale=scale)
        A, _, _ = oracle.decode(q, kc, vc.abs(), lens, n, CROSS, scale=scale)
        err = (o.cpu().double() - o_r).abs()
        assert bool((err <= (2.0**-8 + 1e-3) * (A + o_r.abs())).all())
        assert float((lse.cpu().double() - lse_r).abs().max()) <= 1e-3
        only = guards.empty(q.shape, torch.bfloat16, 7.0)
        binding.sfa_decode_paged(*dev, only, n, CROSS, ws, max_tokens=T, softmax_scale=scale)
        assert torch.equal(only.view(torch.int16), o.view(torch.int16))


@pytest.mark.parametrize("n,Hq,Hkv,Dh,P,T", FORMS)
def test_two_steps_at_once(n, Hq, Hkv, Dh, P, T):
    # two streams, a workspace each
    q, kc, vc = _case(2, T, n, Hq, Hkv, Dh, 93)
    lens = _i32([T, 1])
    kp, table = paging.to_pages(kc, lens, P, n, 4)
    vp, _ = paging.to_pages(vc, lens, P, n, 4)
    dev = [x.cuda() for x in (q, kp, vp, table, lens)]
    want = _decode(q, kp, vp, table, lens, n, CROSS, max_tokens=T)
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[guards.empty(q.shape, torch.bfloat16, 7.0) for _ in range(5)] for _ in streams]
    ws = [guards.empty((binding.sfa_decode_paged_workspace_bytes(2, T, n, Hq, Hkv, Dh, CROSS),), torch.uint8, 0xFF)
          for _ in streams]
    torch.cuda.synchronize()
    for i in range(5):
        for st, w, o in zip(streams, ws, out):
            binding.sfa_decode_paged(*dev, o[i], n, CROSS, w, max_tokens=T, stream=st)
    torch.cuda.synchronize()
    for o in out:
        for x in o:
            assert torch.equal(x.cpu().view(torch.int16), want[0].view(torch.int16))
