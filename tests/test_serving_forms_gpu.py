"""Forms of the serving calls that a user may choose: another softmax scale, an o that is aligned to 16 bytes only, a
stream of their own for appends and page calls, two packed calls at a time.  Tolerances of test_packed_gpu."""
import random

import pytest
import torch

import guards
import paging
from paper_2607_08186_gb300 import binding, build, inputs
from test_packed_gpu import I32, _case, _near, _run
from test_served_gpu import Cache
import oracle

pytestmark = pytest.mark.gpu

WITHIN, CROSS, LOCAL = inputs.WITHIN, inputs.CROSS, inputs.LOCAL
HEADS = [(2, 4, 2, 64), (3, 3, 1, 64), (4, 8, 2, 128), (1, 3, 1, 128), (2, 4, 2, 256), (1, 3, 3, 256)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _call(q, k, v, off, n, mode, o=None, window=0, ws=None, lse=None, **kw):
    rows, Hq, Dh = q.shape
    ws = ws if ws is not None else guards.empty(
        (binding.sfa_fwd_packed_workspace_bytes(len(off) - 1, rows // n, n, Hq, k.shape[1], Dh, mode),), torch.uint8, 0xFF)
    o = o if o is not None else guards.empty(q.shape, torch.bfloat16, 7.0)
    lse = lse if lse is not None else guards.empty((Hq, rows), torch.float32, 7.0)
    binding.sfa_fwd_packed(q, k, v, o, lse, off, n, mode, ws, window=window, **kw)
    return o, lse


@pytest.mark.parametrize("mode,w", [(WITHIN, 0), (CROSS, 0), (LOCAL, 60)])
@pytest.mark.parametrize("n,Hq,Hkv,Dh", HEADS)
def test_packed_scales(mode, w, n, Hq, Hkv, Dh):
    # up to twice the usual scale: scores are off by at most twice as much as derived, 3.2e-4 of the 1e-3
    q, k, v, off = _case([130, 7, 0, 300, 20], n, Hq, Hkv, Dh, 5)
    dev, offd = [x.cuda() for x in (q, k, v)], torch.tensor(off, dtype=I32, device="cuda")
    for scale in (0.3 * Dh**-0.5, 1.9 * Dh**-0.5):
        o, lse = _call(*dev, offd, n, mode, window=w, softmax_scale=scale)
        for a, z in zip(off, off[1:]):
            if a == z:
                continue
            r = slice(a * n, z * n)
            x = [t[r][None] for t in (q, k, v)]
            o_r, lse_r = oracle.sfa_fwd(*x, n, mode, scale=scale, window=w)
            A, _ = oracle.sfa_fwd(x[0], x[1], x[2].abs(), n, mode, scale=scale, window=w)
            _near(o[r].cpu(), o_r[0], A[0], lse[:, r].cpu(), lse_r[0])


@pytest.mark.parametrize("n,Hq,Hkv,Dh", HEADS)
def test_packed_o_aligned_to_16_bytes(n, Hq, Hkv, Dh):
    q, k, v, off = _case([130, 7, 0, 300, 20], n, Hq, Hkv, Dh, 6, before=1, behind=3)
    want = _run(q, k, v, off, n, CROSS)
    raw = guards.empty((q.numel() + 16,), torch.bfloat16, 7.0)
    o = raw[8:8 + q.numel()].view(q.shape)
    assert o.data_ptr() % 32 == 16
    _, lse = _call(*(x.cuda() for x in (q, k, v)), torch.tensor(off, dtype=I32, device="cuda"), n, CROSS, o=o)
    assert torch.equal(o.cpu().view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse.cpu(), want[1])
    assert bool((raw[:8] == 7.0).all()) and bool((raw[8 + q.numel():] == 7.0).all())


@pytest.mark.parametrize("n,Hq,Hkv,Dh", HEADS)
def test_two_packed_calls_at_once(n, Hq, Hkv, Dh):
    q, k, v, off = _case([130, 7, 0, 300, 20] * 6, n, Hq, Hkv, Dh, 8)
    want = _run(q, k, v, off, n, CROSS)
    dev, offd = [x.cuda() for x in (q, k, v)], torch.tensor(off, dtype=I32, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = [[guards.empty((binding.sfa_fwd_packed_workspace_bytes(len(off) - 1, off[-1], n, Hq, Hkv, Dh, CROSS),), torch.uint8, 0xFF),
             [(guards.empty(q.shape, torch.bfloat16, 7.0), guards.empty((Hq, q.shape[0]), torch.float32, 7.0)) for _ in range(4)]]
            for _ in streams]
    torch.cuda.synchronize()
    for i in range(4):
        for st, (ws, out) in zip(streams, bufs):
            _call(*dev, offd, n, CROSS, o=out[i][0], lse=out[i][1], ws=ws, stream=st)
    torch.cuda.synchronize()
    for _, out in bufs:
        for o, lse in out:
            assert torch.equal(o.cpu().view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse.cpu(), want[1])


def test_pages_and_appends_on_another_stream():
    # a run of all page calls and both appends on one side stream, the state and the rows against the plain model
    r = random.Random(5)
    B, width, pages, P, n = 6, 5, 16, 4, 2
    c = Cache(B, width, pages, P, n=n)
    side = torch.cuda.Stream()
    kw = dict(dev_status=c.status, stream=side)
    i32 = lambda x: torch.tensor(x, dtype=I32, device="cuda")  # noqa: E731
    keep = []  # inputs of calls in flight on the side stream

    def rows(shape, seed):
        keep.append((inputs.normal_bf16(shape, seed), inputs.normal_bf16(shape, seed + 1)))
        keep.append(tuple(x.cuda() for x in keep[-1]))
        return keep[-2], keep[-1]

    pool = [c.k.cpu().clone(), c.v.cpu().clone()]

    def put(b, t, j, x):
        for p, y in zip(pool, x):
            p[c.book.table[b][t // P], t % P * n:t % P * n + n] = y[j]

    def copied(pairs):
        for a, z in pairs:
            if a >= 0:
                for p in pool:
                    p[z] = p[a]

    for step in range(12):
        new = [r.choice([0, 1, 3, 6]) if T == 0 else r.choice([0, 1, 2]) for T in c.book.lens]
        before = list(c.book.lens)
        c.book.grow([min(x, width * P - T) for x, T in zip(new, before)])
        got = [z - a for a, z in zip(before, c.book.lens)]
        new = [min(x, width * P - T) for x, T in zip(new, before)]
        off = [0]
        for x in new:
            off.append(off[-1] + x)
        host, dev = rows(((off[-1] + 1) * n, *c.row), 100 + 2 * step)
        add, offd = i32(new), i32(off)
        src, dst, seqs = None, None, None
        side.wait_stream(torch.cuda.current_stream())
        binding.hd_pages_grow(c.refs, c.table, c.lens, add, P, c.ws, served=c.served, **kw)
        binding.sfa_kv_append_paged(*dev, c.k, c.v, c.table, c.lens, n, offsets=offd, served=c.served, **kw)
        for b in range(B):
            if got[b] == new[b]:
                for j in range(new[b]):
                    put(b, c.book.lens[b] - new[b] + j, off[b] + j, [h.view(-1, n, *c.row) for h in host])
        held, empty = [b for b in range(B) if c.book.lens[b]], [b for b in range(B) if not c.book.lens[b]]
        if held and empty:
            dst = empty[:2]
            src = [r.choice(held) for _ in dst]
            copies, sd, dd = torch.empty(len(dst), 2, dtype=I32, device="cuda"), i32(src), i32(dst)
            side.wait_stream(torch.cuda.current_stream())
            binding.hd_pages_fork(c.refs, c.table, c.lens, sd, dd, None, copies, P, c.ws, **kw)
            binding.hd_pages_copy(c.k, c.v, copies, **kw)
            copied(c.book.fork(src, dst))
            keep.append((copies, sd, dd))
        if step % 3 == 2:
            seqs = r.sample(range(B), 2)
            sd, moves = i32(seqs), torch.empty(pages // 2, 2, dtype=I32, device="cuda")
            side.wait_stream(torch.cuda.current_stream())
            binding.hd_pages_free(c.refs, c.table, c.lens, sd, P, **kw)
            binding.hd_pages_compact(c.refs, c.table, c.lens, c.refs, c.table, moves, P, c.ws, **kw)
            binding.hd_pages_copy(c.k, c.v, moves, **kw)
            c.book.free(seqs)
            copied(c.book.compact())
            keep.append((sd, moves))
        keep.append((add, offd))
    torch.cuda.synchronize()
    c.same()
    for p, x in zip(pool, (c.k, c.v)):
        assert torch.equal(p.view(torch.int16), x.cpu().view(torch.int16))
