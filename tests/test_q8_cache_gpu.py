"""8-bit paged cache on the GPU: what appends write, what is read back, and copies of pages, bit for bit against the
64-bit model (scales are powers of two, so every step is exact or one rounding that the model makes too)."""
import pytest
import torch

import guards
import q8
from paper_2607_08186_gb300 import binding, build, inputs

pytestmark = pytest.mark.gpu

I32, U8, F8, BF = torch.int32, torch.uint8, torch.float8_e4m3fn, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=I32, device="cuda")


class Pools:
    """K and V pools on the GPU (fenced) with their models; what nobody has written holds NaN codes and odd scales."""

    def __init__(self, pages, P, n, Hkv, Dh, T, seed=0):
        self.P, self.n, self.Hkv, self.Dh, self.T = P, n, Hkv, Dh, T
        g = torch.Generator().manual_seed(seed)
        self.dev, self.model = [], []
        for _ in range(2):
            codes = torch.randint(0, 256, (pages, Hkv, P * n, Dh), dtype=U8, generator=g)
            scales = torch.randint(0, 256, (pages, Hkv, P // T), dtype=U8, generator=g)
            c, s = guards.empty(codes.shape, U8, what="codes"), guards.empty(scales.shape, U8, what="scales")
            c.copy_(codes), s.copy_(scales)
            self.dev.append((c.view(F8), s))
            self.model.append(q8.Cache(pages, P, n, Hkv, Dh, T, codes.view(F8), scales))
        (self.k, self.ks), (self.v, self.vs) = self.dev

    def append(self, kn, vn, table, lens, offsets=None, served=None, stream=None):
        st = torch.zeros(1, dtype=I32, device="cuda")
        binding.sfa_kv_append_paged_q8(kn, vn, self.k, self.v, self.ks, self.vs, table, lens, self.n, offsets=offsets,
                                       served=served, dev_status=st, stream=stream)
        torch.cuda.synchronize()
        return int(st.item())

    def read(self, table, lens, offsets, k, v):
        st = torch.zeros(1, dtype=I32, device="cuda")
        binding.sfa_kv_read_paged_q8(self.k, self.v, self.ks, self.vs, table, lens, offsets, k, v, self.n, dev_status=st)
        torch.cuda.synchronize()
        return int(st.item())

    def same(self):
        for (c, s), m in zip(self.dev, self.model):
            m.same(c, s)


def _rows(tokens, n, Hkv, Dh, seed):
    """bf16 rows whose magnitudes grow and shrink from token to token, over many binades."""
    x = inputs.normal_bf16((tokens, n, Hkv, Dh), seed).float()
    g = torch.Generator().manual_seed(seed + 1)
    return (x * torch.exp2(torch.randint(-6, 7, (tokens, 1, Hkv, 1), generator=g).float())).to(BF)


def _table(lens, P, pages, width, seed):
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    t = torch.full((len(lens), width), -1, dtype=I32)
    for b, L in enumerate(lens):
        for i in range(-(-L // P)):
            t[b, i] = perm.pop()
    return t


# page sizes odd, prime and one; blocks of a token, of some, of a page; units that a warp takes and that a CTA does,
# with rows beyond what its threads hold (64 tokens x 4 streams x 128)
SHAPES = [(4, 8, 128, 16, 16), (4, 8, 128, 16, 1), (4, 2, 128, 64, 64), (2, 4, 64, 8, 4), (3, 4, 64, 50, 25),
          (1, 2, 256, 7, 7), (1, 1, 64, 1, 1), (8, 2, 256, 12, 6), (5, 3, 80, 9, 3), (70, 1, 16, 3, 1), (1, 2, 128, 131, 131)]


@pytest.mark.parametrize("n,Hkv,Dh,P,T", SHAPES)
def test_append_prompts_then_tokens(n, Hkv, Dh, P, T):
    lens0, width = [37, 1, 0, 129, 16], 160 // P + 1
    cap = [x + 20 for x in lens0]
    pages = sum(-(-x // P) for x in cap) + 2
    t = _table(cap, P, pages, width, 3)
    p = Pools(pages, P, n, Hkv, Dh, T, seed=n + Dh)
    # whole prompts, packed from token 2 on with rows behind them
    off = [2]
    for x in lens0:
        off.append(off[-1] + x)
    N = off[-1] + 3
    kn, vn = _rows(N, n, Hkv, Dh, 5), _rows(N, n, Hkv, Dh, 6)
    st = p.append(kn.view(N * n, Hkv, Dh).cuda(), vn.view(N * n, Hkv, Dh).cuda(), t.cuda(), _i32(lens0), offsets=_i32(off))
    assert st == 0
    for m, x in zip(p.model, (kn, vn)):
        for b, L in enumerate(lens0):
            m.append(x[off[b]:off[b + 1]], t[b], 0)
    p.same()
    # then single tokens, an idle slot and a refused one among them: blocks that hold tokens, and blocks that begin
    lens = list(lens0)
    for step in range(12):
        idle, refused = step % 5, (step + 1) % 5
        lens = [x + 1 if b not in (idle, refused) else x for b, x in enumerate(lens)]
        served = [int(b != refused) for b in range(5)]
        kn, vn = _rows(5, n, Hkv, Dh, 20 + step), _rows(5, n, Hkv, Dh, 50 + step)
        call = [0 if b == idle else x for b, x in enumerate(lens)]
        assert p.append(kn.cuda(), vn.cuda(), t.cuda(), _i32(call), served=_i32(served)) == 0
        for m, x in zip(p.model, (kn, vn)):
            for b in range(5):
                if b not in (idle, refused):
                    m.append(x[b:b + 1], t[b], lens[b] - 1)
        p.same()
    # then more tokens of each, packed, behind those in their blocks
    more = [0, 7, 3, 1, 2]
    off = [0]
    for x in more:
        off.append(off[-1] + x)
    lens = [a + b for a, b in zip(lens, more)]
    kn, vn = _rows(off[-1], n, Hkv, Dh, 90), _rows(off[-1], n, Hkv, Dh, 91)
    assert p.append(kn.view(-1, Hkv, Dh).cuda(), vn.view(-1, Hkv, Dh).cuda(), t.cuda(), _i32(lens), offsets=_i32(off)) == 0
    for m, x in zip(p.model, (kn, vn)):
        for b in range(5):
            m.append(x[off[b]:off[b + 1]], t[b], lens[b] - more[b])
    p.same()
    # and all of it back, a prefix of one of them
    want = list(lens)
    want[3] = 77
    off = [1]
    for x in want:
        off.append(off[-1] + x)
    N = off[-1] + 2
    k, v = guards.empty((N * n, Hkv, Dh), BF, 7.0), guards.empty((N * n, Hkv, Dh), BF, 7.0)
    assert p.read(t.cuda(), _i32(want), _i32(off), k, v) == 0
    for m, got in zip(p.model, (k.cpu(), v.cpu())):
        for b in range(5):
            assert torch.equal(got[off[b] * n:off[b + 1] * n], m.rows(t[b], want[b]).to(BF))
        assert bool((got[:n] == 7.0).all()) and bool((got[off[-1] * n:] == 7.0).all())


def test_read_the_last_tokens():
    n, Hkv, Dh, P, T = 3, 4, 64, 10, 5
    lens = [40, 3, 0, 25]
    t = _table(lens, P, 12, 5, 1)
    p = Pools(12, P, n, Hkv, Dh, T, seed=2)
    for m, (c, s) in zip(p.model, p.dev):  # codes without NaN, scales in their range
        s.copy_(torch.randint(100, 140, s.shape, dtype=U8, generator=torch.Generator().manual_seed(1)))
        c.view(U8).bitwise_and_(0xF7)
        m.e, m.codes = s.cpu().long() - 127, c.cpu().float().double().view(m.codes.shape)
    off = [0, 1, 4, 4, 15]
    k, v = guards.empty((15 * n, Hkv, Dh), BF, 7.0), guards.empty((15 * n, Hkv, Dh), BF, 7.0)
    assert p.read(t.cuda(), _i32(lens), _i32(off), k, v) == 0
    for m, got in zip(p.model, (k.cpu(), v.cpu())):
        for b, L in enumerate(lens):
            x = off[b + 1] - off[b]
            assert torch.equal(got[off[b] * n:off[b + 1] * n], m.rows(t[b], L)[(L - x) * n:].to(BF))


def test_values_at_the_borders():
    """Zeros of both signs, what bf16 holds at its ends, infinities and NaN, borders of the scales' range, ties."""
    n, Hkv, Dh, P, T = 1, 1, 64, 4, 1
    inf, nan = float("inf"), float("nan")
    heads = [[0.0, -0.0], [1e-38, -1e-38], [2.0 ** -133], [3.38e38, -3.38e38, 1.0], [inf, 2.0, -inf, 448.0], [nan, 1.0, -3.0],
             [inf, nan], [448.0 * 2.0 ** 50, 449.0 * 2.0 ** 50, 2.0 ** 59], [448.0, 450.0], [452.0, 1.0], [1.75, 1.0625, 1.1875],
             [448.0 * 2.0 ** -64, 2.0 ** -73, 2.0 ** -74, 1.5 * 2.0 ** -74, 2.0 ** -75], [448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9]]
    x = torch.zeros(len(heads), n, Hkv, Dh, dtype=BF)
    for i, h in enumerate(heads):
        x[i, 0, 0, :len(h)] = torch.tensor(h, dtype=torch.float64).to(BF)
    L = len(heads)
    t = _table([L], P, 6, 4, 0)
    for block in (1, 2, 4):
        p = Pools(6, P, n, Hkv, Dh, block, seed=block)
        for i in range(L):  # a token at a time: blocks whose scale grows by a little, by a lot, or not
            assert p.append(x[i:i + 1].cuda(), x[i:i + 1].cuda(), t.cuda(), _i32([i + 1])) == 0
            for m in p.model:
                m.append(x[i:i + 1], t[0], i)
            p.same()
        k, v = guards.empty((L, Hkv, Dh), BF), guards.empty((L, Hkv, Dh), BF)
        assert p.read(t.cuda(), _i32([L]), _i32([0, L]), k, v) == 0
        want = p.model[0].rows(t[0], L).to(BF)
        for got in (k.cpu(), v.cpu()):
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(got.nan_to_num(0.0, 0.0, 0.0), want.nan_to_num(0.0, 0.0, 0.0))


def test_refused_rows_change_nothing():
    n, Hkv, Dh, P, T = 2, 2, 64, 8, 4
    t = _table([16, 16, 16, 16], P, 9, 3, 2)
    t[1, 1] = 9  # no page of the pool
    t[2, 0] = -1
    x = _rows(4, n, Hkv, Dh, 1)
    p = Pools(9, P, n, Hkv, Dh, T)
    # a length behind the table, pages that are none, and one that is fine
    assert p.append(x.cuda(), x.cuda(), t.cuda(), _i32([25, 9, 3, 16])) == binding.HD_DEVBIT_INDEX
    for m in p.model:
        m.append(x[3:4], t[3], 15)
    p.same()
    assert p.append(x.cuda(), x.cuda(), t.cuda(), _i32([-1, 0, 0, 0])) == binding.HD_DEVBIT_INDEX
    p.same()
    # packed: more tokens than the length, offsets that leave the rows, a bad page under some of a sequence's tokens
    x = _rows(12, n, Hkv, Dh, 2)
    r = x.view(-1, Hkv, Dh).cuda()
    assert p.append(r, r, t.cuda(), _i32([3, 11, 0, 0]), offsets=_i32([0, 4, 10, 10, 10])) == binding.HD_DEVBIT_INDEX
    for m in p.model:
        m.append(x[4:7], t[1], 5)  # tokens 5 ... 7; 8 ... 10 have no page
    p.same()
    assert p.append(r, r, t.cuda(), _i32([0, 0, 0, 16]), offsets=_i32([0, 0, 0, 0, 13])) == binding.HD_DEVBIT_INDEX
    assert p.append(r, r, t.cuda(), _i32([0, 0, 0, 16]), offsets=_i32([-1, 0, 0, 0, 0])) == binding.HD_DEVBIT_INDEX
    p.same()
    # served fewer than it brings: left out without a bit
    assert p.append(r, r, t.cuda(), _i32([0, 0, 0, 16]), offsets=_i32([0, 0, 0, 0, 12]), served=_i32([0, 0, 0, 0])) == 0
    p.same()
    # reading: the same refusals, rows left as they were
    k, v = guards.empty((12 * n, Hkv, Dh), BF, 7.0), guards.empty((12 * n, Hkv, Dh), BF, 7.0)
    assert p.read(t.cuda(), _i32([25, 11, 0, 2]), _i32([0, 1, 4, 4, 12]), k, v) == binding.HD_DEVBIT_INDEX
    assert bool((k == 7.0).all()) and bool((v == 7.0).all())


def test_copy():
    n, Hkv, Dh, P, T = 3, 5, 80, 6, 2
    p = Pools(40, P, n, Hkv, Dh, T)
    pairs = [(3, 7), (-1, -1), (3, 9), (39, 0), (5, 40), (-1, 4)]
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.hd_pages_copy_q8(p.k, p.v, p.ks, p.vs, _i32(pairs), dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == binding.HD_DEVBIT_INDEX  # the last two
    for m in p.model:
        for a, b in pairs[:4]:
            if a >= 0:
                m.codes[b], m.e[b] = m.codes[a], m.e[a]
    p.same()
    binding.hd_pages_copy_q8(p.k, p.v, p.ks, p.vs, _i32([]).view(0, 2))
    # scales of one byte a page
    q = Pools(3, 1, 1, 1, 16, 1)
    binding.hd_pages_copy_q8(q.k, q.v, q.ks, q.vs, _i32([(2, 1)]))
    for m in q.model:
        m.codes[1], m.e[1] = m.codes[2], m.e[2]
    q.same()


def test_many_sequences_and_a_large_prompt():
    """More sequences than a warp has lanes, most of them empty; and units of more CTAs than fit at a time."""
    n, Hkv, Dh, P, T = 2, 2, 64, 4, 2
    B = 70
    new = [0 if b % 3 else b % 11 for b in range(B)]
    new[41] = 900
    off = [0]
    for x in new:
        off.append(off[-1] + x)
    t = _table(new, P, 400, 225, 8)
    p = Pools(400, P, n, Hkv, Dh, T)
    x, y = _rows(off[-1], n, Hkv, Dh, 3), _rows(off[-1], n, Hkv, Dh, 4)
    assert p.append(x.view(-1, Hkv, Dh).cuda(), y.view(-1, Hkv, Dh).cuda(), t.cuda(), _i32(new), offsets=_i32(off)) == 0
    for m, r in zip(p.model, (x, y)):
        for b in range(B):
            m.append(r[off[b]:off[b + 1]], t[b], 0)
    p.same()


def test_on_another_stream_and_replayed():
    n, Hkv, Dh, P, T = 2, 2, 64, 8, 8
    t = _table([64], P, 9, 8, 0)
    p = Pools(9, P, n, Hkv, Dh, T)
    x, y = _rows(6, n, Hkv, Dh, 3), _rows(6, n, Hkv, Dh, 4)
    xd, yd, td, lens = x[:1].cuda(), y[:1].cuda(), t.cuda(), _i32([0])
    one = torch.ones(1, dtype=I32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lens.add_(one)
        binding.sfa_kv_append_paged_q8(xd, yd, p.k, p.v, p.ks, p.vs, td, lens, n, stream=torch.cuda.current_stream())
    for i in range(6):
        xd.copy_(x[i:i + 1]), yd.copy_(y[i:i + 1])
        g.replay()
        torch.cuda.synchronize()
        for m, r in zip(p.model, (x, y)):
            m.append(r[i:i + 1], t[0], i)
    p.same()
