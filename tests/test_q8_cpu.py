"""8-bit paged cache, host side: what the C ABI and the binding refuse before anything is enqueued, and the arithmetic
that the kernels share, run on the CPU against its definition."""
import ctypes
import os
import random
import subprocess
import tempfile

import pytest
import torch

import q8
from paper_2607_08186_gb300 import binding, build

FAKE = 1 << 20  # aligned non-null address; never dereferenced (validation fails first)
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P_ = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _append(lib, B=2, N=2, pages=20, P=8, width=8, n=2, Hkv=2, Dh=64, T=4, new=FAKE, pool=FAKE, scales=FAKE, offsets=None,
            lens=FAKE, served=None, status=None):
    return lib.sfa_kv_append_paged_q8(P_(new), P_(new), P_(pool), P_(pool), P_(scales), P_(scales), P_(FAKE), P_(lens),
                                      P_(offsets), P_(served), B, N, pages, P, width, n, Hkv, Dh, T, P_(status), None)


def test_append_refusals(lib):
    for bad in (dict(B=0), dict(N=3), dict(N=-1, offsets=FAKE), dict(P=0), dict(n=0), dict(Dh=8), dict(Dh=72), dict(Hkv=0),
                dict(T=0), dict(T=3), dict(T=16), dict(new=0), dict(new=FAKE + 8), dict(pool=FAKE + 8), dict(pool=0),
                dict(scales=0), dict(scales=FAKE + 8), dict(offsets=FAKE + 2), dict(lens=0), dict(served=FAKE + 1),
                dict(status=FAKE + 2)):
        assert _append(lib, **bad) == 1, bad
    for bad in (dict(pages=1 << 28), dict(width=1 << 28), dict(Hkv=1 << 20), dict(N=1 << 30, offsets=FAKE),
                dict(Hkv=40000, Dh=16), dict(pages=1 << 26, Hkv=8), dict(P=1 << 24, T=1 << 24, width=1, pages=1)):
        assert _append(lib, **bad) == 2, bad
    assert _append(lib, N=0, offsets=FAKE, new=0) == 0  # nothing to append


def _read(lib, B=2, N=6, pages=20, P=8, width=8, n=2, Hkv=2, Dh=64, T=4, out=FAKE, pool=FAKE, scales=FAKE, offsets=FAKE,
          lens=FAKE):
    return lib.sfa_kv_read_paged_q8(P_(pool), P_(pool), P_(scales), P_(scales), P_(FAKE), P_(lens), P_(offsets), P_(out),
                                    P_(out), B, N, pages, P, width, n, Hkv, Dh, T, None, None)


def test_read_refusals(lib):
    for bad in (dict(B=0), dict(N=-1), dict(P=0), dict(n=0), dict(Dh=24), dict(T=5), dict(out=0), dict(out=FAKE + 8),
                dict(pool=0), dict(scales=0), dict(scales=FAKE + 4), dict(offsets=0), dict(offsets=FAKE + 2), dict(lens=FAKE + 1)):
        assert _read(lib, **bad) == 1, bad
    for bad in (dict(pages=1 << 28), dict(N=1 << 30)):
        assert _read(lib, **bad) == 2, bad
    assert _read(lib, N=0, out=0) == 0


def _decode(lib, B=2, T=64, pages=20, P=8, width=8, n=2, Hq=4, Hkv=2, Dh=64, block=4, mode=0, window=0, ptr=FAKE,
            scales=FAKE, table=FAKE, ws=FAKE, ws_bytes=1 << 40, status=None, lse=FAKE):
    return lib.sfa_decode_paged_q8(P_(ptr), P_(ptr), P_(ptr), P_(scales), P_(scales), P_(table), P_(FAKE), P_(ptr), P_(lse),
                                   B, T, pages, P, width, n, Hq, Hkv, Dh, block, 0.0, mode, window, P_(ws), ws_bytes,
                                   P_(status), None)


def test_decode_refusals(lib):
    for bad in (dict(B=0), dict(T=0), dict(pages=0), dict(P=0), dict(width=0), dict(n=0), dict(Hq=5), dict(Hkv=0),
                dict(mode=3), dict(mode=2, window=0), dict(ptr=FAKE + 8), dict(ptr=0), dict(scales=0), dict(scales=FAKE + 1), dict(table=FAKE + 2),
                dict(table=0), dict(T=65), dict(lse=FAKE + 2), dict(status=FAKE + 2), dict(block=0), dict(block=3)):
        assert _decode(lib, **bad) == 1, bad
    for bad in (dict(Dh=96), dict(B=65536), dict(pages=1 << 27, P=8), dict(P=1 << 29, width=2, T=8, block=1),
                dict(B=60000, width=1 << 16, P=1, block=1), dict(Hq=70000, Hkv=70000), dict(B=60000, Hq=32000, Hkv=32000)):
        assert _decode(lib, **bad) == 2, bad
    need = binding.sfa_decode_paged_q8_workspace_bytes(2, 64, 2, 4, 2, 64, 0)
    assert need > 0
    assert _decode(lib, ws=0) == 4 and _decode(lib, ws=FAKE + 8) == 4 and _decode(lib, ws_bytes=need - 1) == 4
    for bad in ((2, 64, 2, 4, 2, 96, 0), (2, 0, 2, 4, 2, 64, 0), (2, 64, 2, 4, 2, 64, 3)):
        assert binding.sfa_decode_paged_q8_workspace_bytes(*bad) == 0
    assert binding.sfa_decode_paged_q8_workspace_bytes(2, 64, 2, 4, 2, 64, 2, 2**31 - 1) == \
        binding.sfa_decode_paged_q8_workspace_bytes(2, 64, 2, 4, 2, 64, 2, 128)


def test_counts_beyond_32_bits_are_refused(lib):
    for B, Hkv in ((65535, 131072), (65535, 65536), (65535, 1 << 20)):  # CTAs of one split: 2^33, 2^32 and 2^36
        assert binding.sfa_decode_paged_q8_workspace_bytes(B, 16, 1, Hkv, Hkv, 64, 1) == 0


def test_workspace_serves_every_shorter_step(lib):
    r = random.Random(3)
    for _ in range(400):
        B, n, (Hq, Hkv) = r.choice([1, 2, 7, 33, 300]), r.choice([1, 2, 3, 4, 8]), r.choice([(4, 4), (32, 8), (96, 8), (24, 2)])
        Dh, mode = r.choice([64, 128, 256]), r.choice([0, 1, 2])
        L = r.randint(1, 40000)
        w = r.randint(1, 50000) if mode == 2 else 0
        most = binding.sfa_decode_paged_q8_workspace_bytes(B, L, n, Hq, Hkv, Dh, mode, w)
        less = binding.sfa_decode_paged_q8_workspace_bytes(B, r.randint(1, L), n, Hq, Hkv, Dh, mode, r.randint(1, w) if w else 0)
        assert 0 < less <= most


def test_copy_refusals(lib):
    def copy(k=FAKE, s=FAKE, c=FAKE, F=2, pages=10, nbytes=64, ns=3):
        return lib.hd_pages_copy_q8(P_(k), P_(FAKE), P_(s), P_(FAKE), P_(c), F, pages, nbytes, ns, None, None)

    assert [copy(k=0), copy(k=FAKE + 4), copy(s=0), copy(s=FAKE + 2), copy(c=0), copy(c=FAKE + 4), copy(F=-1), copy(nbytes=0),
            copy(nbytes=24), copy(ns=0), copy(pages=0)] == [1] * 11
    assert copy(nbytes=1 << 35) == 2 and copy(ns=1 << 31) == 2 and copy(F=0, c=0) == 0


def test_binding_refuses_wrong_tensors(lib):
    f8, u8, i32, bf = torch.float8_e4m3fn, torch.uint8, torch.int32, torch.bfloat16
    k = torch.zeros(6, 2, 16, 64, dtype=u8).view(f8)
    ks = torch.zeros(6, 2, 4, dtype=u8)
    table, lens, off = torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(4, dtype=i32)
    q, new, ws = torch.zeros(3, 2, 4, 64, dtype=bf), torch.zeros(3, 2, 2, 64, dtype=bf), torch.zeros(1 << 16, dtype=u8)
    rows = torch.zeros(10, 2, 64, dtype=bf)
    calls = {"on cpu": (k, k, ks, ks, table), "three blocks": (k, k, ks[:, :, :3].contiguous(), ks, table),
             "v scales": (k, k, ks, ks[:5], table), "codes as uint8": (k.view(u8), k.view(u8), ks, ks, table),
             "flat scales": (k, k, ks.view(-1), ks, table), "flat table": (k, k, ks, ks, table[0]),
             "three dimensions": (k[0], k[0], ks, ks, table)}
    for name, (a, b, c, d, t) in calls.items():
        with pytest.raises(ValueError):
            binding.sfa_decode_paged_q8(q, a, b, c, d, t, lens, q, 2, 0, ws)
        with pytest.raises(ValueError):
            binding.sfa_kv_append_paged_q8(new, new, a, b, c, d, t, lens, 2)
        with pytest.raises(ValueError):
            binding.sfa_kv_read_paged_q8(a, b, c, d, t, lens, off, rows, rows, 2)
    with pytest.raises(ValueError):
        binding.sfa_decode_paged_q8(q, k, k, ks, ks, table, lens, q, 3, 0, ws)  # 16 rows are no whole tokens of 3 streams
    with pytest.raises(ValueError):
        binding.hd_pages_copy_q8(k, k, ks, ks, torch.zeros(2, 2, dtype=i32))  # on the CPU
    with pytest.raises(ValueError):
        binding.hd_pages_copy_q8(k[:0], k[:0], ks[:0], ks[:0], torch.zeros(2, 2, dtype=i32))


@pytest.fixture(scope="module")
def shared():
    """The kernels' scale arithmetic, compiled for the host."""
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "q8.cu"), os.path.join(d, "q8.so")
        with open(src, "w") as f:
            f.write('#include "%s/paper_2607_08186_gb300/csrc/q8.cuh"\n'
                    'extern "C" void bytes(int* out) { for (unsigned i = 0; i < 0x7f80; ++i) out[i] = hdsfa::q8::scale_byte(i); }\n'
                    % ROOT)
        subprocess.run([build.nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-shared",
                        *build.ARCH, src, "-o", so], check=True, capture_output=True)
        return ctypes.CDLL(so)


def test_scale_of_every_magnitude(shared):
    got = torch.empty(0x7F80, dtype=torch.int32)
    shared.bytes(ctypes.c_void_p(got.data_ptr()))
    values = torch.arange(0x7F80, dtype=torch.int16).view(torch.bfloat16).tolist()
    assert got.tolist() == [q8.exponent(v) + 127 for v in values]


def test_model_rounds_as_the_type_does():
    """The model's rounding against torch's conversion, at all codes, the middles between them and beside these."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    c = torch.unique(codes[torch.isfinite(codes)])
    mid = (c[1:] + c[:-1]) / 2
    x = torch.cat([c, mid, torch.nextafter(mid, torch.tensor(1e9)), torch.nextafter(mid, torch.tensor(-1e9))])
    x = x[x.abs() <= 448]
    assert torch.equal(q8.nearest(x).float(), x.to(torch.float8_e4m3fn).float())
    assert q8.nearest(torch.tensor([1e9, -500.0])).tolist() == [448.0, -448.0]
    assert bool(torch.isnan(q8.nearest(torch.tensor([float("inf"), float("nan")]))).all())


@pytest.mark.parametrize("T", [1, 2, 3, 5, 16])
def test_units_of_packed_prompts(T):
    """Numbers offsets[b] / T + 2 b + j, j < blocks touched, are all different and below N / T + 2 B."""
    r = random.Random(T)
    for _ in range(300):
        B = r.randint(1, 9)
        new = [r.choice([0, 0, 1, 2, r.randint(0, 40)]) for _ in range(B)]
        off = [r.choice([0, 0, 3])]
        for x in new:
            off.append(off[-1] + x)
        N, seen = off[-1] + r.choice([0, 7]), []
        for b, x in enumerate(new):
            first = r.randint(0, 50)
            blocks = (first + x - 1) // T - first // T + 1 if x else 0
            start = off[b] // T + 2 * b
            assert blocks <= (off[b + 1] // T + 2 * b + 2) - start
            seen += [start + j for j in range(blocks)]
        assert len(set(seen)) == len(seen) and max(seen, default=0) <= N // T + 2 * B - 1


def test_parts_of_a_shared_wave():
    """Part x of S has the units floor(x all / S) ... of the sequences' tiles, each with 6 units of its start in front: every
    tile is in one part, no two partials have the number x + b, and a sequence's have successive ones, 128 at most."""
    r = random.Random(5)
    start = 6
    for _ in range(400):
        B, total, kind = r.randint(2, 128), r.choice([1, 2, 9, 19, 76, 152, 228, 456]), r.random()
        tiles = [0 if r.random() < 0.2 else r.randint(1, 5 if kind < 0.4 else 3000) if r.random() < 0.95 else 8000000 for _ in range(B)]
        size = [t + start if t else 0 for t in tiles]
        every, most = sum(size), max(size)
        S = max(1, min(total, every))
        if most * S > 126 * every:
            S = 126 * every // most
        per, rest = every // S, every % S
        parts, numbers = {}, set()
        for x in range(S):
            u0, u1 = x * per + x * rest // S, (x + 1) * per + (x + 1) * rest // S
            assert (u0, u1) == (x * every // S, (x + 1) * every // S) and (u0 < u1 or not every)
            before = 0
            for b in range(B):
                lo, hi = max(u0, before + start), min(u1, before + size[b])
                if size[b] and lo < hi:
                    assert x + b not in numbers and x + b < total + B
                    numbers.add(x + b)
                    parts.setdefault(b, []).append((x + b, lo - before - start, hi - before - start))
                before += size[b]
        before = 0
        for b in range(B):
            if tiles[b]:
                of = lambda u: ((u + 1) * S - 1) // every
                x0 = of(before + start)
                n = of(before + size[b] - 1) - x0 + 1
                mine = parts[b]
                assert n <= 128 and [p[0] for p in mine] == list(range(x0 + b, x0 + b + n))
                assert mine[0][1] == 0 and mine[-1][2] == tiles[b] and all(p[2] == q[1] for p, q in zip(mine, mine[1:]))
            before += size[b]
