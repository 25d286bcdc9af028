"""Paged cache, host side: what the C ABI and the binding refuse before anything is enqueued, and the
index arithmetic that the kernels share, run on the CPU against its definition (bad pages among it)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2607_08186_gb300 import binding, build

FAKE = 1 << 20  # aligned non-null address; never dereferenced (validation fails first)
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


P_ = ctypes.c_void_p


def _decode(lib, B=2, T=64, pages=20, P=8, width=8, n=2, Hq=4, Hkv=2, Dh=64, mode=0, window=0, ptr=FAKE, table=FAKE,
            ws=FAKE, ws_bytes=1 << 40, status=None, lse=FAKE):
    return lib.sfa_decode_paged(P_(ptr), P_(ptr), P_(ptr), P_(table), P_(FAKE), P_(ptr), P_(lse), B, T, pages, P, width, n,
                                Hq, Hkv, Dh, 0.0, mode, window, P_(ws), ws_bytes, P_(status), None)


def test_decode_paged_refusals(lib):
    for bad in (dict(B=0), dict(T=0), dict(pages=0), dict(P=0), dict(width=0), dict(n=0), dict(Hq=5), dict(Hkv=0),
                dict(mode=3), dict(mode=2, window=0), dict(ptr=FAKE + 8), dict(ptr=0), dict(table=FAKE + 2), dict(table=0),
                dict(T=65), dict(lse=FAKE + 2), dict(status=FAKE + 2)):
        assert _decode(lib, **bad) == 1, bad
    for bad in (dict(Dh=96), dict(B=65536), dict(pages=1 << 27, P=8), dict(P=1 << 29, width=2, T=8),
                dict(B=60000, width=1 << 16, P=1), dict(Hq=70000, Hkv=70000)):
        assert _decode(lib, **bad) == 2, bad
    need = binding.sfa_decode_paged_workspace_bytes(2, 64, 2, 4, 2, 64, 0)
    assert need > 0
    assert _decode(lib, ws=0) == 4 and _decode(lib, ws=FAKE + 8) == 4 and _decode(lib, ws_bytes=need - 1) == 4
    assert binding.sfa_decode_paged_workspace_bytes(2, 64, 2, 4, 2, 96, 0) == 0
    assert binding.sfa_decode_paged_workspace_bytes(2, 0, 2, 4, 2, 64, 0) == 0
    assert binding.sfa_decode_paged_workspace_bytes(2, 64, 2, 4, 2, 64, 3) == 0
    # a window beyond the sequence is that of the whole sequence
    assert binding.sfa_decode_paged_workspace_bytes(2, 64, 2, 4, 2, 64, 2, 2**31 - 1) == \
        binding.sfa_decode_paged_workspace_bytes(2, 64, 2, 4, 2, 64, 2, 128)


def _append(lib, B=2, N=2, pages=20, P=8, width=8, n=2, Hkv=2, Dh=64, new=FAKE, pool=FAKE, offsets=None, lens=FAKE):
    return lib.sfa_kv_append_paged(P_(new), P_(new), P_(pool), P_(pool), P_(FAKE), P_(lens), P_(offsets), B, N, pages, P,
                                   width, n, Hkv, Dh, None, None)


def test_append_paged_refusals(lib):
    for bad in (dict(B=0), dict(N=3), dict(N=-1, offsets=FAKE), dict(P=0), dict(n=0), dict(Dh=4), dict(Hkv=0),
                dict(new=0), dict(new=FAKE + 8), dict(pool=FAKE + 8), dict(offsets=FAKE + 2), dict(lens=0)):
        assert _append(lib, **bad) == 1, bad
    for bad in (dict(pages=1 << 28), dict(width=1 << 28), dict(Hkv=1 << 20), dict(N=1 << 30, offsets=FAKE)):
        assert _append(lib, **bad) == 2, bad
    assert _append(lib, N=0, offsets=FAKE, new=0) == 0  # nothing to append


def test_page_calls_refusals(lib):
    need = binding.hd_pages_workspace_bytes(4, 10)
    assert need >= 4 * (3 * 10 + 4) and binding.hd_pages_workspace_bytes(0, 10) == 0
    f, z = P_(FAKE), P_(0)

    def grow(refs=f, table=f, lens=f, add=f, B=4, width=5, pages=10, P=8, ws=f, b=need):
        return lib.hd_pages_grow(refs, table, lens, add, B, width, pages, P, ws, b, None, None)

    def fork(F=2, src=f, copies=f, B=4, ws=f, b=need):
        return lib.hd_pages_fork(f, f, f, src, f, z, F, copies, B, 5, 10, 8, ws, b, None, None)

    def free(F=1, seqs=f, pages=10):
        return lib.hd_pages_free(f, f, f, seqs, F, 4, 5, pages, 8, None, None)

    def compact(nr=f, nt=f, moves=f, pages=10, ws=f, b=need):
        return lib.hd_pages_compact(f, f, f, nr, nt, moves, 4, 5, pages, 8, ws, b, None, None)

    def copy(k=f, c=f, F=2, pages=10, nbytes=64):
        return lib.hd_pages_copy(k, f, c, F, pages, nbytes, None, None)

    bad = [grow(refs=P_(FAKE + 8)), grow(table=z), grow(lens=P_(FAKE + 1)), grow(add=z), grow(B=0), grow(P=0),
           fork(F=-1), fork(F=5), fork(src=z), fork(copies=P_(FAKE + 4)), free(F=-1), free(seqs=z), free(pages=0),
           compact(nr=P_(FAKE + 4)), compact(nt=z), compact(moves=P_(FAKE + 4)), copy(k=z), copy(c=P_(FAKE + 4)),
           copy(F=-1), copy(nbytes=0), copy(nbytes=24), copy(pages=0)]
    assert bad == [1] * len(bad)
    assert grow(width=1 << 29) == 2 and grow(B=1 << 30) == 2 and copy(nbytes=1 << 35) == 2
    assert [grow(ws=z), grow(b=need - 1), fork(ws=P_(FAKE + 4)), compact(b=0)] == [4] * 4
    assert [fork(F=0, src=z, copies=z, ws=z), free(F=0, seqs=z), copy(F=0, c=z)] == [0] * 3


def _packed(lib, B=2, N=40, n=2, Hq=4, Hkv=2, Dh=64, mode=0, window=0, ptr=FAKE, off=FAKE, ws=FAKE, ws_bytes=1 << 40, status=0):
    return lib.sfa_fwd_packed(P_(ptr), P_(ptr), P_(ptr), P_(ptr), P_(ptr), P_(off), B, N, n, Hq, Hkv, Dh, 0.0, mode, window,
                              P_(ws), ws_bytes, P_(status), None)


def test_packed_refusals(lib):
    for bad in (dict(B=0), dict(N=0), dict(n=0), dict(Hq=5), dict(mode=7), dict(mode=2), dict(ptr=FAKE + 8), dict(ptr=0),
                dict(off=0), dict(off=FAKE + 2), dict(status=FAKE + 1)):
        assert _packed(lib, **bad) == 1, bad
    for bad in (dict(Dh=96), dict(Dh=128, mode=3), dict(N=1 << 30), dict(N=1 << 27, Hq=64)):
        assert _packed(lib, **bad) == 2, bad
    need = binding.sfa_fwd_packed_workspace_bytes(2, 40, 2, 4, 2, 64, 0)
    assert need > 0 and binding.sfa_fwd_packed_workspace_bytes(2, 0, 2, 4, 2, 64, 0) == 0
    assert _packed(lib, ws=0) == 4 and _packed(lib, ws=FAKE + 8) == 4 and _packed(lib, ws_bytes=need - 1) == 4


def _cpu_pool(pages=6, P=8, n=2, Hkv=2, Dh=64):
    return torch.zeros(pages, P * n, Hkv, Dh, dtype=torch.bfloat16)


def test_binding_refuses_wrong_tensors(lib):
    i32 = torch.int32
    k = _cpu_pool()
    table, lens = torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32)
    q = torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)

    def decode(q=q, k=k, v=k, table=table, lens=lens, o=q, n=2, ws=ws, lse=None):
        with pytest.raises(ValueError) as e:
            binding.sfa_decode_paged(q, k, v, table, lens, o, n, 0, ws, lse=lse)
        return str(e.value)

    assert "CUDA" in decode()                                    # no fallback: host tensors are refused
    assert "lens" in decode(lens=lens.long())
    assert "lens" in decode(lens=lens[:2])
    assert "q must" in decode(q=q.float())
    assert "o must" in decode(o=q[:2])
    assert "v_pages" in decode(v=k[:5])
    assert "k_pages" in decode(k=k.transpose(0, 1).contiguous().transpose(0, 1))  # the right shape, other strides
    assert "page_table" in decode(table=torch.zeros(4, 3, dtype=i32).t())
    assert "page_tokens" in decode(n=3)
    assert "lse" in decode(lse=torch.zeros(3, 2, 4))
    assert "workspace" in decode(ws=ws.view(i32))
    assert "k_pages" in decode(k=k[0])

    def append(kn, n=2, offsets=None):
        with pytest.raises(ValueError) as e:
            binding.sfa_kv_append_paged(kn, kn, k, k, table, lens, n, offsets=offsets)
        return str(e.value)

    assert "k_new" in append(torch.zeros(3, 1, 2, 64, dtype=torch.bfloat16))
    assert "k_new" in append(torch.zeros(7, 2, 64, dtype=torch.bfloat16), offsets=torch.zeros(4, dtype=i32))
    assert "offsets" in append(torch.zeros(8, 2, 64, dtype=torch.bfloat16), offsets=torch.zeros(3, dtype=i32))
    p = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    off, lse = torch.zeros(3, dtype=i32), torch.zeros(4, 8)

    def packed(q=p, k=p, v=p, o=p, lse=lse, off=off, n=2, ws=ws):
        with pytest.raises(ValueError) as e:
            binding.sfa_fwd_packed(q, k, v, o, lse, off, n, 0, ws)
        return str(e.value)

    assert "CUDA" in packed() and "lse" in packed(lse=lse.double()) and "offsets" in packed(off=off.long())
    assert "v must" in packed(v=p[:4]) and "o must" in packed(o=p.float()) and "N * n" in packed(n=3)
    assert "q must" in packed(q=p[0]) and "workspace" in packed(ws=None)
    refs = torch.zeros(6, dtype=i32)
    for call in (lambda: binding.hd_pages_grow(refs, table, lens, lens[:2], 8, ws),
                 lambda: binding.hd_pages_grow(refs, table, lens, lens, 8, ws),  # on the host
                 lambda: binding.hd_pages_grow(refs.long(), table, lens, lens, 8, ws),
                 lambda: binding.hd_pages_fork(refs, table, lens, lens, lens[:2], None, table[:, :2], 8, ws),
                 lambda: binding.hd_pages_free(refs, table, lens, lens.float(), 8),
                 lambda: binding.hd_pages_compact(refs, table, lens, refs, table, torch.zeros(2, 2, dtype=i32), 8, ws),
                 lambda: binding.hd_pages_copy(k, k[:3], torch.zeros(2, 2, dtype=i32)),
                 lambda: binding.hd_pages_copy(k, k, torch.zeros(4, dtype=i32)),
                 lambda: binding.hd_pages_grow(refs, table[0], lens, lens, 8, ws)):
        with pytest.raises(ValueError):
            call()


def test_page_row_on_the_host(tmp_path):
    # the kernels' own page_row, compiled for the host: every position's row lies in the pool, and a
    # table entry outside it gives -1
    src = tmp_path / "rows.cu"
    src.write_text('#include "%s/paper_2607_08186_gb300/csrc/pages.cuh"\n'
                   'extern "C" int rows(int np, int mp, int prow, const int* t, int p) {\n'
                   '  return hdsfa::page_row(hdsfa::make_page_geom(np, mp, prow), t, p); }\n' % ROOT)
    so = tmp_path / "rows.so"
    subprocess.run([build.nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-shared",
                    *build.ARCH, str(src), "-o", str(so)], check=True, capture_output=True)
    f = ctypes.CDLL(str(so)).rows
    g = torch.Generator().manual_seed(1)
    for np_, prow in ((1, 1), (7, 1), (5, 3), (9, 64), (3, 60), (1000, 128), (2**31 // 96 - 1, 96), (2, 2**29)):
        mp = 5
        t = torch.randint(0, np_, (mp,), generator=g).tolist()
        for bad in (-1, np_, -2**31, 2**31 - 1):
            entries = t[:2] + [bad] + t[3:]
            arr = (ctypes.c_int * mp)(*entries)
            for i in range(mp):
                if (i + 1) * prow > 2**31:
                    break
                for r in {0, prow // 2, prow - 1}:
                    row = f(np_, mp, prow, arr, i * prow + r)
                    assert row == (-1 if i == 2 else entries[i] * prow + r)
                    assert row < np_ * prow
        if mp * prow < 2**31:
            assert f(np_, mp, prow, (ctypes.c_int * mp)(*t), mp * prow) == -1  # behind the table
