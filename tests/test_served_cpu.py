"""What the grow and the append with `served` refuse, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

from paper_2607_08186_gb300 import binding, build

FAKE = 1 << 20  # aligned non-null address; never dereferenced (validation fails first)
P_ = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_refusals(lib):
    need = binding.hd_pages_workspace_bytes(4, 10)

    def grow(served=FAKE, add=FAKE, B=4, ws=FAKE, b=need):
        return lib.hd_pages_grow_served(P_(FAKE), P_(FAKE), P_(FAKE), P_(add), P_(served), B, 5, 10, 8, P_(ws), b, None, None)

    def append(served=FAKE, N=2, new=FAKE, offsets=None, n=2):
        return lib.sfa_kv_append_paged_served(P_(new), P_(new), P_(FAKE), P_(FAKE), P_(FAKE), P_(FAKE), P_(offsets),
                                              P_(served), 2, N, 20, 8, 8, n, 2, 64, None, None)

    assert [grow(served=0), grow(served=FAKE + 2), grow(add=0), grow(B=0)] == [1] * 4
    assert [grow(ws=0), grow(b=need - 1)] == [4] * 2
    assert [append(served=0), append(served=FAKE + 1), append(N=3), append(new=0), append(n=0)] == [1] * 5
    assert append(N=0, offsets=FAKE, new=0) == 0


def test_binding_refuses_wrong_tensors(lib):
    i32 = torch.int32
    k = torch.zeros(6, 16, 2, 64, dtype=torch.bfloat16)
    table, lens, refs = torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(6, dtype=i32)
    kn, ws = torch.zeros(3, 2, 2, 64, dtype=torch.bfloat16), torch.zeros(4096, dtype=torch.uint8)
    for served, word in ((lens[:2], "served"), (lens.long(), "served"), (lens, "CUDA")):
        with pytest.raises(ValueError, match=word):
            binding.hd_pages_grow(refs, table, lens, lens, 8, ws, served=served)
        with pytest.raises(ValueError, match=word):
            binding.sfa_kv_append_paged(kn, kn, k, k, table, lens, 2, served=served)


def test_tensors_without_the_expected_dimensions_are_value_errors(lib):
    i32, bf16 = torch.int32, torch.bfloat16
    table, lens, off = torch.zeros(3, 4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(4, dtype=i32)
    k = torch.zeros(6, 16, 2, 64, dtype=bf16)
    for pool in (torch.zeros(0, 16, 2, 64, dtype=bf16), torch.zeros((), dtype=bf16)):
        with pytest.raises(ValueError):
            binding.hd_pages_copy(pool, pool, torch.zeros(0, 2, dtype=i32))
    for new in (torch.zeros((), dtype=bf16), torch.zeros(4, dtype=bf16)):
        with pytest.raises(ValueError, match="k_new"):
            binding.sfa_kv_append_paged(new, new, k, k, table, lens, 2, offsets=off)
