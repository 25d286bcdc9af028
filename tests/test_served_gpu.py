"""A grow that finds no page, and the append that follows it without a look at the status: no row that a
sequence or its fork holds changes.  Everything here is whole numbers and bit copies."""
import pytest
import torch

import guards
import paging
from paper_2607_08186_gb300 import binding, build, inputs

pytestmark = pytest.mark.gpu

I32 = torch.int32
INDEX, PAGES = binding.HD_DEVBIT_INDEX, binding.HD_DEVBIT_PAGES


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=I32, device="cuda")


class Cache:
    """A paged cache on the GPU with the plain model beside it."""

    def __init__(self, B, width, pages, P, n=2, Hkv=2, Dh=64, seed=1):
        self.n, self.P = n, P
        self.book = paging.Book(B, width, pages, P)
        self.refs, self.lens = guards.zeros((pages,), I32), guards.zeros((B,), I32)
        self.table = guards.empty((B, width), I32, -1)
        self.served = guards.empty((B,), I32, 99)
        self.ws = guards.empty((binding.hd_pages_workspace_bytes(B, pages),), torch.uint8, 0xAB)
        self.status = guards.zeros((1,), I32)
        self.k, self.v = (guards.like(inputs.normal_bf16((pages, P * n, Hkv, Dh), seed + i).cuda()) for i in (0, 1))
        for i, x in enumerate((self.k, self.v)):
            x.copy_(inputs.normal_bf16(tuple(x.shape), seed + i))
        self.row = (Hkv, Dh)

    def grow(self, add):
        """hd_pages_grow with served, against the model; what was served."""
        before = list(self.book.lens)
        self.book.grow(add)
        binding.hd_pages_grow(self.refs, self.table, self.lens, _i32(add), self.P, self.ws, dev_status=self.status,
                              served=self.served)
        got = self.served.tolist()
        assert got == [z - a for a, z in zip(before, self.book.lens)]
        self.same()
        return got

    def same(self):
        assert self.lens.tolist() == self.book.lens and self.refs.tolist() == self.book.refs
        assert self.table.tolist() == self.book.table and int(self.status.item()) == self.book.status

    def append(self, new, seed, offsets=None, **kw):
        """Random new rows appended with served; (k, v) of the pool as they have to be where counts say `new`."""
        n, total = self.n, len(new) if offsets is None else offsets[-1] + 2
        shape = (total, n, *self.row) if offsets is None else (total * n, *self.row)
        kn, vn = inputs.normal_bf16(shape, seed), inputs.normal_bf16(shape, seed + 1)
        want = [self.k.cpu().clone(), self.v.cpu().clone()]
        for b, c in enumerate(new):
            for i in range(c):
                t = self.book.lens[b] - c + i
                page, at = self.book.table[b][t // self.P], t % self.P * n
                for w, x in zip(want, (kn, vn)):
                    w[page, at:at + n] = x[b] if offsets is None else x[(offsets[b] + i) * n:(offsets[b] + i + 1) * n]
        binding.sfa_kv_append_paged(kn.cuda(), vn.cuda(), self.k, self.v, self.table, self.lens, n,
                                    offsets=None if offsets is None else _i32(offsets), dev_status=self.status,
                                    served=self.served, **kw)
        torch.cuda.synchronize()
        for w, x in zip(want, (self.k, self.v)):
            assert torch.equal(w.view(torch.int16), x.cpu().view(torch.int16))
        assert int(self.status.item()) == self.book.status


def test_a_refused_token_leaves_a_shared_page_alone():
    # slot 0 fills both of its pages, slot 1 is forked from it at a page's end (which takes no page), and the pool
    # is empty: neither gets a page for its next token, and neither's last row, which they share, changes
    c = Cache(3, 4, 3, 4)
    assert c.grow([8, 0, 4]) == [8, 0, 4]
    copies = guards.empty((1, 2), I32, 77)
    binding.hd_pages_fork(c.refs, c.table, c.lens, _i32([0]), _i32([1]), None, copies, c.P, c.ws, dev_status=c.status)
    assert c.book.fork([0], [1]) == [(-1, -1)] and c.book.refs == [2, 2, 1]
    c.same()
    assert c.grow([1, 1, 1]) == [0, 0, 0] and c.book.status == PAGES
    c.append([0, 0, 0], 10)
    # slot 2 ends: its page serves the first that asks
    binding.hd_pages_free(c.refs, c.table, c.lens, _i32([2]), c.P, dev_status=c.status)
    c.book.free([2])
    assert c.grow([1, 1, 0]) == [1, 0, 0]
    c.append([1, 0, 0], 12)
    assert c.grow([1, 1, 0]) == [1, 0, 0]
    c.append([1, 0, 0], 14)


def test_prompts_of_which_some_find_no_pages():
    c = Cache(4, 5, 4, 4)
    c.grow([5, 8, 0, 0])
    c.append([5, 8, 0, 0], 20, offsets=[0, 5, 13, 13, 13])
    # every page is held: slot 0's tokens find room in its last one, slot 1 (whose last four rows a plain append would
    # write over) and the new slot 2 get none, slot 3 brings nothing
    assert c.grow([3, 4, 9, 0]) == [3, 0, 0, 0] and c.book.status == PAGES
    c.append([3, 0, 0, 0], 22, offsets=[1, 4, 8, 17, 17])


def test_lengths_out_of_range_are_not_served():
    c = Cache(4, 2, 6, 4)
    c.grow([4, 1, 0, 0])
    assert c.grow([5, -1, 8, 9]) == [0, 0, 8, 0] and c.book.status == INDEX
    c.append([0, 0, 1, 0], 30)


def test_served_below_what_is_brought():
    # a caller's own counts: less than the rows a sequence brings leaves all of them out, more changes nothing
    c = Cache(3, 4, 8, 4)
    c.grow([6, 6, 6])
    c.served.copy_(_i32([2, 3, 9]))
    c.append([0, 3, 3], 40, offsets=[0, 3, 6, 9])


@pytest.mark.parametrize("offsets", [None, [0, 3, 4, 4]])
def test_captured_and_on_another_stream(offsets):
    # grow and append captured together follow their state: the third replay finds no page for slot 0
    B, n, P = 3, 2, 4
    new = [1, 1, 1] if offsets is None else [3, 1, 0]
    c = Cache(B, 4, 4, P)
    c.grow([3, 2, 0] if offsets is None else [1, 3, 0])
    shape = (B, n, *c.row) if offsets is None else (4 * n, *c.row)
    kn, vn = inputs.normal_bf16(shape, 50).cuda(), inputs.normal_bf16(shape, 51).cuda()
    add, off = _i32(new), None if offsets is None else _i32(offsets)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        binding.hd_pages_grow(c.refs, c.table, c.lens, add, P, c.ws, dev_status=c.status, served=c.served, stream=side)
        binding.sfa_kv_append_paged(kn, vn, c.k, c.v, c.table, c.lens, n, offsets=off, dev_status=c.status,
                                    served=c.served, stream=side)
    refused = 0
    for _ in range(8):
        before = list(c.book.lens)
        c.book.grow(new)
        got = [z - a for a, z in zip(before, c.book.lens)]
        want = [c.k.cpu().clone(), c.v.cpu().clone()]
        for b in range(B):
            refused += got[b] < new[b]
            for i in range(got[b]):
                t = c.book.lens[b] - got[b] + i
                for w, x in zip(want, (kn.cpu(), vn.cpu())):
                    rows = x[b] if offsets is None else x[(offsets[b] + i) * n:(offsets[b] + i + 1) * n]
                    w[c.book.table[b][t // P], t % P * n:t % P * n + n] = rows
        graph.replay()
        torch.cuda.synchronize()
        assert c.served.tolist() == got
        c.same()
        for w, x in zip(want, (c.k, c.v)):
            assert torch.equal(w.view(torch.int16), x.cpu().view(torch.int16))
    assert refused > 0 and c.book.status == PAGES
