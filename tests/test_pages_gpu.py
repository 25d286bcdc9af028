"""Bookkeeping of a paged cache's pages on the GPU, step by step against a plain Python model: every
count, table entry, length and copy equal, and the status bits."""
import random

import pytest
import torch

import guards
import paging
from paper_2607_08186_gb300 import binding, build

pytestmark = pytest.mark.gpu

I32 = torch.int32
INDEX, PAGES = binding.HD_DEVBIT_INDEX, binding.HD_DEVBIT_PAGES


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _i32(x, shape=None):
    t = torch.tensor(x, dtype=I32, device="cuda")
    return t if shape is None else t.view(shape)


class Device:
    """The same state on the GPU, every buffer between guard bytes."""

    def __init__(self, B, width, pages, P):
        self.P, self.pages = P, pages
        self.refs, self.lens = guards.zeros((pages,), I32), guards.zeros((B,), I32)
        self.table = guards.empty((B, width), I32, -1)
        self.ws = guards.empty((binding.hd_pages_workspace_bytes(B, pages),), torch.uint8, 0xAB)
        self.status = guards.zeros((1,), I32)

    def load(self, book):
        self.refs.copy_(_i32(book.refs)), self.lens.copy_(_i32(book.lens)), self.table.copy_(_i32(book.table))

    def grow(self, add):
        binding.hd_pages_grow(self.refs, self.table, self.lens, _i32(add), self.P, self.ws, dev_status=self.status)

    def fork(self, src, dst, tokens=None):
        copies = guards.empty((len(src), 2), I32, 77)
        binding.hd_pages_fork(self.refs, self.table, self.lens, _i32(src), _i32(dst), None if tokens is None else _i32(tokens),
                              copies, self.P, self.ws, dev_status=self.status)
        return [tuple(x) for x in copies.tolist()]

    def free(self, seqs):
        binding.hd_pages_free(self.refs, self.table, self.lens, _i32(seqs), self.P, dev_status=self.status)

    def compact(self, in_place=False):
        moves = guards.empty((self.pages // 2, 2), I32, 77)
        nr, nt = (self.refs, self.table) if in_place else (guards.empty(self.refs.shape, I32, 55),
                                                           guards.empty(self.table.shape, I32, 55))
        binding.hd_pages_compact(self.refs, self.table, self.lens, nr, nt, moves, self.P, self.ws, dev_status=self.status)
        self.refs, self.table = nr, nt
        return [tuple(x) for x in moves.tolist()]


def _same(dev, book):
    assert dev.lens.tolist() == book.lens
    assert dev.refs.tolist() == book.refs
    assert dev.table.tolist() == book.table
    assert int(dev.status.item()) == book.status
    held = [0] * book.pages  # counts are what the tables say
    for b, T in enumerate(book.lens):
        for i in range(paging.pages_of(T, book.P)):
            held[book.table[b][i]] += 1
    assert held == book.refs


@pytest.mark.parametrize("B,width,pages,P,seed", [(4, 6, 17, 4, 1), (3, 5, 40, 1, 2), (40, 9, 200, 3, 3), (9, 30, 64, 16, 4),
                                                  (1500, 4, 4099, 5, 5), (20, 300, 9000, 2, 6), (2, 1, 1, 8, 7)])
def test_random_steps(B, width, pages, P, seed):
    r = random.Random(seed)
    book, dev = paging.Book(B, width, pages, P), Device(B, width, pages, P)
    for step in range(24):
        what = r.choice(["grow", "grow", "fork", "free", "compact"])
        if what == "grow":
            add = [r.choice([0, 1, 1, P, r.randint(0, max(1, width * P // 3))]) for _ in range(B)]
            add = [min(a, width * P - T) for a, T in zip(add, book.lens)]
            book.grow(add), dev.grow(add)
        elif what == "fork":
            empty = [b for b in range(B) if book.lens[b] == 0]
            full = [b for b in range(B) if book.lens[b] > 0]
            if not empty or not full:
                continue
            dst = r.sample(empty, r.randint(1, len(empty)))
            src = [r.choice(full) for _ in dst]
            tokens = None if r.random() < 0.3 else [r.randint(0, book.lens[a]) for a in src]
            assert book.fork(src, dst, tokens) == dev.fork(src, dst, tokens)
        elif what == "free":
            seqs = [r.randrange(B) for _ in range(r.randint(1, max(1, B // 2)))]  # a slot may come twice
            book.free(seqs), dev.free(seqs)
        else:
            assert book.compact() == dev.compact(in_place=step % 2 == 0)
        _same(dev, book)


def test_grow_serves_in_order_and_leaves_the_rest():
    book, dev = paging.Book(6, 4, 5, 8), Device(6, 4, 5, 8)
    for add in ([8, 1, 0, 16, 8, 0], [0, 7, 0, 8, 1, 0], [-1, 0, 99, 0, 0, 1], [0, 0, 33, 0, 0, 0]):
        book.grow(add), dev.grow(add)
        _same(dev, book)
    assert book.status == INDEX | PAGES


def test_grow_bad_lengths_are_left_out():
    dev = Device(4, 4, 9, 8)
    dev.lens.copy_(_i32([-1, 33, 2**31 - 1, 0]))
    dev.grow([1, 1, 2**31 - 1, 1])
    assert dev.lens.tolist() == [-1, 33, 2**31 - 1, 1] and dev.refs.tolist() == [1] + [0] * 8
    assert int(dev.status.item()) == INDEX


@pytest.mark.parametrize("src,dst,tokens", [
    ([0, 0, 0], [2, 2, 3], [9, 12, 4]),              # a destination twice: the first one counts
    ([0, 9, -1, 1], [2, 3, 4, -2], [1, 1, 1, 1]),    # slots that are not there
    ([0, 1], [1, 0], [1, 1]),                        # destinations in use
    ([0, 2], [2, 3], [13, 0]),                       # a slot that this call fills is empty as a source
    ([0, 2], [2, 3], [13, 5]),
    ([0, 0], [0, 2], [5, 21]),                       # onto itself; more tokens than there are
    ([0, 1], [2, 3], [-1, 8]),
    ([0, 1, 0], [2, 3, 4], None),
    ([5, 5], [2, 3], None),                          # an empty source
])
def test_fork_edges(src, dst, tokens):
    book, dev = paging.Book(6, 5, 20, 8), Device(6, 5, 20, 8)
    for x in (book, dev):
        x.grow([20, 16, 0, 0, 0, 0])
    assert book.fork(src, dst, tokens) == dev.fork(src, dst, tokens)
    _same(dev, book)


def test_fork_without_a_free_page():
    book, dev = paging.Book(5, 4, 4, 8), Device(5, 4, 4, 8)
    for x in (book, dev):
        x.grow([20, 0, 0, 0, 0])
    # one page is free: the first that asks gets it, whole pages are shared all the same
    assert book.fork([0, 0, 0, 0], [1, 2, 3, 4], [17, 18, 16, 3]) == dev.fork([0, 0, 0, 0], [1, 2, 3, 4], [17, 18, 16, 3])
    _same(dev, book)
    assert book.status == PAGES and book.lens == [20, 17, 0, 16, 0]


def test_corrupt_tables_are_reported_and_stay_in_bounds():
    book, dev = paging.Book(3, 4, 12, 8), Device(3, 4, 12, 8)
    for x in (book, dev):
        x.grow([30, 20, 0])
    dev.table[0, 1], dev.table[0, 2], dev.table[1, 0] = -7, 12, 11  # no pages; one that nobody holds
    assert dev.fork([0, 1], [2, 2], None) == [(-1, -1), (-1, -1)]
    assert int(dev.status.item()) == INDEX and dev.lens.tolist() == [30, 20, 0]
    dev.status.zero_()
    saved = dev.refs.clone(), dev.table.clone()
    dev.compact()
    assert int(dev.status.item()) == INDEX
    assert dev.table[0, 1:3].tolist() == [-1, -1] and int(dev.table[1, 0]) == -1
    dev.refs, dev.table = saved
    dev.status.zero_()
    dev.free([0, 1, 7, -1])
    assert int(dev.status.item()) == INDEX and dev.lens.tolist() == [0, 0, 0]
    assert dev.table.eq(-1).all() and int(dev.refs.min()) == 0
    # pages 1, 2 and 4 (the entries that were overwritten) are still counted; nothing else is
    assert dev.refs.nonzero().flatten().tolist() == [1, 2, 4]


def test_shared_pages_outlive_their_first_holder():
    book, dev = paging.Book(3, 4, 12, 8), Device(3, 4, 12, 8)
    for x in (book, dev):
        x.grow([20, 0, 0])
        x.fork([0, 0], [1, 2], [20, 16])
        x.free([0, 0, 2])
    _same(dev, book)
    assert book.refs[:2] == [1, 1] and book.lens == [0, 20, 0]


@pytest.mark.parametrize("page", [(1, 1, 8), (6, 2, 64), (64, 8, 128), (60, 4, 256)])
def test_copies(page):
    pages = 40
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randint(-2**15, 2**15, (pages, *page), generator=g).to(torch.int16).view(torch.bfloat16) for _ in range(2))
    perm = torch.randperm(pages, generator=g).tolist()
    pairs = [(perm[i % 7], perm[10 + i]) for i in range(25)]  # sources may come again
    pairs[4:4] = [(-1, -1)] * 2
    kd, vd = guards.like(k.cuda()), guards.like(v.cuda())
    kd.copy_(k), vd.copy_(v)
    st = torch.zeros(1, dtype=I32, device="cuda")
    binding.hd_pages_copy(kd, vd, _i32(pairs), dev_status=st)
    for a, b in pairs:
        if a >= 0:
            k[b], v[b] = k[a], v[a]
    assert torch.equal(kd.cpu().view(torch.int16), k.view(torch.int16))
    assert torch.equal(vd.cpu().view(torch.int16), v.view(torch.int16)) and int(st.item()) == 0
    binding.hd_pages_copy(kd, vd, _i32([(0, pages), (pages, 0), (-1, 3), (5, -1), (2**31 - 1, 1)]), dev_status=st)
    assert int(st.item()) == INDEX and torch.equal(kd.cpu().view(torch.int16), k.view(torch.int16))
    none = torch.empty(0, 2, dtype=I32, device="cuda")
    binding.hd_pages_copy(kd, vd, none)


def test_captured_steps():
    # a step (free, fork, grow) captured once and replayed follows its state
    B, width, pages, P = 5, 6, 40, 4
    book, dev = paging.Book(B, width, pages, P), Device(B, width, pages, P)
    for x in (book, dev):
        x.grow([9, 14, 0, 0, 0])
    src, dst, tok, add = _i32([0, 1, 0]), _i32([2, 3, 4]), _i32([5, 8, 9]), _i32([1, 1, 3, 3, 3])
    copies = torch.empty(3, 2, dtype=I32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.hd_pages_free(dev.refs, dev.table, dev.lens, dst, P, dev_status=dev.status)
        binding.hd_pages_fork(dev.refs, dev.table, dev.lens, src, dst, tok, copies, P, dev.ws, dev_status=dev.status)
        binding.hd_pages_grow(dev.refs, dev.table, dev.lens, add, P, dev.ws, dev_status=dev.status)
    for _ in range(4):
        graph.replay()
        book.free([2, 3, 4])
        want = book.fork([0, 1, 0], [2, 3, 4], [5, 8, 9])
        book.grow([1, 1, 3, 3, 3])
        assert [tuple(x) for x in copies.tolist()] == want
        _same(dev, book)
