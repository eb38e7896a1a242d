"""The book of a cache's pages (mt_kv_reserve, mt_kv_fork, mt_kv_release, mt_kv_compact) against a restatement with lists, exactly, and mt_kv_copy."""
import random

import pytest
import torch

from lm_util import init, random_cache
from more_lm_util import Book
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """A book on the device beside its restatement; every call is made on both and compared."""

    def __init__(self, n_pages, page, rows, width):
        init()
        self.pages = mt.KvPages.empty(n_pages, page, rows, width)
        self.book = Book([0] * n_pages, [[0] * width for _ in range(rows)], [0] * rows, page)

    def load(self):
        b, k = self.book, self.pages
        k.refs.copy_(i32(b.refs)); k.tables.copy_(i32(b.tables).view(k.tables.shape)); k.lengths.copy_(i32(b.lengths))

    def same(self, errors):
        b, k = self.book, self.pages
        assert mt.mt_get_async_status() == (min(errors, key=lambda e: (e[0], e[1])) if errors else (0, -1))
        assert k.lengths.tolist() == b.lengths
        assert k.refs.tolist() == b.refs
        assert k.tables.tolist() == b.tables

    def reserve(self, rows, counts, n_slots=None):
        n_slots = sum(max(c, 0) for c in counts) if n_slots is None else n_slots
        slots = torch.full((n_slots,), -9, dtype=torch.int64, device="cuda")
        mt.mt_kv_reserve(self.pages, i32(rows), i32(counts), slots)
        want, errors = self.book.reserve(rows, counts, n_slots)
        assert slots.tolist() == want
        self.same(errors)
        return errors

    def fork(self, parents, children):
        copies = torch.full((len(parents), 3), -9, dtype=torch.int32, device="cuda")
        mt.mt_kv_fork(self.pages, i32(parents), i32(children), copies)
        want, errors = self.book.fork(parents, children)
        assert copies.tolist() == [list(c) for c in want]
        self.same(errors)
        return errors

    def release(self, rows):
        mt.mt_kv_release(self.pages, i32(rows))
        errors = self.book.release(rows)
        self.same(errors)
        return errors

    def compact(self, most):
        copies = torch.full((most, 3), -9, dtype=torch.int32, device="cuda")
        mt.mt_kv_compact(self.pages, copies)
        want = self.book.compact(most)
        assert copies.tolist() == [list(c) for c in want]
        self.same([])

    def sound(self):
        """References are what the tables say, and a shared page is full."""
        b, seen, partly = self.book, [0] * len(self.book.refs), set()
        for r in range(len(b.lengths)):
            for x in b.held(r):
                seen[x] += 1
            if b.lengths[r] % b.page:
                partly.add(b.held(r)[-1])
        assert seen == b.refs and all(seen[x] == 1 for x in partly)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n_pages,rows,width", [(40, 9, 7), (700, 40, 30), (70000, 30, 5), (200003, 6, 20)])
def test_a_long_story(n_pages, rows, width, page):
    """Rows that grow, fork, change places and end, in a random order, with the whole state compared after each call."""
    rng = random.Random(n_pages + page)
    k = Both(n_pages, page, rows, width)
    for step in range(45):
        b = k.book
        what = rng.choice(["reserve", "reserve", "fork", "fork", "release", "compact"])
        some = rng.sample(range(rows), rng.randint(1, rows))
        if what == "reserve":
            some = [r for r in some if b.lengths[r] < width * page] or some[:0]
            if some:
                k.reserve(some, [rng.choice([0, 1, 1, min(page, width * page - b.lengths[r]), rng.randint(0, width * page - b.lengths[r])]) for r in some])
        elif what == "fork":
            k.fork([rng.randrange(rows) for _ in some], some)
        elif what == "release":
            k.release(some[: 1 + len(some) // 2])
        else:
            k.compact(rng.choice([1, 3, n_pages // 2]))
        k.sound()


@pytest.mark.parametrize("rows,width,n_pages,many", [(5000, 3, 20000, 1500), (1100, 4, 3000, 1100), (4097, 2, 9000, 40), (300, 900, 40000, 300)])
def test_large_calls(rows, width, n_pages, many):
    """More places, rows or table entries than one CTA keeps in shared memory or takes by itself."""
    rng = random.Random(rows)
    k = Both(n_pages, 16, rows, width)
    some = rng.sample(range(rows), many)
    k.reserve(some, [rng.randint(0, 16 * width) if width < 10 else rng.randint(0, 16 * 80) for _ in some])
    children = rng.sample(range(rows), many)
    k.fork([rng.choice(some) for _ in children], children)
    k.sound()
    k.reserve(children, [rng.randint(0, 16 * width - k.book.lengths[c]) % 7 for c in children])
    k.release(children[::2])
    k.compact(n_pages // 2)
    k.sound()


def test_edges_of_pages():
    """Lengths at and beside the ends of pages."""
    k = Both(30, 16, 8, 4)
    k.reserve([0, 1, 2, 3, 4], [0, 1, 15, 16, 17])
    k.reserve([0, 1, 2, 3, 4], [64, 15, 1, 16, 15])
    k.fork([0, 1, 2], [5, 6, 7])
    k.reserve([5], [1])
    k.reserve([7, 6, 5], [1, 1, 0])
    k.sound()


def test_beams_that_change_places():
    k = Both(60, 16, 6, 6)
    k.reserve([0, 1, 2, 3], [20, 33, 48, 7])
    k.fork([1, 0, 3, 2], [0, 1, 2, 3])                          # each other's
    k.sound()
    k.fork([0, 0, 0, 0], [0, 1, 2, 3])                          # one wins
    k.sound()
    k.fork([3, 3, 1, 4], [4, 5, 3, 0])                          # from one without tokens too
    k.sound()
    k.release([0, 1, 2, 3, 4, 5])
    assert set(k.book.refs) == {0}


def test_when_pages_run_out():
    k = Both(6, 16, 6, 5)
    k.reserve([0, 1], [40, 20])                                 # five of six
    assert k.reserve([2, 3, 4], [16, 1, 0]) == [(5, 1)]         # the second has none left, the third needs none
    k.release([2])
    assert k.fork([0, 0, 1], [3, 4, 5]) == [(5, 1), (5, 2)]
    k.sound()
    assert k.reserve([0, 1, 2, 3, 4], [8, 12, 100, 1, 16])[0] == (1, 2)
    k.sound()


def test_places_that_are_left_out():
    k = Both(40, 16, 8, 4)
    k.reserve([0, 1, 2], [30, 5, 64])
    assert k.reserve([3, 3, -1, 8, 4, 2, 5], [1, 1, 1, 1, -2, 1, 1]) == [(1, i) for i in (1, 2, 3, 4, 5)]
    assert k.reserve([0, 1, 6], [10, 10, 10], n_slots=25) == [(1, 2)]
    assert k.reserve([0], [1], n_slots=9) == []
    assert k.fork([0, 1, 9, 0, 0, -1], [6, 6, 7, 7, 99, 4]) == [(1, 1), (1, 2), (1, 3), (1, 4), (1, 5)]
    assert k.release([1, 1, 50, -3, 6]) == [(1, 1), (1, 2), (1, 3)]
    k.sound()
    k.book.lengths[5], k.book.lengths[7] = 65, -1               # passes the table; negative
    k.load()
    assert k.reserve([5, 7, 4], [0, 0, 1]) == [(1, 0), (1, 1)]
    assert k.fork([5, 7, 0, 0], [3, 4, 7, 5]) == [(1, 0), (1, 1), (1, 2), (1, 3)]
    assert k.release([7, 5]) == [(1, 0), (1, 1)]


def test_pages_outside_the_cache():
    """A table that names no page: the fork is left out; the row's other pages come back when it ends."""
    k = Both(10, 16, 4, 3)
    k.reserve([0, 1], [40, 10])
    k.book.tables[0][1] = 10
    k.load()
    assert k.fork([0, 1], [2, 3]) == [(1, 0)]
    mt.mt_kv_release(k.pages, i32([0]))
    assert k.pages.refs.tolist() == [0, 1, 0, 1, 1] + [0] * 5 and k.pages.lengths.tolist() == [0, 10, 0, 10]
    mt.mt_get_async_status()


@pytest.mark.parametrize("page", [10, -1, 2 ** 31 - 1])
def test_a_page_outside_is_neither_appended_to_nor_given_back(page):
    """The partly filled page of row 0 lies outside, and so does a page that row 1 gives back."""
    k = Both(10, 16, 4, 3)
    k.reserve([0, 1, 2], [20, 40, 16])                         # pages 0 1, 2 3 4, 5
    k.book.tables[0][1] = k.book.tables[1][0] = page
    k.load()
    for counts in ([3, 1, 0], [20, 1, 0]):                     # within the page, and past it
        slots = torch.full((sum(counts),), -9, dtype=torch.int64, device="cuda")
        mt.mt_kv_reserve(k.pages, i32([0, 1, 2]), i32(counts), slots)
        assert mt.mt_get_async_status() == (1, 0)
        n = k.pages.lengths.tolist()[1]
        assert slots.tolist() == [-1] * counts[0] + [4 * 16 + n - 1 - 32] and k.pages.lengths.tolist() == [20, n, 16, 0]
    assert k.pages.refs.tolist() == [1] * 6 + [0] * 4
    copies = torch.empty((1, 3), dtype=torch.int32, device="cuda")
    mt.mt_kv_fork(k.pages, i32([2]), i32([1]), copies)
    assert mt.mt_get_async_status() == (1, 0)
    assert k.pages.refs.tolist() == [1, 1, 1, 0, 0, 2] + [0] * 4 and k.pages.lengths.tolist() == [20, 16, 16, 0]
    mt.mt_kv_release(k.pages, i32([2, 0]))
    assert mt.mt_get_async_status() == (1, 1)
    assert k.pages.refs.tolist() == [0, 1, 1, 0, 0, 1] + [0] * 4 and k.pages.lengths.tolist() == [0, 16, 0, 0]


def test_a_page_nobody_holds_is_not_given_back():
    k = Both(10, 16, 3, 3)
    k.reserve([0], [20])
    k.book.refs[1] = 0
    k.load()
    mt.mt_kv_release(k.pages, i32([0]))
    assert mt.mt_get_async_status() == (1, 0) and k.pages.refs.tolist() == [0] * 10


def test_nothing_to_do():
    k = Both(10, 16, 3, 3)
    none = i32([]).view(0, 3)
    mt.mt_kv_fork(k.pages, i32([]), i32([]), none)
    mt.mt_kv_release(k.pages, i32([]))
    mt.mt_kv_compact(k.pages, none)
    k.reserve([], [])
    k.reserve([], [], n_slots=5)
    k.compact(4)
    k = Both(0, 16, 3, 0)
    k.reserve([0, 1], [0, 0])
    k.fork([0], [1])
    k.release([2])
    k.compact(2)


@pytest.mark.parametrize("heads,dim,page", [(1, 64, 16), (8, 128, 64), (3, 64, 32), (5, 128, 256)])
def test_copies(heads, dim, page):
    """Tokens of pages in every layer, bit by bit; everything else stays."""
    init()
    g = torch.Generator(device="cuda").manual_seed(page)
    caches = [random_cache(50, page, heads, dim, g) for _ in range(3)]
    caches.append(random_cache(50, page, heads + 1, 192 - dim, g))
    before = [[t.clone() for t in c.tensors] for c in caches]
    some = torch.randperm(50, generator=torch.Generator().manual_seed(1))[:24].view(-1, 2).tolist()
    copies = [(a, b, t) for (a, b), t in zip(some, [page, 1, 0, page - 1, 7, page // 2, page, 3, 5, page, 2, page])]
    copies.insert(3, (-1, -1, 0))
    copies.append((9, 9, page))
    mt.mt_kv_copy(mt.KvCopier(caches), i32(copies))
    assert mt.mt_get_async_status() == (0, -1)
    for c, was in zip(caches, before):
        for t, w in zip(c.tensors, was):
            for a, b, n in copies:
                if a >= 0:
                    w[b, :, :n] = w[a, :, :n].clone()
            assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))


def test_copies_that_are_left_out():
    init()
    c = random_cache(8, 16, 2, 64, torch.Generator(device="cuda").manual_seed(0))
    before = [t.clone() for t in c.tensors]
    mt.mt_kv_copy(mt.KvCopier([c]), i32([(0, 1, 16), (8, 2, 16), (2, -5, 16), (3, 4, 17), (5, 6, -1), (-1, 7, 3)]))
    assert mt.mt_get_async_status() == (1, 1)
    for t, w in zip(c.tensors, before):
        w[1] = w[0]
        assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))


def test_many_layers_and_many_copies():
    """More caches than one launch takes, more copies than it has CTAs."""
    init()
    g = torch.Generator(device="cuda").manual_seed(0)
    caches = [random_cache(30, 16, 1, 64, g) for _ in range(67)]
    want = [c.tensors[2].clone() for c in caches]
    mt.mt_kv_copy(mt.KvCopier(caches), i32([(i, 15 + i, 16) for i in range(15)]))
    for c, w in zip(caches, want):
        w[15:] = w[:15]
        assert torch.equal(c.tensors[2], w)
    big = random_cache(12000, 16, 1, 64, g)
    want = big.tensors[0].clone()
    copies = torch.stack([torch.arange(6000), 6000 + torch.arange(6000), torch.full((6000,), 16)], 1).int().cuda()
    copies[100:5000] = -1
    mt.mt_kv_copy(mt.KvCopier([big]), copies)
    want[6000:6100], want[11000:] = want[:100], want[5000:6000]
    assert torch.equal(big.tensors[0], want)


def test_captured_and_replayed():
    """A token step's bookkeeping as a graph; and two graphs, and calls beside them, on streams of their own."""
    k = Both(200, 16, 12, 8)
    rows, ones = list(range(12)), [1] * 12
    k.reserve(rows, [10 + i for i in rows])
    slots = torch.zeros(12, dtype=torch.int64, device="cuda")
    r, c = i32(rows), i32(ones)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_kv_reserve(k.pages, r, c, slots, stream=torch.cuda.current_stream())
    for _ in range(20):
        graph.replay()
        torch.cuda.synchronize()
        want, errors = k.book.reserve(rows, ones, 12)
        assert slots.tolist() == want
        k.same(errors)
    other = Both(200, 16, 12, 8)
    other.reserve(rows, [5 + i for i in rows])
    copies = torch.zeros((6, 3), dtype=torch.int32, device="cuda")
    p, ch = i32([0, 1, 2, 3, 4, 5]), i32([6, 7, 8, 9, 10, 11])
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2):
        mt.mt_kv_fork(other.pages, p, ch, copies, stream=torch.cuda.current_stream())
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(a):
            graph.replay()
        with torch.cuda.stream(b):
            graph2.replay()
        torch.cuda.synchronize()
        k.book.reserve(rows, ones, 12)
        other.book.fork([0, 1, 2, 3, 4, 5], [6, 7, 8, 9, 10, 11])
    k.same([])
    other.same([])
    other.sound()
