"""Copying pages, and the book of pages against the same book written out entry by entry: every number has to be equal."""
import random

import pytest
import torch

from page_book import Book, cdiv
from paper_2506_09092_b200 import binding as B

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


class Pair:
    """The library's book and pools beside the written-out one and a host copy of the pools."""

    def __init__(self, pages, page_rows, slots, cols, pools=2, values=24, seed=0):
        self.book, self.want = B.PageBook(pages, page_rows, slots, cols), Book(pages, page_rows, slots, cols)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.data = [torch.randn(pages, page_rows, values * (i + 1), generator=gen, device="cuda").half() for i in range(pools)]
        self.pools = B.page_pools(self.data) if pools else None
        self.mirror = [t.clone() for t in self.data]
        self.result = torch.full((1,), 77, dtype=torch.int32, device="cuda")

    def scratch(self, n):
        self.buf = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        return self.buf, n

    def moved(self, pairs):
        for m in self.mirror:
            old = m.clone()
            for a, b in pairs:
                m[b] = old[a]

    def fork(self, src, dst):
        n = len(src)
        buf, size = self.scratch(B.pages_fork_scratch_bytes(self.book, n))
        B.pages_fork(self.book, ints(src), ints(dst), n, buf, size, torch.cuda.current_stream())
        self.want.fork(src, dst)
        self.check()

    def resize(self, slots, want):
        n = len(want)
        buf, size = self.scratch(B.pages_resize_scratch_bytes(self.book, n))
        B.pages_resize(self.book, self.pools, None if slots is None else ints(slots), ints(want), n, self.result, buf, size,
                       torch.cuda.current_stream())
        result, pairs = self.want.resize(slots, want)
        assert self.result.item() == result
        self.moved(pairs)
        self.check()
        return result

    def compact(self):
        buf, size = self.scratch(B.pages_compact_scratch_bytes(self.book))
        B.pages_compact(self.book, self.pools, self.result, buf, size, torch.cuda.current_stream())
        used, pairs = self.want.compact()
        assert self.result.item() == used
        self.moved(pairs)
        self.check()

    def check(self):
        assert bool((self.buf[-64:] == 0xA5).all())
        assert self.book.refs.tolist() == self.want.refs
        assert self.book.lens.tolist() == self.want.lens
        assert self.book.table.tolist() == self.want.table
        assert self.want.consistent()
        for a, b in zip(self.data, self.mirror):
            assert torch.equal(a, b)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("pages,page_rows,slots,cols", [(40, 4, 6, 9), (300, 16, 20, 30), (17, 1, 5, 8), (5000, 3, 300, 24)])
def test_random_steps(pages, page_rows, slots, cols, seed):
    """Sequences grow, shrink, end and fork in any order; some lists have slots twice, wrong slots or
    lengths, or want more pages than there are."""
    rng = random.Random(seed)
    p = Pair(pages, page_rows, slots, cols, seed=seed)
    for step in range(30):
        n = rng.randint(1, 2 * slots)
        pick = [rng.randrange(-1, slots + 1) if rng.random() < 0.1 else rng.randrange(slots) for _ in range(n)]
        what = rng.random()
        if what < 0.55:
            want = []
            for s in pick:
                have = p.want.lens[s] if 0 <= s < slots else 0
                want.append(rng.choice([have + 1, have + rng.randint(0, 2 * page_rows), max(0, have - rng.randint(0, 2 * page_rows)),
                                        rng.randint(0, cols * page_rows // 2), 0, -1]))
                want[-1] = min(want[-1], cols * page_rows + (rng.random() < 0.003))
            p.resize(pick, want)
        elif what < 0.85:
            p.fork(pick, [rng.randrange(-1, slots + 1) if rng.random() < 0.1 else rng.randrange(slots) for _ in range(n)])
        else:
            p.compact()
    p.compact()


def test_beam_step():
    """Eight sequences of one prompt continue from three of them: copies of the shared tails for all but one of each."""
    p = Pair(64, 16, 8, 6)
    p.resize([0], [40])
    p.fork([0] * 7, range(1, 8))
    assert p.want.refs[:3] == [8] * 3
    p.resize(None, [41] * 8)
    assert p.want.refs[:3] == [8, 8, 1] and sum(r > 0 for r in p.want.refs) == 10
    p.fork([3, 3, 3, 5, 5, 3, 1, 1], range(8))
    p.resize(None, [42] * 8)
    p.resize(None, [0] * 8)
    assert not any(p.want.refs)


def test_a_sequence_that_alone_grows_takes_a_copy_and_the_others_keep_theirs():
    p = Pair(30, 8, 4, 4)
    p.resize([1], [13])
    p.fork([1, 1], [0, 3])
    p.resize([3], [14])
    p.resize([3, 0], [15, 20])                         # 0 and 1 share: 0 copies
    p.resize([1], [14])                                # alone now: in place
    p.resize([0, 1, 3], [0, 0, 0])


def test_a_tail_given_back_in_the_same_call_is_no_longer_shared():
    p = Pair(30, 8, 4, 4)
    p.resize([1], [13])
    p.fork([1], [0])
    p.resize([1, 0], [0, 14])
    assert sum(p.want.refs) == 2


def test_not_enough_pages_changes_nothing():
    p = Pair(8, 4, 4, 8)
    assert p.resize([0, 1], [12, 16]) == 0
    assert p.resize([2, 0, 3], [4, 0, 21]) == 3
    assert p.resize([2, 3], [9, 4]) == 3
    assert p.resize([0, 2], [0, 16]) == 0
    assert p.resize([3], [33]) == -1
    assert p.resize([3, 1], [33, 0]) == -1
    assert p.resize([3], [1]) == 1


@pytest.mark.parametrize("pages", [1, 15, 16, 17, 4095, 16384, 16385, 40000])
def test_free_pages_are_found_and_moved_at_all_places(pages):
    rng = random.Random(pages)
    p = Pair(pages, 1, 4, pages, pools=1, values=8)
    p.resize([0, 1], [pages // 2, pages - pages // 2])
    keep = sorted(rng.sample(range(pages), max(1, pages // 3)))
    # give back a random half of the pages: a book put together by hand
    refs = [0] * pages
    for k in keep:
        refs[k] = 1
    table = [keep + [0] * (pages - len(keep))] + [[0] * pages for _ in range(3)]
    p.want.refs, p.want.lens, p.want.table = refs, [len(keep), 0, 0, 0], table
    p.book.refs.copy_(ints(refs))
    p.book.lens.copy_(ints(p.want.lens))
    p.book.table.copy_(torch.tensor(table, dtype=torch.int32))
    half = (pages - len(keep)) // 2
    p.resize([2], [half])
    p.resize([3], [pages - len(keep) - half])
    p.resize([1], [1])
    p.resize([0], [0])
    p.compact()


def test_many_entries_and_long_rows():
    """More entries than one block holds, and pages given back by many blocks at once."""
    slots, cols = 3000, 40
    p = Pair(1 << 17, 2, slots, cols, pools=1, values=8)
    rng = random.Random(5)
    order = list(range(slots))
    rng.shuffle(order)
    p.resize(order, [rng.randint(0, 2 * cols) for _ in order])
    p.fork([rng.randrange(slots) for _ in order], order)
    p.resize(order, [max(0, min(2 * cols, n + rng.randint(-30, 2))) for n in (p.want.lens[s] for s in order)])
    p.resize(order, [0] * slots)
    assert not any(p.want.refs)


def test_the_largest_book():
    pages = 1 << 20
    book = B.PageBook(pages, 1, 2, pages)
    n = B.pages_resize_scratch_bytes(book, 2)
    scratch, result = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    s = torch.cuda.current_stream()
    B.pages_resize(book, None, None, ints([pages - 5, 5]), 2, result, scratch, n, s)
    assert result.item() == 0 and bool((book.refs == 1).all())
    assert torch.equal(book.table[0, :pages - 5], torch.arange(pages - 5, dtype=torch.int32, device="cuda"))
    B.pages_resize(book, None, None, ints([3, 10]), 2, result, scratch, n, s)
    assert result.item() == 0 and book.table[1, 5:10].tolist() == [3, 4, 5, 6, 7]
    B.pages_resize(book, None, None, ints([2, 8]), 2, result, scratch, n, s)
    m = B.pages_compact_scratch_bytes(book)
    scratch = torch.empty(m, dtype=torch.uint8, device="cuda")
    B.pages_compact(book, None, result, scratch, m, s)
    assert result.item() == 10 and book.table[1, :8].tolist() == [2, 6, 7, 8, 9, 3, 4, 5]
    assert book.refs.nonzero().flatten().tolist() == list(range(10))
    # lengths that no number of pages suffices for
    B.pages_resize(book, None, None, ints([pages, pages]), 2, result, torch.empty(n, dtype=torch.uint8, device="cuda"), n, s)
    assert result.item() == (pages - 2) + (pages - 8) - (pages - 10)


def test_a_book_that_contradicts_itself_stays_inside_its_arrays():
    """Page numbers and lengths that mean nothing: wrong books come out, but no access outside (the guards around the arrays
    and the pools' other pages stay as they are)."""
    book = B.PageBook(50, 4, 6, 5)
    book.refs.random_(-3, 4)
    book.lens.copy_(ints([100, -7, 1 << 30, 6, 20, 3]))
    book.table.random_(-100, 100)
    data = torch.randn(50, 4, 8, device="cuda").half()
    pools = B.page_pools([data])
    s = torch.cuda.current_stream()
    for n, call in ((6, lambda b, k: B.pages_resize(book, pools, None, ints([21, 3, 0, 19, 20, 9][:6]), 6, None, b, k, s)),
                    (6, lambda b, k: B.pages_resize(book, pools, None, ints([1, 1, 19, 2, 3, 4]), 6, None, b, k, s)),
                    (6, lambda b, k: B.pages_fork(book, ints([2, 3, 9, 0, -1, 5]), ints([0, 1, 2, 3, 4, 5]), 6, b, k, s))):
        size = max(B.pages_resize_scratch_bytes(book, n), B.pages_fork_scratch_bytes(book, n))
        buf = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        call(buf, size)
        assert bool((buf[size:] == 0xA5).all())
    size = B.pages_compact_scratch_bytes(book)
    buf = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    B.pages_compact(book, pools, None, buf, size, s)
    assert bool((buf[size:] == 0xA5).all())
    assert not book.data[50:52].any() and not book.data[58:60].any() and not book.data[90:].any()


@pytest.mark.parametrize("pools", [1, 3, 130])
@pytest.mark.parametrize("values", [8, 1000, 20000])
def test_copies(pools, values):
    pages, gen = 23, torch.Generator(device="cuda").manual_seed(values)
    if pools > 3 and values > 1000:
        pages = 9
    data = [torch.randint(-30000, 30000, (pages, values + 8 * (i % 3)), generator=gen, device="cuda", dtype=torch.int16) for i in range(pools)]
    src, dst = [0, 5, 5, 99, 3, -1, 8, 7], [1, 2, 4, 6, 3, 6, 1 << 30, 6]
    want = [t.clone() for t in data]
    for t in want:
        t[[1, 2, 4, 6]] = t[[0, 5, 5, 7]]
    B.pages_copy(B.page_pools(data), ints(src), ints(dst), len(src), torch.cuda.current_stream())
    for a, b in zip(data, want):
        assert torch.equal(a, b)


def test_copies_of_parts_and_far_pages():
    """Keys and values side by side as two pools, and pages more than 2^31 bytes from the start."""
    joint = torch.randn(10, 2, 16, 4, 64, device="cuda").bfloat16()
    want = joint.clone()
    want[7, 0], want[7, 1] = joint[2, 0], joint[2, 1]
    B.pages_copy(B.page_pools([joint[:, 0], joint[:, 1]]), ints([2]), ints([7]), 1, torch.cuda.current_stream())
    assert torch.equal(joint, want)
    buf = torch.empty(300 << 23, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (300, 4096), (1 << 23, 1))
    far.normal_()
    want = far.clone()
    want[299], want[1] = far[0], far[298]
    B.pages_copy(B.page_pools([far]), ints([0, 298]), ints([299, 1]), 2, torch.cuda.current_stream())
    assert torch.equal(far, want)


def test_captured_and_replayed():
    """A graph of fork, resize and compact, replayed on a book that is put back in between."""
    p = Pair(100, 8, 8, 6)
    p.resize(None, [13, 20, 0, 3, 40, 8, 9, 17])
    start, pools = p.book.data.clone(), [t.clone() for t in p.data]
    src, dst, want = ints([4, 0, 0, 1]), ints([2, 5, 0, 4]), ints([14, 21, 41, 4, 21, 14, 0, 18])
    n = max(B.pages_fork_scratch_bytes(p.book, 4), B.pages_resize_scratch_bytes(p.book, 8), B.pages_compact_scratch_bytes(p.book))
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")

    def step():
        s = torch.cuda.current_stream()
        B.pages_fork(p.book, src, dst, 4, scratch, n, s)
        B.pages_resize(p.book, p.pools, None, want, 8, p.result, scratch, n, s)
        B.pages_compact(p.book, p.pools, p.result, scratch, n, s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    p.want.fork([4, 0, 0, 1], [2, 5, 0, 4])
    result, pairs = p.want.resize(None, want.tolist())
    assert result == 0 and pairs
    p.moved(pairs)
    p.moved(p.want.compact()[1])
    for _ in range(3):
        p.book.data.copy_(start)
        for t, k in zip(p.data, pools):
            t.copy_(k)
        graph.replay()
        p.buf = torch.full((64,), 0xA5, dtype=torch.uint8)
        p.check()
