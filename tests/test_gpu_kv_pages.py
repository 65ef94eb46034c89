"""kv_fork, kv_reserve, kv_compact and kv_copy against the same bookkeeping on lists (kv_pages_util.py): whole numbers and copies, equal
throughout."""
import random

import pytest

from kv_pages_util import BAD_BATCH, BAD_PAGE, BLOCK, NO_PAGE, Book

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def L(torch):
    import paper_2208_07339_amd as L
    return L


def ints(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Both:
    """The device's state beside the book's."""

    def __init__(self, torch, L, pages, refs, kv_len, slots, page_tokens):
        self.torch, self.L = torch, L
        self.book = Book(pages, refs, kv_len, slots, page_tokens)
        self.pool = L.KvPool(ints(torch, refs), page_tokens)
        self.seqs = L.KvSeqs(ints(torch, pages), ints(torch, kv_len), ints(torch, slots), ints(torch, [0]))
        self.moves = L.KvMoves.allocate(max(len(kv_len), len(refs)), len(kv_len))

    @staticmethod
    def random(torch, L, r, n, stride, n_pages, page_tokens, most=None):
        """Sequences that share some pages with those before them; the rest of the pool is free."""
        order = list(range(n_pages))
        r.shuffle(order)
        refs, pages, kv_len = [0] * n_pages, [], []
        for b in range(n):
            k = r.randint(0, stride)
            row = [-1] * stride
            shared = r.randint(0, k) if b and r.random() < 0.6 else 0
            other = pages[r.randrange(b)] if b else None
            for j in range(k):
                if j < shared and other[j] >= 0:
                    row[j] = other[j]
                elif order and (most is None or len(order) > n_pages - most):
                    row[j] = order.pop()
            held = next((j for j, e in enumerate(row) if e < 0), stride)
            row = [e if j < held else -1 for j, e in enumerate(row)]
            for e in row[:held]:
                refs[e] += 1
            pages.append(row)
            kv_len.append(r.randint(max(0, held - 1) * page_tokens, held * page_tokens))
        slots = list(range(n + 3))
        r.shuffle(slots)
        return Both(torch, L, pages, refs, kv_len, slots[:n], page_tokens)

    def check(self, tables=True):
        b = self.book
        assert self.seqs.kv_len.tolist() == b.kv_len
        assert self.seqs.slots.tolist() == b.slots
        assert self.pool.refs.tolist() == b.refs
        assert self.seqs.pages.tolist() == b.pages
        np, ns = self.moves.count.tolist()
        assert (np, ns) == (len(b.page_moves), len(b.slot_moves))
        assert self.moves.pages[:np].tolist() == b.page_moves
        assert self.moves.slots[:ns].tolist() == b.slot_moves
        assert self.seqs.status.item() == b.status

    def fork(self, parent, grow=0):
        self.L.kv_fork(self.pool, self.seqs, ints(self.torch, parent), self.moves, grow=grow)
        self.book.fork(parent, grow)

    def reserve(self, rows, more=False):
        start = [0]
        for x in rows:
            start.append(start[-1] + x)
        ready = ints(self.torch, [-7] * len(rows))
        self.L.kv_reserve(self.pool, self.seqs, ints(self.torch, start), self.moves, ready=ready, more=more)
        assert ready.tolist() == self.book.reserve(start, more)

    def compact(self):
        used = ints(self.torch, [-7])
        self.L.kv_compact(self.pool, self.seqs, self.moves, used=used)
        assert used.item() == self.book.compact()

    def set_len(self, kv_len):
        self.seqs.kv_len.copy_(ints(self.torch, kv_len))
        self.book.kv_len = list(kv_len)


@pytest.mark.parametrize("n, stride, seed", [(1, 1, 0), (1, 70, 1), (4, 21, 2), (5, 1, 3), (16, 300, 4), (63, 9, 5), (64, 5, 6), (65, 17, 7),
                                             (128, 79, 8), (257, 6, 9), (1000, 3, 10), (2048, 2, 11), (2047, 5, 12)])
def test_fork(torch, L, n, stride, seed):
    r = random.Random(seed)
    s = Both.random(torch, L, r, n, stride, n * stride + 5, 64)
    for parent in ([r.randrange(n) for _ in range(n)], [r.randint(-1, n - 1) for _ in range(n)], list(range(n)),
                   [0] * n, [n - 1] * n, list(range(1, n)) + [-1], [-1] * n):
        s.fork(parent, grow=r.choice([0, 1, 5]))
        s.check()
        assert s.book.refs == s.book.counted() and len(set(s.book.slots)) == n


def test_fork_what_cannot_be(torch, L):
    pages = [[0, 1, -1], [0, 9, -5], [2 ** 31 - 1, 3, -1], [-2 ** 31, -1, -1]]
    s = Both(torch, L, pages, [2, 1, 0, 1, 0], [100, -3, 2 ** 31 - 1, 40], [3, 1, 0, 2], 64)
    s.fork([0, 1, 2, 3])
    assert s.book.status == BAD_BATCH | BAD_PAGE
    s.check()
    s.fork([1, 1, 2, 2], grow=1)
    s.check()
    s.fork([4, -2, 2 ** 31 - 1, 0])
    s.check()
    assert s.book.kv_len == [0, 0, 0, -3] and s.book.pages[3] == [0, -1, -1]


@pytest.mark.parametrize("n, stride, page, seed", [(1, 3, 32, 0), (4, 21, 64, 1), (5, 9, 96, 2), (16, 300, 32, 3), (64, 5, 256, 4), (129, 7, 64, 5),
                                                   (1000, 4, 96, 6), (2048, 3, 64, 7), (2, 3000, 32, 8)])
def test_reserve(torch, L, n, stride, page, seed):
    """Single tokens, prompts, drafted tokens taken back, sequences that bring nothing; with pages enough."""
    r = random.Random(seed)
    s = Both.random(torch, L, r, n, stride, 3 * n * stride + 70, page)
    for step in range(6):
        most, rows, kv_len = stride * page, [], []
        for length in s.book.kv_len:
            kind = r.random()
            if kind < 0.3:
                length, x = length + 1, 1
            elif kind < 0.5:
                x = r.randint(1, 3 * page)
                length += x
            elif kind < 0.7:  # shorter, and on from there
                length = r.randint(0, length)
                x = r.choice([1, 31, 32, 33, page, 2 * page + 1])
                length += x
            elif kind < 0.8:
                x = length  # all of it again
            else:
                x = 0
            if length > most:
                length, x = most, min(x, most)
            rows.append(x), kv_len.append(length)
        s.set_len(kv_len)
        s.reserve(rows, more=step % 2 == 1)
        s.check()
        assert s.book.refs == s.book.counted() and not s.book.status
        s.fork([r.randrange(n) if r.random() < 0.5 else i for i in range(n)])
        s.check()


@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("share", [2, 3, 8])
def test_reserve_beams_in_step(torch, L, page, share):
    """Beams of an item that share everything get tokens one by one: pages of their own when a block gets full, but for the last."""
    n, stride = 2 * share, 5
    s = Both(torch, L, [[-1] * stride] * n, [0] * 64, [0] * n, list(range(n)), page)
    s.set_len([70] + [0] * (share - 1) + [33] + [0] * (share - 1))
    s.reserve([70] + [0] * (share - 1) + [33] + [0] * (share - 1))
    s.check()
    s.fork([0] * share + [share] * share, grow=1)
    for step in range(70):
        before = s.book.refs.count(0)
        s.reserve([1] * n, more=True)
        s.check()
        # what is not shared any more: at most one page a beam and step, none where the last holder keeps its page
        assert before - s.book.refs.count(0) <= n
        parent = list(range(n))
        if step % 9 == 0:
            parent = [1] * share + list(range(share, n))
        s.fork(parent, grow=1)
        s.check()
    assert s.book.refs == s.book.counted() and not s.book.status


def test_reserve_too_few_pages(torch, L):
    page, n, stride = 64, 6, 8
    for free in range(0, 14):
        s = Both(torch, L, [[-1] * stride] * n, [0] * (4 + free), [0] * n, list(range(n)), page)
        s.set_len([95, 0, 0, 0, 0, 0])
        s.reserve([95, 0, 0, 0, 0, 0])
        s.fork([0, 0, 0, -1, -1, -1], grow=1)  # three share a page in which a block gets full
        s.set_len(s.book.kv_len[:3] + [130, 64, 0])
        s.reserve([1, 1, 1, 130, 64, 0])
        s.check()
        assert s.book.refs == s.book.counted()
        assert bool(s.book.status & NO_PAGE) == (free < 4)
    # shared pages behind the first, which a shortened sequence writes anew
    for free in range(0, 7):
        s = Both(torch, L, [[-1] * stride] * n, [0] * (4 + free), [0] * n, list(range(n)), page)
        s.set_len([250, 0, 0, 0, 0, 0])
        s.reserve([250, 0, 0, 0, 0, 0])
        s.fork([0, 0, -1, -1, -1, -1])
        s.set_len([250, 231, 0, 0, 0, 0])
        s.reserve([0, 200, 0, 0, 0, 0])
        s.check()
        # positions 31 .. 230 fill blocks 0 .. 6, which are in four pages
        assert s.book.refs == s.book.counted() and bool(s.book.status & NO_PAGE) == (free < 4)


def test_reserve_what_cannot_be(torch, L):
    pages = [[0, 1, -1], [99, -1, -1], [-1, -1, -1], [2, -1, -1], [-1] * 3, [-1] * 3, [-1, 7, -9]]
    s = Both(torch, L, pages, [1, 1, 1] + [0] * 40, [200, 20, 5, -1, 40, 2 ** 31 - 1, 130], list(range(7)), 64)
    # beyond the table; a page that does not exist; fewer positions than rows; a negative length; rows that fall; too long; fine
    start = [0, 60, 80, 90, 91, 90, 95, 225]
    ready = ints(torch, [-7] * 7)
    L.kv_reserve(s.pool, s.seqs, ints(torch, start), s.moves, ready=ready)
    assert ready.tolist() == s.book.reserve(start) == [0, 20, 0, 0, 0, 0, 130]
    s.check()
    assert s.book.status == BAD_BATCH | BAD_PAGE


@pytest.mark.parametrize("n_pages, seed", [(1, 0), (63, 1), (64, 2), (65, 3), (255, 4), (257, 5), (5000, 6), (10241, 9), (65536, 7), (131072, 8)])
def test_compact(torch, L, n_pages, seed):
    r = random.Random(seed)
    n, stride = (8, 40) if n_pages < 50000 else (40, 3000)
    s = Both.random(torch, L, r, n, stride, n_pages, 32)
    for _ in range(2):
        s.compact()
        s.check()
        assert s.book.refs == s.book.counted()
        used = sum(c > 0 for c in s.book.refs)
        assert all(s.book.refs[:used])
        s.fork([i if r.random() < 0.6 else -1 for i in range(n)])
    s.fork([-1] * n)
    s.compact()
    s.check()
    assert not any(s.book.refs)


def test_a_pool_of_the_largest_size(torch, L):
    """The last pages of the largest pool are given, shared, found and moved."""
    n_pages = L.KV_MAX_PAGES
    refs = [1] * (n_pages - 3) + [0, 1, 0]  # held by the program itself
    s = Both(torch, L, [[-1] * 3] * 2, refs, [64, 0], [0, 1], 32)
    s.reserve([64, 0])
    s.check()
    assert s.book.pages[0] == [n_pages - 3, n_pages - 1, -1]
    s.set_len([65, 0])
    s.reserve([1, 0])
    s.check()
    assert s.book.status == NO_PAGE


def filled(torch, L, g, n_pages, page, n_slots, heads, d):
    c = L.KvCache.allocate(n_pages, page, n_slots, heads, d)
    c.codes.copy_(torch.randint(-127, 128, c.codes.shape, dtype=torch.int8, device="cuda", generator=g))
    c.consts.copy_(torch.rand(c.consts.shape, device="cuda", generator=g))
    c.ring.copy_(torch.randn(c.ring.shape, device="cuda", generator=g))
    return c


def bits(torch, c):
    return [c.codes.clone(), c.consts.clone().view(torch.int16), c.ring.clone().view(torch.int16)]


@pytest.mark.parametrize("heads, d, page", [(1, 64, 32), (2, 80, 96), (3, 128, 64), (5, 1, 64), (2, 33, 128), (1, 100, 64), (2, 256, 32), (40, 128, 64),
                                            (7, 8, 256)])
def test_copy(torch, L, heads, d, page):
    g = torch.Generator(device="cuda")
    g.manual_seed(heads * 1000 + d)
    r = random.Random(d)
    n_pages, n_slots, per = 23, 19, page // BLOCK
    c = filled(torch, L, g, n_pages, page, n_slots, heads, d)
    want = bits(torch, c)
    order, rings = r.sample(range(n_pages), 14), r.sample(range(n_slots), 18)
    pages = [[order[i % 3], order[3 + i], r.randint(0, per), 0] for i in range(11)]
    slots = []
    for i, (first, count) in enumerate([(0, 0), (0, 1), (0, 63), (32, 63), (64, 33), (96, 40), (32, 32), (2 ** 20, 45), (0, 64), (63, 2), (32, 33)]):
        slots.append([rings[i % 3], rings[3 + i], first, count])
    m = L.KvMoves(ints(torch, pages + [[0, 1, 1, 0]]), ints(torch, slots + [[0, 1, 0, 9]]), ints(torch, [len(pages), len(slots)]))
    status = ints(torch, [0])
    L.kv_copy(c, m, status)
    for f, t, k, _ in pages:
        want[0][t, :, :k] = want[0][f, :, :k]
        want[1][t, :, :k] = want[1][f, :, :k]
    for f, t, first, count in slots:
        at = [(first + i) % 64 for i in range(count)]
        want[2][t][:, :, at] = want[2][f][:, :, at]
    for x, y in zip(bits(torch, c), want):
        assert torch.equal(x, y)
    assert status.item() == 0


def test_copy_what_cannot_be(torch, L):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    c = filled(torch, L, g, 4, 64, 3, 2, 64)
    want = bits(torch, c)
    m = L.KvMoves(ints(torch, [[4, 0, 1, 0], [0, -1, 1, 0], [0, 1, 3, 0], [0, 1, -1, 0], [2, 3, 2, 0]]),
                  ints(torch, [[3, 0, 0, 5], [0, -1, 0, 5], [0, 1, 0, 65], [0, 1, 0, -1], [0, 1, -1, 5]]), ints(torch, [5, 5]))
    status = ints(torch, [0])
    L.kv_copy(c, m, status)
    assert status.item() == BAD_PAGE | BAD_BATCH
    want[0][3], want[1][3] = want[0][2], want[1][2]
    assert all(torch.equal(x, y) for x, y in zip(bits(torch, c), want))
    for count in ([-1, -5], [0, 0]):
        L.kv_copy(c, L.KvMoves(m.pages, m.slots, ints(torch, count)))
    L.kv_copy(c, L.KvMoves(m.pages[4:], m.slots[:1], ints(torch, [2 ** 31 - 1, 0])))  # a count beyond the list: the list's end
    assert all(torch.equal(x, y) for x, y in zip(bits(torch, c), want))


def test_copy_beyond_32_bits(torch, L):
    """Pages and slots whose places are beyond 2^31 elements."""
    heads, d = 4, 128
    c = L.KvCache.allocate(70000, 64, 70000, heads, d)  # 4.6 GB of codes, 9.2 GB of ring
    c.codes[7], c.codes[69999], c.codes[69998] = 3, 5, 9
    c.ring[8], c.ring[69999], c.ring[69990] = 1.5, 2.5, 3.5
    m = L.KvMoves(ints(torch, [[69999, 7, 2, 0], [69998, 69997, 1, 0]]), ints(torch, [[69999, 8, 0, 64], [69990, 69991, 32, 64]]), ints(torch, [2, 2]))
    L.kv_copy(c, m)
    assert bool((c.codes[7] == 5).all()) and bool((c.codes[69997][:, 0] == 9).all()) and bool((c.codes[69998] == 9).all())
    assert bool((c.ring[8] == 2.5).all()) and bool((c.ring[69991] == 3.5).all())


def test_another_stream_and_replays(torch, L):
    """A fork with its pages and copies, captured once, replayed with other parents and eager work between."""
    r = random.Random(5)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    n, stride, page = 12, 6, 64
    s = Both.random(torch, L, r, n, stride, 200, page)
    s.set_len([max(1, x) for x in s.book.kv_len])
    c = filled(torch, L, g, 200, page, n + 3, 2, 64)
    parent, rows = ints(torch, list(range(n))), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        L.kv_fork(s.pool, s.seqs, parent, s.moves)
        L.kv_reserve(s.pool, s.seqs, rows, s.moves, more=True)
        L.kv_copy(c, s.moves)
    for step in range(8):
        p = [r.randrange(n) for _ in range(n)]
        lengths = [min(stride * page, x + r.randint(0, 40)) for x in s.book.kv_len]
        s.set_len(lengths)
        # (pages for the positions that the lengths went up by)
        s.reserve([max(0, min(x, 40)) for x in lengths])
        s.check()
        want = bits(torch, c)
        parent.copy_(ints(torch, p))
        torch.cuda.synchronize()
        graph.replay()
        s.book.fork(p)
        s.book.reserve(list(range(n + 1)), more=True)
        s.check()
        for f, t, k, _ in s.book.page_moves:
            want[0][t, :, :k], want[1][t, :, :k] = want[0][f, :, :k], want[1][f, :, :k]
        for f, t, first, count in s.book.slot_moves:
            at = [(first + i) % 64 for i in range(count)]
            want[2][t][:, :, at] = want[2][f][:, :, at]
        assert all(torch.equal(x, y) for x, y in zip(bits(torch, c), want))
