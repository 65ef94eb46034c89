"""kv_reserve where pages are too few: what a sequence that is not served holds stays as it is, its data too, whatever the others write."""
import random

import pytest

from kv_pages_util import BLOCK, NO_PAGE
from kv_served_util import ServedBook, full_blocks, written_over
from test_gpu_kv_pages import Both, ints

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


class Served(Both):
    def __init__(self, torch, L, pages, refs, kv_len, slots, page_tokens):
        super().__init__(torch, L, pages, refs, kv_len, slots, page_tokens)
        self.book = ServedBook(pages, refs, kv_len, slots, page_tokens)

    def reserve(self, rows, more=False):
        start = [0]
        for x in rows:
            start.append(start[-1] + x)
        ready = ints(self.torch, [-7] * len(rows))
        self.L.kv_reserve(self.pool, self.seqs, ints(self.torch, start), self.moves, ready=ready, more=more)
        got = ready.tolist()
        # of what the device gives, not of what the book says
        assert written_over(self.seqs.pages.tolist(), got, full_blocks(self.seqs.kv_len.tolist(), rows), rows, self.book.page) == []
        assert got == self.book.reserve(start, more)
        return got


def test_the_last_holder_is_shorter(torch, L):
    """Two share 95 positions; the last, shortened to 63, would write the second block, which the first holds and gets no page for."""
    s = Served(torch, L, [[0], [0]], [2], [96, 64], [0, 1], 128)
    assert s.reserve([1, 1]) == [0, 0]
    s.check()
    assert s.book.status == NO_PAGE and s.book.pages == [[0], [0]] and s.book.refs == [2]
    # of one length, or the last longer: what it writes is not the other's
    for lengths in ([96, 96], [64, 96]):
        s = Served(torch, L, [[0], [0]], [2], lengths, [0, 1], 128)
        assert s.reserve([1, 1]) == [0, lengths[1]]
        s.check()
    # a page for the first: the last keeps the one that they share
    s = Served(torch, L, [[0], [0]], [2, 0], [96, 64], [0, 1], 128)
    assert s.reserve([1, 1]) == [96, 64]
    s.check()
    assert s.book.pages == [[1], [0]]


@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("n, seed", [(3, 0), (9, 1), (70, 2), (400, 3), (1500, 4)])
def test_sharers_of_different_lengths(torch, L, n, page, seed):
    """Groups that share their pages, each sequence of its own length, all of which bring tokens; from no free page to enough."""
    r = random.Random(100 * seed + page)
    demoted = 0
    for turn in range(8):
        stride, per = 6, page // BLOCK
        pages, lengths, rows, count = [], [], [], 0
        while len(pages) < n:
            k, size = r.randint(1, 3), r.randint(1, 5)
            row = list(range(count, count + k)) + [-1] * (stride - k)
            count += k
            top = r.randint((k - 1) * page + 1, k * page - 1)
            for _ in range(min(size, n - len(pages))):
                old = r.choice([top, max(0, top - r.randint(0, 32)), top // BLOCK * BLOCK, r.randint(0, top // BLOCK) * BLOCK])
                x = r.choice([0, 1, 1, BLOCK - old % BLOCK, r.randint(1, 40)])
                pages.append(list(row)), rows.append(x), lengths.append(old + x)
        order = list(range(len(pages)))
        r.shuffle(order)  # (groups side by side or apart)
        if turn % 2:
            pages, lengths, rows = ([v[i] for i in order] for v in (pages, lengths, rows))
        free = r.choice([0, 0, 1, 2, n // 3, n // 2, 2 * n])
        number = list(range(count + free))
        r.shuffle(number)
        pages = [[number[e] if e >= 0 else -1 for e in row] for row in pages]
        refs = [0] * (count + free)
        for row in pages:
            for e in row:
                if e >= 0:
                    refs[e] += 1
        if turn == 3:
            refs[number[0]] += 1  # the program holds a page, too
        s = Served(torch, L, pages, refs, lengths, list(range(n)), page)
        got = s.reserve(rows)
        s.check()
        demoted += got.count(0)
        # a second call for those that were not served, with the pages that have become free
        s.reserve([y if x == 0 else 0 for x, y in zip(got, rows)])
        s.check()
    assert demoted


@pytest.mark.parametrize("heads, d, page", [(2, 64, 128), (3, 40, 64), (1, 128, 256)])
def test_what_the_others_hold_is_not_written_to(torch, L, heads, d, page):
    """Forks of one prompt, the last of them shortened, with no page left: caches as if each had been filled by itself; then a page is there and
    all go on."""
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    n, most = 3, page + 6
    length = page - 1
    x = torch.randn(2, n, most, heads, d, device="cuda", generator=g).half()
    x[:, 1:, :length] = x[:, :1, :length]
    old = [length, length, length - 32]
    y = torch.randn(2, n, most, heads, d, device="cuda", generator=g).half()
    for b in range(n):
        x[:, b, old[b]:] = y[:, b, old[b]:]
    n_pages = 3
    cache = L.KvCache.allocate(n_pages, page, n, heads, d)
    pool, seqs, moves = L.KvPool.allocate(n_pages, page), L.KvSeqs.allocate(n, 2), L.KvMoves.allocate(n, n)
    ready, status = ints(torch, [-7] * n), ints(torch, [0])
    pool.refs[1:] += 1  # pages that the program holds

    def put(rows, first):
        start = ints(torch, [sum(rows[:b]) for b in range(n + 1)])
        seqs.kv_len.copy_(ints(torch, [f + m for f, m in zip(first, rows)]))
        L.kv_reserve(pool, seqs, start, moves, ready=ready)
        L.kv_copy(cache, moves, status)
        k, v = (torch.cat([x[w, b, f:f + m] for b, (f, m) in enumerate(zip(first, rows))]) for w in range(2))
        L.kv_append(cache, L.KvBatch(start, ready, seqs.pages, seqs.slots, sum(rows), max(rows), most, status), k, v)
        return ready.tolist()

    def held(lengths):
        """What the cache has of every sequence, and what one of its own would have."""
        start = ints(torch, [sum(lengths[:b]) for b in range(n + 1)])
        plain, pages = L.KvCache.allocate(2 * n, page, n, heads, d), torch.arange(2 * n, dtype=torch.int32, device="cuda").view(n, 2)
        b = L.KvBatch(start, ints(torch, lengths), pages, None, sum(lengths), max(lengths), most)
        k, v = (torch.cat([x[w, q, :lengths[q]] for q in range(n)]) for w in range(2))
        L.kv_append(plain, b, k, v)
        got = L.kv_read(cache, L.KvBatch(start, ints(torch, lengths), seqs.pages, seqs.slots, sum(lengths), max(lengths), most, status))
        return got, L.kv_read(plain, b)

    assert put([length, 0, 0], [0, 0, 0]) == [length, 0, 0]
    L.kv_fork(pool, seqs, ints(torch, [0, 0, 0]), moves)
    L.kv_copy(cache, moves, status)
    rows = [1, 1, 1]  # all fill their open block, the last one the block before the others'
    got = put(rows, old)
    assert got == [0, 0, 0] and seqs.status.item() == NO_PAGE
    for a, b in zip(*held(old)):
        assert torch.equal(a, b)
    # one page: the second and the last are still left out
    pool.refs[1] -= 1
    got = put(rows, old)
    assert got == [old[0] + rows[0], 0, 0]
    for a, b in zip(*held([got[0], old[1], old[2]])):
        assert torch.equal(a, b)
    pool.refs[2] -= 1
    got = put([0, rows[1], rows[2]], [got[0], old[1], old[2]])
    assert got == [o + m for o, m in zip(old, rows)]
    for a, b in zip(*held(got)):
        assert torch.equal(a, b)
    assert status.item() == 0 and pool.refs.tolist() == [1, 1, 1]
