"""kv_reserve: the table of a sequence that is not served stays as it is, entries that name no page of the pool included, and a later call
tells of them again."""
import pytest

from kv_pages_util import BAD_PAGE, NO_PAGE
from test_gpu_kv_served import Served, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [8, 9, 2 ** 31 - 1])
@pytest.mark.parametrize("negative", [-1, -2, -5, -100, -(2 ** 31) + 2 ** 20])
def test_entries_behind_the_first(bad, negative):
    import torch

    import paper_2208_07339_amd as L
    # one page in use (shared, to be replaced by the first sequence), and few free ones
    for n_pages, served in ((3, False), (8, True)):
        pages = [[0, 1, bad, negative, negative, -1], [0, 1, -1, -1, -1, negative]]
        s = Served(torch, L, pages, [2, 2] + [0] * (n_pages - 2), [150, 64], [0, 1], 32)
        rows = [149, 0]  # positions 1 .. 149: pages 0 to 4, of which 0 and 1 are the other's too
        for turn in range(2):
            s.seqs.status.zero_()
            s.book.status = 0
            assert s.reserve(rows) == [150 if served else 0, 64]
            s.check()
            if served:
                assert s.book.status == BAD_PAGE
                break
            assert s.book.status == BAD_PAGE | NO_PAGE and s.seqs.pages.tolist() == pages
        # and with pages enough, which another sequence gives back
        if not served:
            s = Served(torch, L, s.seqs.pages.tolist(), [2, 2] + [0] * 6, [150, 64], [0, 1], 32)
            assert s.reserve(rows) == [150, 64]
            s.check()


def test_the_lowest_numbers_name_no_page_either():
    """-2^31 and those next to it, where a sequence is served and where it is not (then -1 may take their place)."""
    import torch

    import paper_2208_07339_amd as L
    low = -(2 ** 31)
    for n_pages, served in ((4, False), (8, True)):
        s = L.KvSeqs(ints(torch, [[0, 1, low, low + 1, low + n_pages]]), ints(torch, [150]), ints(torch, [0]), ints(torch, [0]))
        pool, moves, ready = L.KvPool(ints(torch, [1, 2] + [0] * (n_pages - 2)), 32), L.KvMoves.allocate(8, 1), ints(torch, [-7])
        L.kv_reserve(pool, s, ints(torch, [0, 149]), moves, ready=ready)
        got = s.pages.tolist()[0]
        if served:  # page 1 is shared, by the program, and to be written to
            assert ready.item() == 150 and s.status.item() == 0 and got == [0, 2, 3, 4, 5]
            assert pool.refs.tolist() == [1, 1, 1, 1, 1, 1, 0, 0]
        else:
            assert ready.item() == 0 and s.status.item() == NO_PAGE and got[:2] == [0, 1] and max(got[2:]) < 0
            assert pool.refs.tolist() == [1, 2, 0, 0]
