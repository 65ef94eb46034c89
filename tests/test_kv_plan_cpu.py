"""How kv_attention cuts calls up (llmint8_debug_kv_plan_for): host arithmetic, no GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def L():
    import os

    import paper_2208_07339_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2208_07339_amd.build import build
        build()
    L.lib()
    return L


def plan(L, seqs, n_rows, max_rows, max_len, heads_q, heads, d, window=0):
    """-> (rows to a tile, parts, halves, workgroups), or a status."""
    from paper_2208_07339_amd.binding import KvPlan, _KvBatch
    batch, p = _KvBatch(None, None, None, None, None, seqs, n_rows, 1, max_rows, max_len), KvPlan()
    status = L.lib().llmint8_debug_kv_plan_for(C.byref(batch), heads_q, heads, d, window, C.byref(p))
    return status or (p.tile, p.parts, p.halves, p.workgroups)


def test_forms(L):
    # one token: a tile of the kernel for few rows to each head, and parts where the axis is long
    assert plan(L, 1, 1, 1, 76, 12, 12, 64) == (32, 1, 0, 12)
    assert plan(L, 1, 1, 1, 4001, 40, 40, 128) == (32, 6, 0, 240)
    # rows of all query heads that share keys together
    assert plan(L, 64, 64, 1, 4101, 32, 8, 128) == (32, 1, 0, 512)
    # prompts: 128 rows, 256 where the axis is long, parts where rows are few, halves where the tiles are
    assert plan(L, 1, 2048, 2048, 2048, 32, 32, 128) == (128, 1, 0, 512)
    assert plan(L, 1, 8192, 8192, 8192, 40, 40, 128) == (256, 1, 0, 1280)
    assert plan(L, 1, 1024, 1024, 21035, 32, 8, 128) == (256, 2, 0, 256)
    assert plan(L, 1, 1500, 1500, 1500, 16, 16, 128) == (128, 1, 1, 192)
    assert plan(L, 1, 1500, 1500, 1500, 16, 16, 129)[2] == 0  # halves are for heads of up to 128
    # a window leaves less to see
    assert plan(L, 1, 2100, 2100, 4200, 32, 32, 64) == (256, 1, 0, 288)
    assert plan(L, 1, 2100, 2100, 4200, 32, 32, 64, 1000) == (128, 1, 0, 544)
    assert plan(L, 1, 2100, 2100, 4200, 32, 32, 64, 4201) == (256, 1, 0, 288)
    # max_rows beyond the rows that there are changes nothing
    assert plan(L, 1, 1, 4096, 4001, 40, 40, 128) == plan(L, 1, 1, 1, 4001, 40, 40, 128)


@pytest.mark.parametrize("window", [0, 1, 1000, 2 ** 31 - 1])
def test_parts_are_what_the_workspace_is_for(L, window):
    from paper_2208_07339_amd.binding import _KvBatch
    for seqs, rows, length, hq, h, d in [(1, 1, 4001, 40, 40, 128), (2, 1, 131072, 64, 8, 128), (1, 1024, 21035, 32, 8, 128), (3, 50, 9000, 8, 2, 200)]:
        batch = _KvBatch(None, None, None, None, None, seqs, seqs * rows, 1, rows, length)
        n = L.lib().llmint8_kv_attention_workspace_bytes(C.byref(batch), hq, h, d)
        parts = plan(L, seqs, seqs * rows, rows, length, hq, h, d, window)[1]
        need = parts * seqs * rows * hq * (4 * d + 8)
        assert parts == 1 or need < n
        assert window or n == need + 512


def test_refusals(L):
    assert plan(L, 1, 1, 1, 100, 4, 2, 64)[0] == 32
    for bad in ((0, 1, 1, 100, 4, 2, 64), (1, 0, 1, 100, 4, 2, 64), (1, 1, 0, 100, 4, 2, 64), (1, 1, 1, -1, 4, 2, 64), (1, 1, 1, 2 ** 30, 4, 2, 64),
                (1, 1, 1, 100, 3, 2, 64), (1, 1, 1, 100, 0, 0, 64), (1, 1, 1, 100, 4, 2, 0), (1, 1, 1, 100, 4, 2, 257), (1, 1, 1, 100, 4, 2, 64, -1)):
        assert plan(L, *bad) == 1, bad
    f = L.lib().llmint8_debug_kv_plan_for
    from paper_2208_07339_amd.binding import KvPlan, _KvBatch
    assert f(None, 4, 2, 64, 0, C.byref(KvPlan())) == 1
    assert f(C.byref(_KvBatch(None, None, None, None, None, 1, 1, 1, 1, 100)), 4, 2, 64, 0, None) == 1


def test_workgroups_without_rows(L):
    """The kernel for few rows is launched with the longest sequence's tiles for all: not where most of these would not be there."""
    # 256 sequences, one of 2 048 rows, the others of one: 131 072 workgroups for 2 303 rows
    assert plan(L, 256, 2303, 2048, 2048, 8, 8, 128, 128)[0] == 128
    assert plan(L, 4096, 4095 + 131072, 131072, 131072, 1, 1, 64, 1)[3] < 10000
    assert plan(L, 1, 1 << 28, 1 << 28, 0, 4, 4, 1)[3] * 256 < 1 << 32  # rows that see nothing
    for seqs in (1, 3, 64, 100, 1000):
        for rows in (33, 100, 1000, 10000):
            for length in (1, 100, 1000, 100000):
                for window in (0, 1, 100):
                    n = plan(L, seqs, seqs - 1 + rows, rows, length, 8, 8, 64, window)[3]
                    tiles = 8 * (seqs + rows // 32 + 1)  # of 32 rows, that there are
                    assert n <= max(512, tiles) + 8192, (seqs, rows, length, window, n)


@pytest.mark.parametrize("seqs, rows, length, heads_q, heads, form", [
    # more tiles of 256 rows than the chip holds at once: two halves where those of 128 rows are no more than two rounds
    (20, 96, 6000, 32, 8, (128, 1, 1)), (1, 2688, 8688, 24, 24, (128, 1, 1)),
    # behind a long past a second round of halves is as long as the first: one round of whole tiles
    (1, 1024, 6000, 40, 40, (256, 1, 0)), (1, 900, 16000, 40, 8, (256, 1, 0)), (4, 300, 4200, 24, 24, (256, 1, 0)), (40, 129, 5000, 4, 4, (256, 1, 0)),
    (3, 1500, 6000, 10, 10, (256, 1, 0)), (1, 1100, 3000, 40, 40, (128, 1, 0)), (2, 500, 3000, 40, 40, (128, 1, 0)),
    # one round of halves, or a second that is short
    (1, 1024, 8000, 32, 8, (128, 1, 1)), (60, 50, 5000, 8, 1, (128, 1, 1)), (1, 4096, 4096, 16, 16, (128, 1, 1)), (1, 8192, 8192, 8, 8, (128, 1, 1)),
    (1, 3000, 3000, 16, 16, (128, 1, 1))])
def test_halves_by_rounds(L, seqs, rows, length, heads_q, heads, form):
    assert plan(L, seqs, seqs * rows, rows, length, heads_q, heads, 128)[:3] == form


@pytest.mark.parametrize("seqs, rows, length, heads_q, heads, tiles, parts", [
    (1, 500, 500, 48, 1, 750, 1), (1, 100, 5000, 48, 1, 150, 1), (1, 1000, 1000, 16, 2, 500, 1), (1, 1000, 1000, 12, 12, 384, 1),
    (1, 20, 2000, 48, 1, 30, 8), (1, 500, 500, 32, 32, 512, 1), (1, 1, 4001, 40, 40, 40, 6)])
def test_workgroups_are_the_tiles_that_there_are(L, seqs, rows, length, heads_q, heads, tiles, parts):
    """Few parts: not rounded up to one for each XCD, which would leave XCDs without work."""
    assert plan(L, seqs, seqs * rows, rows, length, heads_q, heads, 128)[:4] == (32, parts, 0, tiles * parts)


@pytest.mark.parametrize("d, most", [(128, 512), (129, 256), (256, 256)])
def test_parts_of_several_sequences_are_one_round(L, d, most):
    """Heads of more than 128 leave registers for one workgroup to a compute unit, others for two."""
    for seqs, rows, length, heads_q, heads in [(8, 6, 4000, 16, 2), (2, 1, 100000, 16, 2), (30, 1, 3000, 16, 2), (3, 1, 5000, 16, 16), (32, 5, 1000, 16, 2)]:
        tile, parts, _, workgroups = plan(L, seqs, seqs * rows, rows, length, heads_q, heads, d)
        assert tile == 32 and parts > 1 and most * 3 // 4 <= workgroups <= most, (seqs, parts, workgroups)


@pytest.mark.parametrize("seqs, rows, length, heads_q, heads, d, window, tile", [
    (12, 100, 1000, 24, 24, 128, 100, 128), (1, 1900, 1900, 32, 32, 80, 100, 128), (10, 200, 200, 40, 40, 128, 0, 128), (7, 301, 350, 16, 2, 256, 0, 128),
    (1, 1000, 1000, 32, 32, 256, 100, 128), (1, 3000, 3000, 48, 1, 128, 16, 128),
    # two rounds, or fewer; tiles that a kernel with larger ones would have as many of
    (1, 1000, 1000, 32, 32, 128, 100, 32), (1, 500, 500, 16, 16, 256, 0, 32), (100, 33, 33, 3, 3, 128, 0, 32), (200, 30, 90, 40, 40, 128, 0, 32)])
def test_rounds_of_the_kernel_for_few_rows(L, seqs, rows, length, heads_q, heads, d, window, tile):
    assert plan(L, seqs, seqs * rows, rows, length, heads_q, heads, d, window)[0] == tile
