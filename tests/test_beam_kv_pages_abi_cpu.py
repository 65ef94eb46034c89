"""No-GPU checks of the boundary of beam search and of the cache's pages: sizes and the refusals that come before anything touches a
device."""
import ctypes as C

import pytest

INVALID, SHAPE, WORKSPACE = 1, 2, 3
P = 1 << 20  # an address that is never read: every call here is refused


@pytest.fixture(scope="module")
def L():
    import os

    import paper_2208_07339_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2208_07339_amd.build import build
        build()
    L.lib()
    return L


def made(cls, values, kw):
    c = cls(*values)
    for name, value in kw.items():
        setattr(c, name, value)
    return C.byref(c)


def pool(**kw):
    from paper_2208_07339_amd.binding import _KvPool
    return made(_KvPool, (P, 8, 64), kw)


def seqs(**kw):
    from paper_2208_07339_amd.binding import _KvSeqs
    return made(_KvSeqs, (P, 2 * P, 3 * P, None, 4, 5), kw)


def moves(**kw):
    from paper_2208_07339_amd.binding import _KvMoves
    return made(_KvMoves, (P, 2 * P, 3 * P, 8, 4), kw)


def cache(**kw):
    from paper_2208_07339_amd.binding import _KvCache
    return made(_KvCache, (4096, 8192, 12288, 8, 64, 2, 2, 64), kw)


def test_pool_refusals(L):
    lib = L.lib()

    def fork(p=pool(), s=seqs(), parent=7 * P, grow=0, m=moves()):
        return lib.llmint8_kv_fork(p, s, parent, grow, m, None)

    def reserve(p=pool(), s=seqs(), row_start=7 * P, ready=None, m=moves()):
        return lib.llmint8_kv_reserve(p, s, row_start, ready, 0, m, None)

    def compact(p=pool(), s=seqs(), used=None, m=moves()):
        return lib.llmint8_kv_compact(p, s, used, m, None)

    for call in (fork, reserve, compact):
        assert call(p=None) == call(s=None) == call(m=None) == INVALID
        assert call(p=pool(refs=None)) == call(p=pool(refs=P + 2)) == call(p=pool(n_pages=0)) == call(p=pool(page_tokens=0)) == INVALID
        assert call(p=pool(page_tokens=-32)) == INVALID
        assert call(p=pool(page_tokens=48)) == call(p=pool(page_tokens=(1 << 20) + 32)) == call(p=pool(n_pages=(1 << 17) + 1)) == SHAPE
        for name in ("pages", "kv_len", "slots"):
            assert call(s=seqs(**{name: None})) == call(s=seqs(**{name: P + 1})) == INVALID
        assert call(s=seqs(status=2)) == call(s=seqs(n_seqs=0)) == call(s=seqs(page_stride=0)) == INVALID
        assert call(s=seqs(n_seqs=2049), m=moves(max_pages=4096, max_slots=4096)) == call(s=seqs(page_stride=(1 << 17) + 1)) == SHAPE
        for name in ("pages", "slots"):
            assert call(m=moves(**{name: None})) == call(m=moves(**{name: P + 8})) == INVALID
        assert call(m=moves(count=None)) == call(m=moves(count=P + 2)) == call(m=moves(max_pages=0)) == call(m=moves(max_slots=0)) == INVALID
    assert fork(parent=None) == fork(parent=P + 2) == fork(grow=-1) == fork(m=moves(max_slots=3)) == INVALID
    assert fork(parent=2 * P) == fork(parent=3 * P) == INVALID  # lengths or slots as parents: they are written while parents are read
    assert fork(grow=1 << 29) == SHAPE
    assert reserve(row_start=None) == reserve(row_start=P + 2) == reserve(ready=P + 2) == reserve(m=moves(max_pages=3)) == INVALID
    assert reserve(ready=2 * P) == reserve(ready=7 * P) == INVALID  # lengths or rows as the result
    assert compact(used=P + 2) == compact(m=moves(max_pages=3)) == INVALID


def test_copy_refusals(L):
    def copy(c=cache(), m=moves(), status=None):
        return L.lib().llmint8_kv_copy(c, m, status, None)

    assert copy(c=None) == copy(m=None) == copy(status=2) == INVALID
    for name in ("codes", "consts", "ring"):
        assert copy(c=cache(**{name: None})) == copy(c=cache(**{name: 4104})) == INVALID
    for name in ("n_pages", "page_tokens", "n_slots", "heads", "d"):
        assert copy(c=cache(**{name: 0})) == copy(c=cache(**{name: -1})) == INVALID
    for name in ("pages", "slots", "count"):
        assert copy(m=moves(**{name: None})) == copy(m=moves(**{name: P + 2})) == INVALID
    assert copy(m=moves(max_pages=0)) == copy(m=moves(max_slots=-1)) == INVALID
    assert copy(c=cache(page_tokens=48)) == copy(c=cache(d=257)) == copy(c=cache(heads=65536)) == SHAPE
    assert copy(c=cache(page_tokens=1 << 21)) == copy(c=cache(heads=65535), m=moves(max_slots=1 << 17)) == SHAPE


def test_beam_workspace(L):
    f = L.lib().llmint8_beam_select_workspace_bytes
    for items, beams, vocab, n_out in ((1, 4, 50257, 4), (64, 8, 131072, 8), (1, 1, 1, 1), (3, 32, 7, 32), (1000, 4, 32000, 8)):
        n = f(items, beams, vocab, n_out)
        parts = [-(-vocab // (2048 * g)) for g in (2, 4, 8)]  # pieces of a row: a sum and n_out picks each
        assert n in [(items * beams * p * 16 + 255) // 256 * 256 + items * beams * p * 8 * n_out + 256 for p in parts]
    for refused in ((0, 4, 100, 4), (1, 0, 100, 4), (1, 33, 100, 4), (1, 4, 0, 4), (1, 4, 100, 0), (1, 4, 100, 33), (-1, 4, 100, 4),
                    (2 ** 31 - 1, 32, 2 ** 31 - 1, 32), (1, 1, 2 ** 27 + 1, 1), (2 ** 23, 1, 10, 1), (2 ** 17, 32, 131072, 8)):
        assert f(*refused) == 0


def test_beam_refusals(L):
    f = L.lib().llmint8_beam_select
    a = [i * P for i in range(1, 9)]

    def call(logits=a[0], ld=100, f32=0, items=2, beams=3, vocab=100, scores=a[1], ended=None, eos=-1, n_out=3, scores_out=a[2],
             parent=a[3], token=a[4], ended_out=a[5], status=None, ws=a[6], n=1 << 20):
        return f(logits, ld, f32, items, beams, vocab, scores, ended, eos, n_out, scores_out, parent, token, ended_out, status, ws, n, None)

    for name in ("logits", "scores", "scores_out", "parent", "token"):
        assert call(**{name: None}) == call(**{name: P + 1}) == INVALID
    for name in ("ended", "ended_out", "status"):
        assert call(**{name: P + 2, "eos": 1}) == INVALID
    assert call(f32=1, logits=P + 2) == INVALID
    for name in ("items", "beams", "vocab", "n_out"):
        assert call(**{name: 0}) == call(**{name: -1}) == INVALID
    assert call(ld=99) == call(eos=-2) == call(eos=100) == call(ended=a[7]) == INVALID
    assert call(beams=33) == call(n_out=33) == call(items=2 ** 30, beams=32, vocab=2 ** 30, ld=2 ** 30) == SHAPE
    # in place only where as many come out as went in
    assert call(scores_out=a[1], n_out=2) == call(ended=a[7], ended_out=a[7], eos=1, n_out=6) == INVALID
    need = L.lib().llmint8_beam_select_workspace_bytes(2, 3, 100, 3)
    assert call(ws=None) == call(n=need - 1) == WORKSPACE
