"""No-GPU checks of the key/value cache's boundary: sizes, workspaces and the refusals that come before anything touches a device."""
import ctypes as C

import pytest

INVALID, SHAPE, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    import os

    import paper_2208_07339_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2208_07339_amd.build import build
        build()
    L.lib()
    return L


def cache(**kw):
    from paper_2208_07339_amd.binding import _KvCache
    c = _KvCache(4096, 8192, 12288, 8, 64, 2, 2, 64)  # never read: every call here is refused
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def batch(**kw):
    from paper_2208_07339_amd.binding import _KvBatch
    b = _KvBatch(4096, 4096, 4096, None, None, 2, 5, 4, 3, 100)
    for name, value in kw.items():
        setattr(b, name, value)
    return b


def test_sizes(L):
    lib = L.lib()
    assert lib.llmint8_kv_codes_bytes(3, 64, 2, 64) == 3 * 2 * 64 * 2 * 64
    assert lib.llmint8_kv_codes_bytes(3, 64, 2, 65) == 3 * 2 * 64 * 2 * 96  # features padded to 32
    assert lib.llmint8_kv_codes_bytes(1 << 20, 256, 8, 128) == (1 << 20) * 256 * 8 * 2 * 128  # beyond 32 bits
    assert lib.llmint8_kv_consts_bytes(3, 64, 2) == 3 * 2 * 2 * 2 * 2
    assert lib.llmint8_kv_ring_bytes(5, 2, 65) == 5 * 2 * 2 * 64 * 65 * 2
    for refused in ((0, 64, 2, 64), (3, 48, 2, 64), (3, 64, 0, 64), (3, 64, 2, 0), (3, 64, 2, 257)):
        assert lib.llmint8_kv_codes_bytes(*refused) == 0
    assert lib.llmint8_kv_consts_bytes(3, 33, 2) == lib.llmint8_kv_ring_bytes(0, 2, 64) == lib.llmint8_kv_ring_bytes(1, 2, 257) == 0


@pytest.mark.parametrize("kw, heads_q, heads, d", [
    (dict(), 4, 2, 64), (dict(n_seqs=1, n_rows=1, max_rows=1, max_len=131072), 64, 8, 128),
    (dict(n_seqs=1, n_rows=1024, max_rows=1024, max_len=21035), 32, 8, 128), (dict(n_rows=1, max_len=0), 1, 1, 1)])
def test_workspace(L, kw, heads_q, heads, d):
    n = L.lib().llmint8_kv_attention_workspace_bytes(C.byref(batch(**kw)), heads_q, heads, d)
    per = batch(**kw).n_rows * heads_q * (4 * d + 8)  # of a part: sums, and a maximum with a sum for each row
    assert n == 0 or (2 * per <= n <= 512 * per + 512 and (n - 512) % per == 0)
    assert (n > 0) == (batch(**kw).max_len > 10000)  # there long axes are split


def test_workspace_refusals(L):
    f = L.lib().llmint8_kv_attention_workspace_bytes
    assert f(None, 4, 2, 64) == 0
    long = dict(n_seqs=1, n_rows=1, max_rows=1, max_len=131072)
    assert f(C.byref(batch(**long)), 4, 2, 64) > 0
    for heads_q, heads, d in ((3, 2, 64), (1, 2, 64), (4, 0, 64), (4, 2, 0), (4, 2, 257)):
        assert f(C.byref(batch(**long)), heads_q, heads, d) == 0
    for name, value in (("n_seqs", 0), ("n_rows", 0), ("max_rows", 0), ("max_len", -1), ("max_len", 2 ** 31 - 1)):
        assert f(C.byref(batch(**dict(long, **{name: value}))), 4, 2, 64) == 0


def test_refusals(L):
    lib = L.lib()
    p = 1 << 20

    def append(c=cache(), b=batch(), k=p, ld_k=128, v=p, ld_v=128, q=None, ld_q=128, q_out=None, ld_out=128, hq=2, cos=None, n_pos=8,
               rot=0):
        return lib.llmint8_kv_append(C.byref(c), C.byref(b), k, ld_k, v, ld_v, q, ld_q, q_out, ld_out, hq, cos, cos, n_pos, rot, 0, None)

    def attend(c=cache(), b=batch(), q=p, ld=128, hq=2, scale=1.0, causal=1, window=0, out=p, ld_out=128, ws=None, n=0):
        return lib.llmint8_kv_attention(C.byref(c), C.byref(b), q, ld, hq, scale, causal, window, out, ld_out, ws, n, None)

    def read(c=cache(), b=batch(), k=p, v=p):
        return lib.llmint8_kv_read(C.byref(c), C.byref(b), k, v, None)

    for call in (append, attend, read):
        for name in ("codes", "consts", "ring"):
            assert call(c=cache(**{name: None})) == call(c=cache(**{name: 4104})) == INVALID
        for name in ("n_pages", "page_tokens", "n_slots", "heads", "d"):
            assert call(c=cache(**{name: 0})) == call(c=cache(**{name: -1})) == INVALID
        assert call(c=cache(page_tokens=48)) == call(c=cache(d=257)) == call(c=cache(heads=65536)) == SHAPE
        for name in ("row_start", "kv_len", "pages"):
            assert call(b=batch(**{name: None})) == call(b=batch(**{name: 4098})) == INVALID
        for name in ("n_seqs", "n_rows", "page_stride", "max_rows"):
            assert call(b=batch(**{name: 0})) == INVALID
        assert call(b=batch(max_len=-1)) == call(b=batch(slots=2)) == call(b=batch(status=2)) == INVALID
        assert call(b=batch(max_len=1 << 29)) == call(b=batch(n_rows=1 << 29)) == SHAPE
    assert append(k=None) == append(v=None) == append(k=p + 1) == append(ld_k=127) == append(ld_v=127) == append(q=p) == INVALID
    assert append(rot=64) == append(rot=3, cos=p) == append(rot=66, cos=p) == append(rot=-2, cos=p) == append(rot=2, cos=p + 2) == INVALID
    assert append(rot=64, cos=p, n_pos=0) == append(q=p, q_out=p, ld_q=256) == append(q=p, q_out=p, hq=0) == INVALID
    assert attend(q=None) == attend(out=None) == attend(q=p + 1) == attend(hq=3) == attend(hq=0) == attend(ld=127) == INVALID
    assert attend(ld_out=127) == attend(window=-1) == attend(window=5, causal=0) == INVALID
    assert attend(scale=float("nan")) == attend(scale=float("inf")) == attend(scale=-1.0) == INVALID
    one = dict(n_seqs=1, n_rows=1, max_rows=1, max_len=131072)
    assert attend(b=batch(**one)) == attend(b=batch(**one), ws=p, n=64) == WORKSPACE
    assert read(k=None, v=None) == read(k=p + 1) == INVALID
