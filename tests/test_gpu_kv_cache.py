"""kv_append and kv_read against a plain implementation: everything bit for bit."""
import numpy as np
import pytest
from kv_util import Device, rotate, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1, 2, 7, 36, 64, 72, 80, 128, 200, 256])
@pytest.mark.parametrize("strided", [False, True])
def test_append_in_any_cuts(d, strided):
    """Sequences brought in by calls of one row, of some, of many: the same cache as the definition's."""
    rng = np.random.default_rng(d)
    dev = Device(4, 2, d, page=96, most=400, seed=d)
    rot = d // 2 * 2
    tab = table(400, rot) if rot else None
    for new in [(33, 1, 0, 64), (1, 1, 1, 1), (30, 31, 5, 0), (0, 95, 27, 1), (100, 2, 100, 129), (1, 1, 1, 1), (7, 60, 64, 3)]:
        dev.append(new, rng, rot=tab, heads_q=3, strided=strided)
        dev.check_held()
        dev.check_read()
    assert int(dev.status) == 0


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d, rot", [(64, 64), (64, 32), (80, 32), (80, 20), (128, 128), (128, 16), (128, 6), (100, 100), (256, 64)])
def test_rotations(d, rot, pairs):
    rng = np.random.default_rng(d + rot)
    dev = Device(3, 3, d, page=32, most=200, seed=1)
    for new in [(40, 3, 1), (1, 1, 64), (20, 90, 1)]:
        dev.append(new, rng, rot=table(200, rot), pairs=pairs, heads_q=5, strided=True)
    dev.check_held()
    dev.check_read()


def test_row_by_row_is_the_same_as_at_once():
    rng = np.random.default_rng(5)
    k, v = (rng.standard_normal((150, 2, 64)).astype(np.float16) for _ in range(2))
    held = []
    for cut in (1, 7, 32, 33, 150):
        dev = Device(1, 2, 64, page=32, most=160, seed=2)
        for r in range(0, 150, cut):
            n = min(cut, 150 - r)
            dev.append((n,), rng, rot=table(160, 64), k=k[r:r + n], v=v[r:r + n])
        dev.check_held()
        held.append((dev.cache.codes[dev.pages.flatten().long()[:4]].cpu(), dev.cache.ring[int(dev.slots_np[0])].cpu()[:, :, :22]))
    for c, r in held[1:]:
        assert (c == held[0][0]).all() and (r.view(dev.torch.int16) == held[0][1].view(dev.torch.int16)).all()


def test_shortened_sequences():
    """Back by up to 32 positions, and on with other rows: as if the dropped ones had never been."""
    rng = np.random.default_rng(6)
    dev = Device(3, 2, 80, page=64, most=300, seed=3)
    dev.append((100, 64, 37), rng, rot=table(300, 80))
    for lengths, new in [((70, 33, 32), (1, 2, 40)), ((71, 35, 50), (60, 100, 1)), ((100, 103, 33), (33, 1, 9))]:
        for s, n in zip(dev.seq, lengths):
            s.x = s.x[:, :, :n]
        dev.check_read()
        dev.append(new, rng, rot=table(300, 80))
        dev.check_held()
        dev.check_read()


def test_values_of_every_size():
    """Constants from the smallest number to the largest, blocks of zeros, ties of the quantiser."""
    rng = np.random.default_rng(7)
    dev = Device(1, 4, 32, page=64, most=400, seed=4)
    size = np.array([2.0 ** -24, 2.0 ** -20, 1e-5, 1e-3, 0.0, 1.0, 300.0, 2.0 ** 15])
    k = np.clip(rng.standard_normal((256, 4, 32)), -1.9, 1.9) * np.repeat(size, 32)[:, None, None]
    v = np.rint(rng.standard_normal((256, 4, 32)) * 40) * np.repeat(size, 32)[:, None, None] * 0.25 * 127 / 64
    k, v = k.astype(np.float16), np.clip(v, -65504, 65504).astype(np.float16)
    dev.append((256,), rng, k=k, v=v)
    dev.check_held()
    dev.check_read()


def test_what_is_not_finite_is_stored_as_finite_and_told():
    rng = np.random.default_rng(8)
    for at, what, n in [(3, np.inf, 40), (35, np.nan, 40), (39, -np.inf, 40), (0, np.nan, 1)]:
        for kv in range(2):
            dev = Device(2, 2, 64, page=32, most=96, seed=5)
            x = [rng.standard_normal((n + 5, 2, 64)).astype(np.float16) for _ in range(2)]
            x[kv][at, 1, 9] = what
            dev.append((n, 5), rng, k=x[0], v=x[1])
            dev.check_held()
            dev.check_read()
            assert int(dev.status) == dev.L.KV_NOT_FINITE
    dev = Device(1, 1, 4, page=32, most=96, seed=5)  # a rotation that leaves fp16's range
    k = np.full((1, 1, 4), 60000.0, np.float16)
    c = np.full((4, 2), np.float32(np.sqrt(0.5)))
    dev.append((1,), rng, rot=(c, -c), k=k, v=k)
    dev.check_held()
    assert int(dev.status) == dev.L.KV_NOT_FINITE and np.isinf(rotate(k, np.array([0]), c, -c, False)).any()


def test_queries_in_place_and_without_rotation():
    import torch

    import paper_2208_07339_amd as L
    rng = np.random.default_rng(9)
    for d, rot, pairs in [(64, 64, False), (64, 32, True), (36, 12, False), (64, 0, False)]:
        dev = Device(2, 2, d, page=32, most=96, seed=6)
        q, k, v = (rng.standard_normal((41, h, d)).astype(np.float16) for h in (6, 2, 2))
        cos, sin = table(96, rot) if rot else (None, None)
        kw = dict(cos=dev.dev(cos), sin=dev.dev(sin), pairs=pairs) if rot else {}
        joint = dev.dev(np.concatenate((q, k, v), 1))
        qd, kd, vd = joint.split([6, 2, 2], 1)
        batch = dev.batch((40, 1), (40, 1))
        other = L.kv_append(dev.cache, batch, kd, vd, q=qd, **kw)
        same = L.kv_append(dev.cache, batch, kd, vd, q=qd, q_out=qd, **kw)
        want = rotate(q, np.r_[np.arange(40), 0], cos, sin, pairs)
        assert same.data_ptr() == qd.data_ptr()
        for got in (other, same):
            assert np.array_equal(got.cpu().numpy().view(np.uint16), want.view(np.uint16))
        assert torch.equal(kd.cpu(), torch.from_numpy(k)) and torch.equal(vd.cpu(), torch.from_numpy(v))


def test_idle_sequences_keep_their_cache():
    rng = np.random.default_rng(10)
    dev = Device(3, 2, 64, page=32, most=96, seed=7)
    dev.append((35, 20, 50), rng)
    held = [t.clone() for t in (dev.cache.codes, dev.cache.consts, dev.cache.ring)]
    k = dev.dev(rng.standard_normal((3, 2, 64)).astype(np.float16))
    dev.L.kv_append(dev.cache, dev.batch((1, 1, 1), (0, 0, 0)), k, k)
    for a, b in zip(held, (dev.cache.codes, dev.cache.consts, dev.cache.ring)):
        assert (a.view(dev.torch.int8) == b.view(dev.torch.int8)).all()
    assert int(dev.status) == 0
    dev.check_read()


@pytest.mark.parametrize("what", ["rows", "length", "table", "slot", "short", "positions", "most_rows", "most_len"])
def test_batches_that_cannot_be(what):
    """The sequence is left out and told of, the others are served."""
    rng = np.random.default_rng(11)
    dev = Device(3, 2, 64, page=32, most=96, seed=8)
    good = Device(3, 2, 64, page=32, most=96, seed=8)
    new, length = [35, 40, 33], [35, 40, 33]
    k = rng.standard_normal((108, 2, 64)).astype(np.float16)
    kw, more = {}, {}
    start = np.array([0, 35, 75, 108], np.int32)
    if what == "rows":
        start[3] = 109
        kw["row_start"] = dev.dev(start)
    elif what in ("length", "table"):
        length[2] = -5 if what == "length" else 97
        more["max_len"] = 200
    elif what == "slot":
        kw["slots"] = dev.dev(np.array([*dev.slots_np[:2], 5], np.int32))
    elif what == "short":
        length[2] = 32
    elif what == "positions":
        k, length, new = k[:107], [35, 40, 96], [35, 40, 32]
        cos, sin = table(95, 64)
        more.update(cos=dev.dev(cos), sin=dev.dev(sin))
    elif what == "most_rows":
        kw["max_rows"] = 40
        new, length, k = [35, 40, 41], [35, 40, 41], rng.standard_normal((116, 2, 64)).astype(np.float16)
    else:
        length[2], more["max_len"] = 50, 49
    batch = dev.batch(new, length, max_len=more.pop("max_len", None), **kw)
    kd = dev.dev(k)
    dev.L.kv_append(dev.cache, batch, kd, kd, **more)
    good.append((35, 40, 0), rng, k=k[:75], v=k[:75], rot=table(95, 64) if what == "positions" else None)
    assert int(dev.status) == dev.L.KV_BAD_BATCH
    for a, b in zip((dev.cache.codes, dev.cache.consts, dev.cache.ring), (good.cache.codes, good.cache.consts, good.cache.ring)):
        assert (a.view(dev.torch.int8) == b.view(dev.torch.int8)).all()
    if what not in ("short", "positions"):
        dev.status.zero_()
        kr, vr = (dev.torch.full((batch.n_rows, 2, 64), 7.0, dtype=dev.torch.float16, device="cuda") for _ in range(2))
        dev.L.kv_read(dev.cache, batch, kr, vr)
        assert int(dev.status) == dev.L.KV_BAD_BATCH
        if what not in ("rows", "most_rows"):
            assert (kr[75:] == 0).all() and (vr[75:] == 0).all()
        want, _ = good.L.kv_read(good.cache, good.batch((35, 40, 0), (35, 40, 0)))
        assert (kr[:75] == want[:75]).all()


def test_pages_that_do_not_exist():
    rng = np.random.default_rng(12)
    dev, good = (Device(2, 2, 64, page=32, most=96, seed=9) for _ in range(2))
    k = rng.standard_normal((160, 2, 64)).astype(np.float16)
    good.append((80, 80), rng, k=k, v=k)
    for wrong in (-1, dev.cache.codes.shape[0]):
        pages = dev.pages_np.copy()
        pages[1, 1] = wrong
        batch = dev.batch((80, 80), (80, 80), pages=dev.dev(pages))
        kd = dev.dev(k)
        dev.status.zero_()
        dev.L.kv_append(dev.cache, batch, kd, kd)
        assert int(dev.status) == dev.L.KV_BAD_PAGE
        dev.status.zero_()
        kr, vr = dev.L.kv_read(dev.cache, batch)
        assert int(dev.status) == dev.L.KV_BAD_PAGE
        want, _ = good.L.kv_read(good.cache, good.batch((80, 80), (80, 80)))
        keep = np.r_[0:112, 144:160]
        assert (kr[keep] == want[keep]).all() and (vr[keep] == want[keep]).all()
        assert (kr[112:144] == 0).all() and (vr[112:144] == 0).all()
        unused = good.pages_np[1, 1]  # nothing was written for it
        assert (dev.cache.codes[unused] == 77).all()


def test_read_before_the_first_position():
    rng = np.random.default_rng(13)
    dev = Device(2, 1, 64, page=32, most=96, seed=10)
    dev.append((40, 3), rng)
    k, v = dev.L.kv_read(dev.cache, dev.batch((75, 70), (40, 3)))
    for got, kv in ((k, 0), (v, 1)):
        g = got.cpu().numpy()
        assert (g[:35] == 0).all() and (g[75:142] == 0).all()
        assert np.array_equal(g[35:75, 0], dev.seq[0].held()[kv, 0].astype(np.float16))
        assert np.array_equal(g[142:, 0], dev.seq[1].held()[kv, 0].astype(np.float16))


def test_more_than_4_gib_of_codes():
    """Pages behind 2^32 bytes, and a ring of more than 2^31 elements."""
    import torch

    import paper_2208_07339_amd as L
    rng = np.random.default_rng(14)
    heads, d, page, n_pages, n_slots = 8, 128, 64, 36000, 18000
    cache = L.KvCache.allocate(n_pages, page, n_slots, heads, d)
    assert cache.codes.numel() > 1 << 32 and cache.ring.numel() > 1 << 31
    dev = Device(2, heads, d, page=page, most=128, seed=11)
    dev.cache, dev.pages_np, dev.slots_np = cache, np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, 5]], np.int32), np.array([n_slots - 1, 17500], np.int32)
    dev.pages, dev.slots = dev.dev(dev.pages_np), dev.dev(dev.slots_np)
    dev.append((100, 70), rng, rot=table(128, 128))
    dev.check_read()
    dev.check_attention((1, 1), rng, group=4)
    dev.check_attention((100, 70), rng, group=4)
    assert int(dev.status) == 0
    del cache
    torch.cuda.empty_cache()


def test_many_sequences():
    """More than the 64 that a wave looks through at once, most of them without rows."""
    rng = np.random.default_rng(15)
    dev = Device(150, 1, 32, page=32, most=96, seed=12)
    new = [0] * 150
    for b, n in [(0, 3), (63, 40), (64, 1), (65, 33), (127, 5), (149, 70)]:
        new[b] = n
    dev.append(tuple(new), rng, rot=table(96, 32), heads_q=1)
    dev.append(tuple([1] * 150), rng, rot=table(96, 32), heads_q=1)
    dev.check_held()
    dev.check_read()
    dev.check_attention([1] * 150, rng, group=2)
    dev.check_attention([min(40, n) for n in dev.lengths()], rng, group=2)


def test_refusals():
    import ctypes as C

    import torch

    import paper_2208_07339_amd as L
    from paper_2208_07339_amd import binding
    lib = L.lib()
    dev = Device(1, 2, 64, page=32, most=64, seed=13)
    k = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda")
    batch = dev.batch((3,), (3,))
    p, c, b = k.data_ptr(), dev.cache._c, batch._c

    def append(cache=c, k=p, ld=128, q=None, q_out=None, ldq=128, ldo=128, hq=2, cos=None, n_pos=8, rot=0, batch=b):
        return lib.llmint8_kv_append(C.byref(cache), C.byref(batch), k, ld, p, 128, q, ldq, q_out, ldo, hq, cos, cos, n_pos, rot, 0, None)

    def other(of, **kw):
        x = type(of)()
        C.memmove(C.byref(x), C.byref(of), C.sizeof(of))
        for name, value in kw.items():
            setattr(x, name, value)
        return x

    assert append(k=None) == append(k=p + 1) == append(ld=127) == append(q=p) == append(rot=64) == 1
    assert append(rot=3, cos=p) == append(rot=66, cos=p) == append(rot=64, cos=p, n_pos=0) == append(q=p, q_out=p, ldq=256) == 1
    assert append(q=p, q_out=p, ldq=100) == append(q=p, q_out=p, hq=0) == append(rot=-2, cos=p) == 1
    assert append(q=p, q_out=p, hq=65535, ldq=1 << 30, ldo=1 << 30) == 2
    for name in ("codes", "consts", "ring"):
        assert append(other(c, **{name: None})) == 1 and append(other(c, **{name: getattr(c, name) + 8})) == 1
    for name in ("n_pages", "page_tokens", "n_slots", "heads", "d"):
        assert append(other(c, **{name: 0})) == 1
    assert append(other(c, page_tokens=48)) == append(other(c, d=257), ld=1000) == 2
    for name in ("row_start", "kv_len", "pages"):
        assert append(batch=other(b, **{name: None})) == 1 and append(batch=other(b, **{name: getattr(b, name) + 2})) == 1
    for name in ("n_seqs", "n_rows", "page_stride", "max_rows"):
        assert append(batch=other(b, **{name: 0})) == 1
    assert append(batch=other(b, max_len=-1)) == 1 and append(batch=other(b, max_len=1 << 29)) == 2
    assert lib.llmint8_kv_read(C.byref(c), C.byref(b), None, None, None) == 1
    assert lib.llmint8_kv_read(C.byref(c), C.byref(b), p + 1, None, None) == 1
    assert lib.llmint8_kv_read(None, C.byref(b), p, p, None) == lib.llmint8_kv_read(C.byref(c), None, p, p, None) == 1

    def attend(cache=c, q=p, ld=128, hq=2, scale=1.0, causal=1, window=0, out=p, ws=None, ws_bytes=0, batch=b):
        return lib.llmint8_kv_attention(C.byref(cache), C.byref(batch), q, ld, hq, scale, causal, window, out, 128, ws, ws_bytes, None)

    assert attend(q=None) == attend(out=None) == attend(q=p + 1) == attend(hq=3) == attend(hq=0) == attend(ld=100) == 1
    assert attend(scale=float("nan")) == attend(scale=float("inf")) == attend(scale=-1.0) == attend(window=-1) == 1
    assert attend(causal=0, window=3) == 1
    assert attend(batch=other(b, max_len=100000)) == 3  # splits need a workspace
    with pytest.raises(AssertionError):
        L.kv_append(dev.cache, batch, k.float(), k)
    with pytest.raises(AssertionError):
        L.kv_append(dev.cache, batch, k[:2], k)
    with pytest.raises(AssertionError):
        L.kv_append(dev.cache, batch, k.transpose(1, 2), k)
    with pytest.raises(AssertionError):
        L.KvBatch(batch.row_start.long(), batch.kv_len, batch.pages, None, 3, 3, 3)
    with pytest.raises(AssertionError):
        L.KvCache(dev.cache.codes, dev.cache.consts, dev.cache.ring, 64, 64)
    with pytest.raises(binding.Llmint8Error):
        L.kv_attention(dev.cache, batch, k, scale=float("nan"))
