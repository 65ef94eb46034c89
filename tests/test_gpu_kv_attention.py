"""kv_attention against 64 bits.  The bound on every output is that of the number formats (kv_util.attention)."""
import numpy as np
import pytest
from kv_util import Device, table

pytestmark = pytest.mark.gpu

LENGTHS = (1, 2, 31, 32, 33, 63, 64, 65, 127, 200, 511)


def filled(lengths, heads, d, page=64, seed=0, most=None, rng=None, **kw):
    dev = Device(len(lengths), heads, d, page=page, most=most or max(lengths), seed=seed)
    dev.append(tuple(lengths), rng or np.random.default_rng(seed), **kw)
    return dev


@pytest.mark.parametrize("d", [1, 16, 33, 64, 80, 96, 128, 160, 192, 200, 256])
@pytest.mark.parametrize("group", [1, 3, 32])
def test_single_rows(d, group):
    rng = np.random.default_rng(d + group)
    dev = filled(LENGTHS, 2, d, page=96, seed=d)
    dev.check_attention([1] * len(LENGTHS), rng, group=group)
    dev.check_attention([1] * len(LENGTHS), rng, group=group, idle=(0, 5, 10))
    assert int(dev.status) == 0


@pytest.mark.parametrize("group, new", [(1, 2), (1, 32), (4, 8), (5, 6), (1, 33), (8, 5), (48, 1), (40, 7), (3, 130), (1, 300)])
@pytest.mark.parametrize("window", [0, 1, 20, 100])
def test_rows_and_windows(group, new, window):
    """On both sides of the kernels' border, sequences shorter than their rows among them (rows that see nothing)."""
    rng = np.random.default_rng(group * new + window)
    lengths = (1, 31, 32, 33, 70, 129, 330)
    dev = filled(lengths, 2, 64, page=32, seed=new)
    dev.check_attention([new] * 7, rng, group=group, window=window)
    dev.check_attention([min(new, t) for t in lengths], rng, group=group, window=window, idle=(4,))
    assert int(dev.status) == 0


@pytest.mark.parametrize("d", [1, 16, 33, 64, 80, 96, 128, 160, 192, 200, 256])
def test_many_rows(d):
    rng = np.random.default_rng(d)
    lengths = (1, 32, 65, 300, 411)
    dev = filled(lengths, 2, d, page=96, seed=d)
    dev.check_attention(lengths, rng, group=2)
    dev.check_attention((0, 17, 0, 150, 0), rng, group=1, window=64)


@pytest.mark.parametrize("blocks", [1, 2, 3, 54, 55, 56, 57, 58, 62, 63, 64, 65, 110, 111, 112, 113, 114, 128, 168])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_numbers_of_blocks(blocks, rows):
    """Around the numbers that the kernels look up or keep at once, with and without an open block."""
    rng = np.random.default_rng(blocks)
    for length in (32 * blocks, 32 * blocks + 5):
        dev = filled((length,), 1, 32, page=32, seed=blocks)
        dev.check_attention((min(rows, length),), rng)
        assert int(dev.status) == 0


@pytest.mark.parametrize("group, new", [(1, 1), (2, 40)])
def test_rows_that_see_everything(group, new):
    rng = np.random.default_rng(3)
    dev = filled((1, 33, 64, 250), 2, 64, seed=3)
    dev.check_attention([new] * 4, rng, group=group, causal=False)


@pytest.mark.parametrize("group, new, lengths", [(8, 1, (9001, 4, 700)), (1, 1, (6000,)), (1, 64, (5000, 100)), (16, 30, (3333,)),
                                                 (48, 3, (2050, 33))])
def test_long_axes_that_are_split(group, new, lengths):
    rng = np.random.default_rng(new)
    dev = filled(lengths, 1, 128, page=64, seed=new)
    new = [min(new, t) for t in lengths]
    a = dev.check_attention(new, rng, group=group)
    q = rng.standard_normal((sum(new), group, 128)).astype(np.float16)
    # the same bits each time; a larger max_len only cuts the work otherwise
    a, b = (dev.check_attention(new, rng, group=group, q=q) for _ in range(2))
    assert dev.torch.equal(a, b)
    dev.check_attention(new, rng, group=group, q=q, max_len=60000 // 64 * 64)
    dev.check_attention(new, rng, group=group, window=1500)


@pytest.mark.parametrize("new", [1, 50])
def test_scores_far_apart_and_values_of_any_size(new):
    """One position far above the others (weights from 1 to nothing), scores of thousands; values' constants from the smallest
    number to the largest, blocks of zeros; a scale of 0."""
    rng = np.random.default_rng(4)
    n = 32 * 9 + 7
    size = np.repeat([1.0, 2.0 ** -24, 1e-5, 0.0, 1000.0, 1e-3, 1.0, 30000.0, 3.0, 2.0 ** -14], 32)[:n, None, None]
    k = rng.standard_normal((n, 2, 64)).astype(np.float16) * np.float16(4)
    k[5], k[290] = 60, -60
    v = np.clip(rng.standard_normal((n, 2, 64)), -2, 2) * size
    dev = Device(1, 2, 64, page=64, most=n, seed=4)
    dev.append((n,), rng, k=k, v=v.astype(np.float16))
    for scale in (0.125, 5.0, 0.0, 1e-4):
        dev.check_attention((new,), rng, group=2, scale=scale)
    dev.check_attention((new,), rng, group=2, q=np.full((new, 4, 64), 3.0, np.float16), scale=1.0)
    dev.check_attention((new,), rng, group=2, q=np.full((new, 4, 64), 60000.0, np.float16), scale=2.0 ** -15)
    for n2 in (32, 96, 128, 129, 290):  # the last block of every kind
        dev.check_attention((min(new, n2),), rng, group=2, lengths=(n2 // 32 * 32,))


@pytest.mark.parametrize("new", [2, 40])
def test_what_is_hidden_does_not_count(new):
    """Keys and values that were infinite or NaN, at positions that only the last row sees, and the unused places' garbage."""
    rng = np.random.default_rng(5)
    for what in (np.inf, -np.inf, np.nan):
        for length in (64, 75):
            k, v = (rng.standard_normal((length, 2, 64)).astype(np.float16) for _ in range(2))
            k[-1, 0, 3], v[-1, 1, 5] = what, what
            dev = Device(1, 2, 64, page=32, most=length, seed=5)
            dev.append((length,), rng, k=k, v=v)
            out = dev.check_attention((new,), rng)
            assert dev.torch.isfinite(out).all()


@pytest.mark.parametrize("new", [1, 40])
def test_a_row_that_is_not_finite_stays_alone(new):
    rng = np.random.default_rng(6)
    dev = filled((300,), 2, 64, seed=6)
    q = rng.standard_normal((new, 4, 64)).astype(np.float16)
    want = dev.check_attention((new,), rng, group=2, q=q)
    q[new // 2, 1, 3] = np.nan
    got = dev.L.kv_attention(dev.cache, dev.batch((new,), (300,)), dev.dev(q))
    keep = dev.torch.ones((new, 4), dtype=dev.torch.bool)
    keep[new // 2, 1] = False
    assert dev.torch.equal(got.cpu()[keep], want.cpu()[keep]) and got[new // 2, 1].isnan().any()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("d", [64, 36])
def test_strides_and_alignment(new, d):
    import paper_2208_07339_amd as L
    rng = np.random.default_rng(7)
    dev = filled((100, 61), 2, d, seed=7)
    q = rng.standard_normal((2 * new, 4, d)).astype(np.float16)
    want = dev.check_attention((new, new), rng, group=2, q=q)
    batch = dev.batch((new, new), (100, 61))
    for off, extra in [(0, 3), (1, 3), (8, 16)]:
        wide = dev.torch.full((2 * new * (4 * d + extra) + 16,), 9.0, dtype=dev.torch.float16, device="cuda")
        out = wide[off:off + 2 * new * (4 * d + extra)].view(2 * new, 4 * d + extra)[:, :4 * d].unflatten(1, (4, d))
        qs = wide.clone()[off:off + 2 * new * (4 * d + extra)].view(2 * new, 4 * d + extra)[:, :4 * d].unflatten(1, (4, d))
        qs.copy_(dev.dev(q))
        L.kv_attention(dev.cache, batch, qs, out=out)
        assert dev.torch.equal(out, want)
        n = int((wide == 9.0).sum())
        assert n >= 16 + 2 * new * extra  # nothing was written between the rows


@pytest.mark.parametrize("what", ["rows", "length", "table", "slot", "most_rows", "most_len"])
@pytest.mark.parametrize("new", [1, 40])
def test_batches_that_cannot_be(what, new):
    rng = np.random.default_rng(8)
    dev = filled((100, 90, 80), 2, 64, page=32, most=128, seed=8)
    q = rng.standard_normal((3 * new, 2, 64)).astype(np.float16)
    want = dev.check_attention((new,) * 3, rng, q=q).clone()
    kw, lengths, max_len = {}, [100, 90, 80], None
    if what == "rows":
        kw["row_start"] = dev.dev(np.array([0, new, 2 * new, 3 * new + 1], np.int32))
    elif what in ("length", "table"):
        lengths[2], max_len = (-1, None) if what == "length" else (129, 129)
    elif what == "slot":
        kw["slots"] = dev.dev(np.array([*dev.slots_np[:2], -1], np.int32))
    elif what == "most_rows":
        q = np.concatenate((q, q[:1]))
        kw["row_start"], kw["n_rows"] = dev.dev(np.array([0, new, 2 * new, 3 * new + 1], np.int32)), 3 * new + 1
    else:
        lengths[2], max_len = 101, 100
    out = dev.torch.full((len(q), 2, 64), 7.0, dtype=dev.torch.float16, device="cuda")
    dev.L.kv_attention(dev.cache, dev.batch((new,) * 3, lengths, max_len=max_len, **kw), dev.dev(q), out=out)
    assert int(dev.status) == dev.L.KV_BAD_BATCH
    assert dev.torch.equal(out[:2 * new], want[:2 * new])
    if what not in ("rows", "most_rows"):
        assert (out[2 * new:] == 0).all()


@pytest.mark.parametrize("new", [1, 40])
def test_pages_that_do_not_exist(new):
    """Their positions count as hidden."""
    rng = np.random.default_rng(9)
    dev = filled((160,), 1, 64, page=32, seed=9)
    q = rng.standard_normal((new, 2, 64)).astype(np.float16)
    pages = dev.pages_np.copy()
    pages[0, 1] = 1 << 30
    got = dev.L.kv_attention(dev.cache, dev.batch((new,), (160,), pages=dev.dev(pages)), dev.dev(q), causal=False)
    assert int(dev.status) == dev.L.KV_BAD_PAGE
    from kv_util import attention
    held = np.delete(dev.seq[0].held(), np.arange(32, 64), 2)
    want, tol = attention(q, held, np.zeros(new), 0.125, causal=False)
    assert (np.abs(got.cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("new", [1, 40])
def test_another_stream_and_a_graph(new):
    """On a stream of the caller's; recorded once and replayed as the sequences grow, against the same calls made directly."""
    import torch

    import paper_2208_07339_amd as L
    rng = np.random.default_rng(10)
    seqs, heads, d = 3, 2, 64
    dev, ref = (filled((40, 700, 3), heads, d, page=64, most=1024, seed=10) for _ in range(2))
    cos, sin = (dev.dev(t) for t in table(1024, d))
    lengths = np.array([40, 700, 3])
    T = seqs * new
    qkv = torch.zeros((T, 4 * heads, d), dtype=torch.float16, device="cuda")
    q, k, v = qkv.split([2 * heads, heads, heads], 1)
    batch = dev.batch([new] * seqs, lengths, max_len=1024)
    ws, out, qr = L.kv_attention_workspace(dev.cache, batch, 2 * heads), torch.zeros((T, 2 * heads, d), dtype=torch.float16, device="cuda"), torch.zeros((T, 2 * heads, d), dtype=torch.float16, device="cuda")

    def step():
        L.kv_append(dev.cache, batch, k, v, q=q, q_out=qr, cos=cos, sin=sin)
        L.kv_attention(dev.cache, batch, qr, ws=ws, out=out)

    side = torch.cuda.Stream()
    graph = None
    for turn in range(5):
        lengths = lengths + new
        batch.kv_len.copy_(torch.from_numpy(lengths.astype(np.int32)))
        x = torch.from_numpy(rng.standard_normal((T, 4 * heads, d)).astype(np.float16))
        qkv.copy_(x)
        torch.cuda.synchronize()
        if turn == 0:
            with torch.cuda.stream(side):
                step()
        elif graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        rb = ref.batch([new] * seqs, lengths, max_len=1024)
        rq, rk, rv = x.cuda().split([2 * heads, heads, heads], 1)
        want = L.kv_attention(ref.cache, rb, L.kv_append(ref.cache, rb, rk, rv, q=rq, cos=cos, sin=sin))
        assert torch.equal(out, want), turn
    assert int(dev.status) == 0
