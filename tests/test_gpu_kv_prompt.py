"""kv_attention's kernel for many rows in each of its forms: tiles of 128 and of 256 rows, in one part and in several, and tiles whose
blocks two halves of a workgroup share.  Every test asserts the form that its call takes (llmint8_debug_kv_plan_for).  The reference
is kv_util.attention with its tolerance, computed in 64 bits on the GPU since these calls are large."""
import numpy as np
import pytest

from kv_util import Device, table

pytestmark = pytest.mark.gpu

# rows to a tile, more than one part, halves; heads, query heads to a head, new rows and lengths
FORMS = {"rows128": ((128, False, False), 16, 4, [1100], [1800]), "rows128 parts": ((128, True, False), 17, 2, [700, 40], [2200, 333]),
         "rows256": ((256, False, False), 8, 8, [1100, 3], [4200, 90]), "rows256 parts": ((256, True, False), 8, 4, [900], [4200]),
         "halves": ((128, False, True), 16, 1, [1500, 33, 7], [1500, 200, 7])}


def attention64(q, held, pos, scale, causal=True, window=0, gone=()):
    """kv_util.attention of numpy arrays, computed with torch; positions `gone` are seen by none."""
    import torch
    q, held, pos = torch.from_numpy(q).cuda().double(), torch.from_numpy(held).cuda(), torch.from_numpy(pos).cuda()[:, None]
    (rows, hq, d), (heads, n) = q.shape, held.shape[1:3]
    j = torch.arange(n, device="cuda")
    see = j <= pos if causal else torch.ones((rows, n), dtype=torch.bool, device="cuda")
    if window:
        see &= j > pos - window
    see[:, list(gone)] = False
    some, seen = see.any(1, keepdim=True), see.sum(1, keepdim=True)
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    if n == 0:
        return out, tol
    for h in range(hq):
        k, v = held[:, h // (hq // heads)]
        s = (q[:, h] @ k.T * scale).masked_fill(~see, float("-inf"))
        w = (s - s.amax(1, keepdim=True).clamp(min=-1e300)).exp()
        total = torch.where(some, w.sum(1, keepdim=True), 1.0)
        o, size = w @ v / total, w @ v.abs() / total
        e = scale * (q[:, h].abs() @ k.abs().T).masked_fill(~see, 0.0).amax(1, keepdim=True)
        rel = 4 * (d + 16) * 2.0 ** -24 * e + 2.0 ** -19 + 2 * seen * 2.0 ** -24 + 2 * 2.0 ** -11
        out[:, h] = o
        tol[:, h] = (rel * size + 2.0 ** -11 * o.abs() + 2.0 ** -25 + seen * 2.0 ** -25 * v.abs().max() / total) * some
    return out, tol


class Prompt(Device):
    """Sequences of `lengths`, of which the last `new` are the call's rows."""

    def __init__(self, heads, group, new, lengths, d, page=32, seed=0, rng=None, garbage=float("inf"), **kw):
        super().__init__(len(new), heads, d, page=page, most=max(1, *lengths), seed=seed)
        self.rng = rng or np.random.default_rng(seed)
        self.group, self.new = group, list(new)
        self.cache.consts.fill_(garbage)
        if sum(lengths):
            self.append(list(lengths), self.rng, **kw)

    def queries(self):
        return self.rng.standard_normal((sum(self.new), self.heads * self.group, self.d)).astype(np.float16)

    def expect(self, form, batch, window=0):
        p = self.L.debug_kv_plan_for(self.cache, batch, self.heads * self.group, window)
        assert (p.tile, p.parts > 1, bool(p.halves)) == form, (p.tile, p.parts, p.halves)

    def check(self, form, q=None, told=None, scale=None, causal=True, window=0, gone=(), skip=(), **kw):
        """kv_attention against 64 bits.  told: lengths in place of the sequences'; gone: positions of the first sequence on missing
        pages; skip: rows whose results are not looked at."""
        q = self.queries() if q is None else q
        told = self.lengths() if told is None else told
        scale = self.d ** -0.5 if scale is None else scale
        batch = self.batch(self.new, told, **{"max_len": max(self.lengths()), **kw})
        self.expect(form, batch, window)
        out = self.L.kv_attention(self.cache, batch, self.dev(q), scale=scale, causal=causal, window=window)
        row = 0
        for b, (s, n, t) in enumerate(zip(self.seq, self.new, told)):
            want, tol = attention64(q[row:row + n], s.held(t), np.arange(t - n, t), scale, causal, window, gone if b == 0 else ())
            wrong = ~((out[row:row + n].double() - want).abs() <= tol)
            wrong[[r - row for r in skip if row <= r < row + n]] = False
            assert not wrong.any(), (b, n, t, int(wrong.sum()), wrong.nonzero()[0].tolist())
            row += n
        return out


def made(form, d=32, **kw):
    want, heads, group, new, lengths = FORMS[form]
    return want, Prompt(heads, group, new, lengths, d, **kw)


@pytest.mark.parametrize("d", [1, 16, 33, 64, 80, 96, 128, 160, 192, 200, 224, 256])
def test_widths_of_heads(d):
    """Ragged prompts, with and without a window; and wide heads in parts."""
    dev = Prompt(64, 1, [1, 32, 65, 300, 411], [1, 40, 65, 300, 500], d, page=96, seed=d)
    dev.check((128, False, False))
    dev.check((128, False, False), window=390)
    assert int(dev.status) == 0
    if d > 128:
        Prompt(8, 1, [900], [4200], d, seed=d).check((128, True, False))


@pytest.mark.parametrize("d", [33, 64, 96, 128])
@pytest.mark.parametrize("tile, parts, halves, heads, group, new, lengths", [
    (256, False, False, 8, 8, [1100, 3], [4200, 90]), (256, True, False, 20, 1, [300], [4200]),
    (128, False, True, 8, 4, [980, 3], [1900, 90]), (128, True, False, 40, 1, [300], [3900])])
def test_widths_of_heads_in_other_forms(tile, parts, halves, heads, group, new, lengths, d):
    dev = Prompt(heads, group, new, lengths, d, seed=d)
    dev.check((tile, parts, halves))
    assert int(dev.status) == 0


@pytest.mark.parametrize("blocks", [48, 54, 55, 56, 57, 58, 59, 60, 62, 63, 64, 65, 110, 111, 112, 113, 114, 115])
def test_numbers_of_blocks_128_rows(blocks):
    """Around the numbers that the kernel looks up at once, with and without an open block."""
    for length in (32 * blocks, 32 * blocks + 5):
        Prompt(16, 4, [1100], [length], 32, seed=blocks).check((128, False, False))


@pytest.mark.parametrize("blocks", [129, 130, 167, 168, 169, 170, 171, 223, 224, 225, 226])
def test_numbers_of_blocks_256_rows(blocks):
    for length in (32 * blocks, 32 * blocks + 31):
        Prompt(8, 8, [1100], [length], 32, seed=blocks).check((256, False, False))
        Prompt(8, 4, [900], [length], 32, seed=blocks).check((256, True, False))


@pytest.mark.parametrize("blocks", [108, 110, 111, 112, 113, 114, 115, 116, 223, 224, 225, 226])
def test_numbers_of_blocks_halves(blocks):
    """Halves of 54 to 58, and of 112 and 113."""
    for length in (32 * blocks, 32 * blocks + 17):
        Prompt(8, 4, [1000], [length], 128, seed=blocks).check((128, False, True))


@pytest.mark.parametrize("form, heads, group, new, lengths, window", [
    ("rows128", 64, 8, [1100, 64], [1800, 64], 1), ("rows128", 64, 4, [1100, 64], [1800, 64], 31), ("rows128", 40, 4, [1100, 64], [1800, 64], 333),
    ("rows128", 16, 4, [1100], [1800], 1000), ("rows128", 8, 4, [1060], [2500], 1500), ("rows128 parts", 12, 2, [700], [3900], 3000),
    ("rows256", 32, 1, [2100], [5200], 4100), ("rows256", 8, 8, [1100, 3], [4500, 90], 4300), ("rows256 parts", 8, 4, [900], [6000], 4200),
    ("halves", 32, 1, [900], [4200], 1000), ("halves", 8, 4, [900], [4200], 1000), ("halves", 8, 4, [1000], [3500], 3000)])
def test_windows(form, heads, group, new, lengths, window):
    dev = Prompt(heads, group, new, lengths, 128 if (form, window) == ("halves", 3000) else 32, page=96, seed=window)
    dev.check(FORMS[form][0], window=window)
    assert int(dev.status) == 0


@pytest.mark.parametrize("form", FORMS)
def test_rows_that_see_everything(form):
    want, dev = made(form, seed=1)
    dev.check(want, causal=False)


@pytest.mark.parametrize("form", FORMS)
def test_idle_sequences_and_rows_before_the_first_position(form):
    """A sequence shorter than its rows: the first ones see nothing and are zero, also in tiles whose other rows see something."""
    want, heads, group, new, lengths = FORMS[form]
    for told in (new[0] - 77, new[0] // 2, 33, 32, 5, 0):
        rest = [0 if told == 33 else t for t in lengths[1:]]
        dev = Prompt(heads, group, new, [told, *rest], 32, seed=2)
        out = dev.check(want, causal=told != 32, max_len=max(lengths))
        if told != 32:
            assert (out[:new[0] - told] == 0).all()
        assert int(dev.status) == 0


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("form", FORMS)
def test_missing_pages(form, causal):
    """The first page, one in the middle, the last whole one, and several together; unwritten constants are infinite."""
    want, dev = made(form, seed=3)
    n = dev.lengths()[0] // 32
    for missing in ([0], [n // 2], [n - 1], [0, 1, 2, n // 3, n // 2, n // 2 + 1, n - 2]):
        pages = dev.pages_np.copy()
        pages[0, missing] = [-1, dev.cache.codes.shape[0], 1 << 30, -1 << 31, -5, 1 << 20, -1][:len(missing)]
        dev.status.zero_()
        dev.check(want, causal=causal, gone=[32 * j + i for j in missing for i in range(32)], pages=dev.dev(pages))
        assert int(dev.status) == dev.L.KV_BAD_PAGE


@pytest.mark.parametrize("form", FORMS)
def test_rows_that_are_not_finite_stay_alone(form):
    want, dev = made(form, seed=4)
    q, n = dev.queries(), dev.new[0]
    plain = dev.check(want, q=q)
    bad = [0, n // 2, n - 1]
    q[bad, 1, 3] = np.nan
    got = dev.check(want, q=q, skip=bad)
    keep = np.ones(q.shape[:2], bool)
    keep[bad, 1] = False
    assert dev.torch.equal(got.cpu()[keep], plain.cpu()[keep]) and got[bad, 1].isnan().any()
    q[bad, 1, 3] = [np.inf, -np.inf, np.inf]
    dev.check(want, q=q, skip=bad)


@pytest.mark.parametrize("form", FORMS)
def test_scores_far_apart_and_values_of_any_size(form):
    """Constants of values from the smallest number to the largest and blocks of zeros, in every order; scores that differ by
    hundreds; single positions far above the others, early and late; scales of 0 and near it."""
    want, heads, group, new, lengths = FORMS[form]
    rng = np.random.default_rng(5)
    n = sum(lengths)
    size = rng.choice([1.0, 2.0 ** -24, 1e-5, 0.0, 1000.0, 1e-3, 30000.0, 3.0, 2.0 ** -14], -(-n // 32)).repeat(32)[:n, None, None]
    k = rng.standard_normal((n, heads, 32)).astype(np.float16) * np.float16(4)
    k[5], k[lengths[0] // 2], k[lengths[0] - 3] = 30, -60, 60
    v = (np.clip(rng.standard_normal((n, heads, 32)), -2, 2) * size).astype(np.float16)
    dev = Prompt(heads, group, new, lengths, 32, seed=5, rng=rng, k=k, v=v)
    for scale in (0.125, 5.0, 0.0, 1e-4):
        dev.check(want, scale=scale)
    shape = (sum(new), heads * group, 32)
    dev.check(want, q=np.full(shape, 3.0, np.float16), scale=1.0)
    dev.check(want, q=np.full(shape, -60000.0, np.float16), scale=2.0 ** -15)


def test_scores_that_grow_along_the_axis():
    """Keys whose scores grow from block to block by more than fp16's range in all, and fall: every block raises the maximum, or none does."""
    for form in FORMS:
        want, heads, group, new, lengths = FORMS[form]
        for sign in (1, -1):
            rng = np.random.default_rng(6)
            k = rng.standard_normal((sum(lengths), heads, 32)).astype(np.float16)
            at = np.concatenate([np.arange(t) for t in lengths]) // 32
            k[..., 0] = (sign * 7.0 * (at - at.max() / 2))[:, None]
            dev = Prompt(heads, group, new, lengths, 32, seed=6, rng=rng, k=k, v=rng.standard_normal(k.shape).astype(np.float16))
            q = dev.queries()
            q[..., 0] = 1
            dev.check(want, q=q, scale=1.0)


FEW = {"rows32 parts": ((32, True, False), 2, 3, [40, 1], [4200, 2000]), "rows32 many parts": ((32, True, False), 2, 4, [1], [9000])}


@pytest.mark.parametrize("d", [32, 36])
@pytest.mark.parametrize("form", [*FORMS, *FEW])
def test_strides_and_alignment(form, d):
    """The same bits wherever the rows are, with parts and without."""
    want, heads, group, new, lengths = {**FORMS, **FEW}[form]
    dev = Prompt(heads, group, new, lengths, d, seed=7)
    q = dev.queries()
    rows, hq, _ = q.shape
    plain = dev.check(want, q=q)
    batch = dev.batch(dev.new, dev.lengths())
    dev.expect(want, batch)
    for off, extra in [(0, 3), (1, 3), (8, 16)]:
        wide = dev.torch.full((rows * (hq * d + extra) + 16,), 9.0, dtype=dev.torch.float16, device="cuda")

        def view(t):
            return t[off:off + rows * (hq * d + extra)].view(rows, hq * d + extra)[:, :hq * d].unflatten(1, (hq, d))
        qs, out = view(wide.clone()), view(wide)
        qs.copy_(dev.dev(q))
        dev.L.kv_attention(dev.cache, batch, qs, out=out)
        assert dev.torch.equal(out, plain)
        out.fill_(9.0)
        assert (wide == 9.0).all()  # nothing was written between the rows


@pytest.mark.parametrize("what", ["rows", "length", "table", "slot", "most_len"])
@pytest.mark.parametrize("form", FORMS)
def test_batches_that_cannot_be(form, what):
    """One more sequence, which cannot be: the others are served as without it."""
    want, heads, group, new, lengths = FORMS[form]
    dev = Prompt(heads, group, [*new, 40], [*lengths, 80], 32, seed=8)
    q = dev.queries()
    plain = dev.check(want, q=q).clone()
    told, kw, most = dev.lengths(), {}, max(lengths)
    if what == "rows":
        kw["row_start"] = dev.dev(np.cumsum([0, *new, 41]).astype(np.int32))
    elif what == "length":
        told[-1] = -1
    elif what == "table":
        told[-1] = 32 * dev.pages.shape[1] + 1
        most = told[-1]
    elif what == "slot":
        kw["slots"] = dev.dev(np.array([*dev.slots_np[:-1], -1], np.int32))
    else:
        told[-1] = most + 1
    out = dev.torch.full(q.shape, 7.0, dtype=dev.torch.float16, device="cuda")
    batch = dev.batch(dev.new, told, max_len=most, **kw)
    dev.expect(want, batch)
    dev.L.kv_attention(dev.cache, batch, dev.dev(q), out=out)
    assert int(dev.status) == dev.L.KV_BAD_BATCH
    if what == "table":  # (a longer axis is cut up otherwise)
        assert ((out[:-40] - plain[:-40]).abs() <= 2e-3 * plain.abs().max()).all()
    else:
        assert dev.torch.equal(out[:-40], plain[:-40])
    if what != "rows":
        assert (out[-40:] == 0).all()


@pytest.mark.parametrize("form", FORMS)
def test_on_another_stream_and_in_a_graph(form):
    """Recorded once, replayed as the sequences grow into the pages they have, against the same calls made directly."""
    import torch

    want, heads, group, new, lengths = FORMS[form]
    most = max(lengths) + 96
    dev = Device(len(new), heads, 32, page=32, most=most, seed=9)
    rng = np.random.default_rng(9)
    dev.append(lengths, rng, rot=table(most, 32))
    q = dev.dev(rng.standard_normal((sum(new), heads * group, 32)).astype(np.float16))
    batch = dev.batch(new, lengths, max_len=most)
    p = dev.L.debug_kv_plan_for(dev.cache, batch, heads * group)
    assert (p.tile, p.parts > 1, bool(p.halves)) == want
    ws, out = dev.L.kv_attention_workspace(dev.cache, batch, heads * group), torch.empty_like(q)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dev.L.kv_attention(dev.cache, batch, q, ws=ws, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, dev.L.kv_attention(dev.cache, batch, q))
    with torch.cuda.graph(graph):
        dev.L.kv_attention(dev.cache, batch, q, ws=ws, out=out)
    for turn in range(4):
        if turn:
            dev.append([31] * len(new), rng, rot=table(most, 32))
            batch.kv_len.copy_(dev.dev(np.array(dev.lengths(), np.int32)))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dev.L.kv_attention(dev.cache, batch, q)), turn
        row = 0
        for s, n in zip(dev.seq, new):
            t = s.x.shape[2]
            ref, tol = attention64(q[row:row + n].cpu().numpy(), s.held(), np.arange(t - n, t), 32 ** -0.5)
            assert ((out[row:row + n].double() - ref).abs() <= tol).all(), turn
            row += n
    assert int(dev.status) == 0
