"""A plain 64-bit implementation of the 8-bit key/value cache and its attention, and batches to try them on."""
import numpy as np

BLOCK, RING = 32, 64


def dpad(d):
    return (d + 31) // 32 * 32


def rotate(x, pos, cos, sin, pairs):
    """x [rows, heads, d] fp16 turned by the rows of cos, sin [n_pos, half] at `pos`: fp32, every operation rounded."""
    if cos is None:
        return x
    half = cos.shape[1]
    y = x.astype(np.float32)
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    c, s = cos[pos][:, None], sin[pos][:, None]
    first, second = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    y[..., a], y[..., b] = first, second
    with np.errstate(over="ignore"):
        return y.astype(np.float16)


def finite(x):
    return np.nan_to_num(x, nan=0.0, posinf=65504.0, neginf=-65504.0)


class Sequence:
    """What the cache holds of one sequence: every position's fp16 key and value, [2, heads, len, d]."""

    def __init__(self, heads, d):
        self.x = np.zeros((2, heads, 0, d), np.float16)
        self.greatest = 0  # length that it has had

    def append(self, k, v):
        """k, v [n, heads, d], rotated."""
        self.x = np.concatenate((self.x, finite(np.stack((k, v)).transpose(0, 2, 1, 3))), 2)
        self.greatest = max(self.greatest, self.x.shape[2])

    def block(self, j):
        """Constants [2, heads] and codes [2, heads, 32, d] of a full block."""
        x = self.x[:, :, j * BLOCK:(j + 1) * BLOCK].astype(np.float64)
        c = np.abs(x).max((2, 3))
        with np.errstate(divide="ignore", invalid="ignore"):
            q = np.where(c[..., None, None] > 0, np.rint(127.0 * x / c[..., None, None]), 0.0)
        return c, q.astype(np.int8)

    def held(self, length=None):
        """Keys and values as held, 64 bits: [2, heads, length, d]."""
        n = self.x.shape[2] if length is None else length
        y = self.x[:, :, :n].astype(np.float64)
        for j in range(n // BLOCK):
            c, q = self.block(j)
            y[:, :, j * BLOCK:(j + 1) * BLOCK] = c[..., None, None] * q / 127.0
        return y


def tiles(q, values):
    """Codes [32, d] of a block as its tiles, byte by byte from the layout's definition."""
    d = q.shape[1]
    out = np.zeros(BLOCK * dpad(d), np.int8)
    r, f = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    if values:
        at = f // 32 * 1024 + r // 4 % 2 * 512 + f % 32 * 16 + r // 8 * 4 + r % 4
    else:
        at = f // 32 * 1024 + f % 32 // 16 * 512 + r * 16 + f % 16
    out[at] = q
    return out


def attention(q, held, pos, scale, causal=True, window=0):
    """q [rows, heads_q, d] at positions pos over held [2, heads, len, d], 64 bits -> (out, tolerance), both [rows, heads_q, d].

    The tolerance is that of the number formats, by value: with w the weights, A = sum w |v|, V = max |v| and
    E = scale max_j sum |q||k_j|:  scores are sums of d products in fp32, each step off by 2^-24 of at most E, and are
    scaled and exponentiated with a few more such errors (16 allowed): weights off by 2 (d + 16) 2^-24 E + 2^-19 of themselves,
    numerator and denominator sums over n by n 2^-24 at worst; a weight is rounded to fp16 (2^-11 of itself, or
    2^-25 absolute, where the largest is 1), and so may a value be (2^-11); the result is rounded to fp16 (2^-11, or 2^-25)."""
    rows, hq, d = q.shape
    heads, n = held.shape[1:3]
    g = hq // heads
    out, tol = np.zeros((rows, hq, d)), np.zeros((rows, hq, d))
    j = np.arange(n)
    for h in range(hq):
        k, v = held[0, h // g], held[1, h // g]
        s = q[:, h].astype(np.float64) @ k.T * scale
        see = np.ones_like(s, bool) if not causal else j <= pos[:, None]
        if window:
            see &= j > pos[:, None] - window
        some = see.any(1)
        s = np.where(see, s, -np.inf)
        m = np.where(some, s.max(1, initial=-np.inf), 0.0)
        w = np.exp(s - m[:, None])
        l = np.where(some, w.sum(1), 1.0)[:, None]
        o = w @ v / l
        size = w @ np.abs(v) / l
        e = scale * np.where(see, np.abs(q[:, h].astype(np.float64)) @ np.abs(k).T, 0.0).max(1, initial=0.0)[:, None]
        seen = see.sum(1)[:, None]
        top = np.abs(v).max(initial=0.0)
        rel = 4 * (d + 16) * 2.0 ** -24 * e + 2.0 ** -19 + 2 * seen * 2.0 ** -24 + 2 * 2.0 ** -11
        out[:, h] = o
        tol[:, h] = (rel * size + 2.0 ** -11 * np.abs(o) + 2.0 ** -25 + seen * 2.0 ** -25 * top / l) * some[:, None]
    return out, tol


def table(n_pos, rot):
    a = np.outer(np.arange(n_pos), 10000.0 ** (-np.arange(0, rot, 2) / rot))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


class Device:
    """A cache on the GPU whose unused places hold garbage, and the sequences in it."""

    def __init__(self, seqs, heads, d, page=64, most=512, seed=0, spare=3):
        import torch

        import paper_2208_07339_amd as L
        self.L, self.torch, self.heads, self.d, self.page = L, torch, heads, d, page
        rng = np.random.default_rng(seed)
        per = -(-most // page)
        n_pages = seqs * per + spare
        self.pages_np = rng.permutation(n_pages)[:seqs * per].reshape(seqs, per).astype(np.int32)
        self.slots_np = rng.permutation(seqs + 2)[:seqs].astype(np.int32)
        self.cache = L.KvCache.allocate(n_pages, page, seqs + 2, heads, d)
        self.cache.codes.fill_(77)
        self.cache.consts.fill_(float("nan"))
        self.cache.ring.fill_(float("nan"))
        self.pages, self.slots = self.dev(self.pages_np), self.dev(self.slots_np)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.seq = [Sequence(heads, d) for _ in range(seqs)]

    def dev(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def batch(self, new, lengths, max_rows=None, max_len=None, **kw):
        start = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        args = dict(row_start=self.dev(start), kv_len=self.dev(np.asarray(lengths, np.int32)), pages=self.pages, slots=self.slots,
                    n_rows=max(1, int(start[-1])), max_rows=max_rows or max(1, max(new)),
                    max_len=max(lengths) if max_len is None else max_len, status=self.status)
        args.update(kw)
        return self.L.KvBatch(**args)

    def lengths(self):
        return [s.x.shape[2] for s in self.seq]

    def positions(self, new, lengths):
        return np.concatenate([np.arange(t - n, t) for n, t in zip(new, lengths)]).astype(np.int64)

    def append(self, new, rng, rot=None, pairs=False, heads_q=0, k=None, v=None, wide=0, strided=False):
        """Appends random rows; checks the rotated queries bit for bit.  strided: rows are slices of wider ones."""
        T = sum(new)
        lengths = [a + n for a, n in zip(self.lengths(), new)]
        pos = self.positions(new, lengths)
        if k is None:
            k, v = ((rng.standard_normal((T, self.heads, self.d)) * s).astype(np.float16) for s in (2.0, 1.0))
        q = rng.standard_normal((T, max(1, heads_q), self.d)).astype(np.float16)
        cos, sin = rot if rot is not None else (None, None)
        if strided:
            joint = self.dev(np.concatenate((q, k, v, q[:, :1, :]), 1))
            qd, kd, vd, _ = joint.split([q.shape[1], self.heads, self.heads, 1], 1)
        else:
            qd, kd, vd = self.dev(q), self.dev(k), self.dev(v)
        kw = {} if cos is None else dict(cos=self.dev(cos), sin=self.dev(sin), pairs=pairs)
        q_out = self.L.kv_append(self.cache, self.batch(new, lengths), kd, vd, q=qd if heads_q else None, **kw)
        kr, row = rotate(k, pos, cos, sin, pairs), 0
        for s, n in zip(self.seq, new):
            s.append(kr[row:row + n], v[row:row + n])
            row += n
        if heads_q:
            want = rotate(q, pos, cos, sin, pairs)
            assert np.array_equal(q_out.cpu().numpy().view(np.uint16), want.view(np.uint16))
        return q

    def check_held(self):
        """Codes, constants and the ring, bit for bit: there, the open block and the 32 positions below the greatest length."""
        codes, consts, ring = (t.cpu().numpy() for t in (self.cache.codes, self.cache.consts, self.cache.ring))
        bpp = self.page // BLOCK
        for b, s in enumerate(self.seq):
            n = s.x.shape[2]
            for j in range(n // BLOCK):
                c, q = s.block(j)
                at, sub = self.pages_np[b, j // bpp], j % bpp
                for h in range(self.heads):
                    for kv in range(2):
                        assert consts[at, h, sub, kv] == c[kv, h], (b, j, h, kv)
                        got, want = codes[at, h, sub, kv], tiles(q[kv, h], kv == 1)
                        assert np.array_equal(got, want), (b, j, h, kv, int((got != want).sum()))
            p = np.arange(max(0, min(n // BLOCK * BLOCK, s.greatest - BLOCK)), n)
            got = ring[self.slots_np[b]][:, :, p % RING].transpose(1, 0, 2, 3)
            assert np.array_equal(got.view(np.uint16), np.ascontiguousarray(s.x[:, :, p]).view(np.uint16)), b

    def check_read(self):
        n = self.lengths()
        if not sum(n):
            return
        k, v = self.L.kv_read(self.cache, self.batch(n, n))
        row = 0
        for s in self.seq:
            want = s.held().astype(np.float16).transpose(0, 2, 1, 3)
            m = want.shape[1]
            for got, w in zip((k, v), want):
                assert np.array_equal(got[row:row + m].cpu().numpy(), w)
            row += m

    def check_attention(self, new, rng, group=1, lengths=None, scale=None, causal=True, window=0, q=None, idle=(), **kw):
        lengths = self.lengths() if lengths is None else list(lengths)
        T = sum(new)
        if q is None:
            q = rng.standard_normal((T, self.heads * group, self.d)).astype(np.float16)
        scale = self.d ** -0.5 if scale is None else scale
        told = [0 if b in idle else n for b, n in enumerate(lengths)]
        out = self.L.kv_attention(self.cache, self.batch(new, told, **kw), self.dev(q), scale=scale, causal=causal, window=window)
        got, row = out.cpu().numpy().astype(np.float64), 0
        for b, (s, n, t) in enumerate(zip(self.seq, new, told)):
            want, tol = attention(q[row:row + n], s.held(t), np.arange(t - n, t), scale, causal, window)
            far = np.abs(got[row:row + n] - want)
            assert (far <= tol).all(), (b, n, t, float((far - tol).max()), float(far.max()))
            row += n
        return out
