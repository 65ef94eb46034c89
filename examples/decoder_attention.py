"""A decoder's attention layer in 8 bits, as it serves: ragged prompts, then a token a sequence at a time.

    python examples/decoder_attention.py [--hidden 4096 --heads-q 32 --heads 32 --prompts 2048,1000,17 --tokens 64]

Joint projection (llmint8_linear) -> rotation and cache (llmint8_kv_append) -> attention over the cache
(llmint8_kv_attention) -> output projection (llmint8_linear), all on one stream, in buffers allocated once; the step for a token a
sequence is captured into a graph and replayed.  Weights and inputs are random.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2208_07339_amd as L  # noqa: E402

ALPHA, CAP = 6.0, 32  # outlier threshold, most outlier columns


class Linear:
    """x W for up to s rows, W [h, o] held in 8 bits."""

    def __init__(self, W, s):
        (h, o), dev = W.shape, W.device
        self.qw, self.out = L.quantize_weight(W), torch.empty((s, o), dtype=torch.float16, device=dev)
        self.outl = L.Outliers(*(torch.zeros(n, dtype=torch.int32, device=dev) for n in (CAP, 1, 1)), CAP)
        self.rows = L.QuantizedRows(torch.empty(L.xq_bytes(s, h), dtype=torch.int8, device=dev),
                                    torch.empty(s, dtype=torch.float16, device=dev),
                                    torch.empty((s, L.opad(CAP)), dtype=torch.float16, device=dev), s, h)
        self.ws = L.Workspace.allocate(s, h, o, CAP, dev)

    def __call__(self, x):
        return L.linear(x, self.qw, ALPHA, self.outl, self.rows, self.ws, self.out[:x.shape[0]])


class Attention:
    """w_qkv [hidden, (heads_q + 2 heads) d], w_out [heads_q d, hidden]; `rows`: the most rows of a call; cos, sin [positions, d / 2]."""

    def __init__(self, w_qkv, w_out, heads_q, cache, rows, cos, sin):
        self.heads_q, self.cache, self.cos, self.sin = heads_q, cache, cos, sin
        self.qkv, self.proj = Linear(w_qkv, rows), Linear(w_out, rows)
        self.att = torch.empty((rows, heads_q, cache.d), dtype=torch.float16, device=w_qkv.device)

    def __call__(self, x, batch, ws):
        n, c = x.shape[0], self.cache
        q, k, v = self.qkv(x).view(n, -1, c.d).split([self.heads_q, c.heads, c.heads], 1)  # slices: nothing is copied
        L.kv_append(c, batch, k, v, q=q, q_out=q, cos=self.cos, sin=self.sin)
        out = L.kv_attention(c, batch, q, ws=ws, out=self.att[:n])
        return self.proj(out.view(n, -1))


class Sequences:
    """Sequences with pages of `cache` for `most` positions each, and the batches of calls for them."""

    def __init__(self, n, cache, most):
        dev, per = cache.codes.device, -(-most // cache.page_tokens)
        self.cache, self.n, self.most = cache, n, most
        self.pages = torch.arange(n * per, dtype=torch.int32, device=dev).view(n, per)
        self.kv_len = torch.zeros(n, dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def batch(self, rows):
        """rows: this call's of each sequence.  The batch reads kv_len when its call runs: add to it before."""
        start = torch.tensor([0] + rows, device=self.kv_len.device).cumsum(0).to(torch.int32)
        return L.KvBatch(row_start=start, kv_len=self.kv_len, pages=self.pages, slots=None, n_rows=sum(rows), max_rows=max(rows),
                         max_len=self.most, status=self.status)

    def prompt(self, layer, x, rows):
        batch = self.batch(rows)
        self.kv_len += torch.tensor(rows, dtype=torch.int32, device=self.kv_len.device)
        return layer(x, batch, L.kv_attention_workspace(self.cache, batch, layer.heads_q))

    def step(self, layer, x):
        """-> a function that runs the layer for one more token of every sequence, x [n, hidden] -> the returned tensor, from a
        graph; runs none itself."""
        batch = self.batch([1] * self.n)
        ws = L.kv_attention_workspace(self.cache, batch, layer.heads_q)
        before = self.kv_len.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # once for the libraries' own set-up, as sequences without positions: the cache stays as it is
            self.kv_len.zero_()
            layer(x, batch, ws)
            self.kv_len.copy_(before)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.kv_len += 1
            out = layer(x, batch, ws)

        def run():
            graph.replay()
            return out
        run.keeps = x, batch, ws  # the graph reads them: they have to live as long as it
        return run


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--heads-q", type=int, default=32)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--prompts", type=lambda s: [int(x) for x in s.split(",")], default=[2048, 1000, 17])
    p.add_argument("--tokens", type=int, default=64)
    a = p.parse_args(argv)
    torch.manual_seed(0)
    d, n, most = a.hidden // a.heads_q, len(a.prompts), max(a.prompts) + a.tokens
    page = 128
    cache = L.KvCache.allocate(n * -(-most // page), page, n, a.heads, d)
    angle = torch.outer(torch.arange(most), 10000.0 ** (-torch.arange(0, d, 2) / d)).cuda()

    def weight(h, o):
        return (torch.randn(h, o, device="cuda") * h ** -0.5).half()
    layer = Attention(weight(a.hidden, (a.heads_q + 2 * a.heads) * d), weight(a.heads_q * d, a.hidden), a.heads_q, cache,
                      sum(a.prompts), angle.cos(), angle.sin())
    seqs = Sequences(n, cache, most)

    def timed(f):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        r = f()
        end.record()
        end.synchronize()
        return r, begin.elapsed_time(end)

    x = torch.randn(sum(a.prompts), a.hidden, device="cuda").half()
    seqs.prompt(layer, x, a.prompts)
    seqs.kv_len.zero_()
    out, ms = timed(lambda: seqs.prompt(layer, x, a.prompts))
    print(f"prompts of {a.prompts}: {ms:.3f} ms, {sum(a.prompts) / ms * 1e3:.0f} tokens/s")
    token = torch.randn(n, a.hidden, device="cuda").half()
    run = seqs.step(layer, token)
    out, ms = timed(lambda: [run() for _ in range(a.tokens)][-1])
    print(f"{a.tokens} steps of {n} sequences: {ms / a.tokens * 1e3:.1f} us a step")
    fp16 = 2 * 2 * cache.heads * d * int(seqs.kv_len.sum())
    print(f"positions {seqs.kv_len.tolist()}, status {seqs.status.item()}; fp16 keys and values of them: {fp16 / 1e6:.1f} MB, held in "
          f"{sum(t.numel() * t.element_size() for t in (cache.codes, cache.consts, cache.ring)) / 1e6:.1f} MB of pages and ring")
    assert seqs.status.item() == 0 and torch.isfinite(out).all()


if __name__ == "__main__":
    main()
