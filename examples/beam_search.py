"""Beam search with a small decoder whose products and cache are in 8 bits: one captured step, replayed.

    python examples/beam_search.py [--layers 2 --hidden 2048 --heads-q 16 --heads 16 --vocab 32000 --prompts 300,17 --beams 4 --tokens 48]

A step: the best continuations (llmint8_beam_select), the sequences they come from (llmint8_kv_fork), pages for the next token
(llmint8_kv_reserve), then in every layer the copies that follow (llmint8_kv_copy) and the layer itself (decoder_attention.py), then the
logits (llmint8_linear).  Nothing of it waits for the host.  Weights are random, so the answers mean nothing.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2208_07339_amd as L  # noqa: E402
from decoder_attention import Attention, Linear  # noqa: E402

PAGE = 64


class Decoder:
    """Layers of attention between an embedding and its logits, with room for items x beams sequences of up to `most` positions."""

    def __init__(self, layers, hidden, heads_q, heads, vocab, items, beams, most, rows, n_pages=None):
        d, dev, n = hidden // heads_q, "cuda", items * beams
        self.items, self.beams, self.n, self.most = items, beams, n, most
        per = -(-most // PAGE)
        angle = torch.outer(torch.arange(most), 10000.0 ** (-torch.arange(0, d, 2) / d)).cuda()
        self.pool = L.KvPool.allocate(n * per if n_pages is None else n_pages, PAGE)
        self.seqs = L.KvSeqs.allocate(n, per)
        self.moves = L.KvMoves.allocate(n, n)

        def weight(h, o):
            return (torch.randn(h, o, device=dev) * h ** -0.5).half()
        self.layers = []
        for _ in range(layers):
            cache = L.KvCache.allocate(self.pool.refs.numel(), PAGE, n, heads, d)
            self.layers.append(Attention(weight(hidden, (heads_q + 2 * heads) * d), weight(hidden, hidden), heads_q, cache, rows,
                                         angle.cos(), angle.sin()))
        self.embedding = torch.randn(vocab, hidden, device=dev).half()
        self.head = Linear(weight(hidden, vocab), n)
        # the search: scores and ends of the beams, what a step selects, and the tokens so far
        self.scores = torch.empty(n, device=dev)
        self.ended, self.parent, self.token, self.ready = (torch.zeros(n, dtype=torch.int32, device=dev) for _ in range(4))
        self.logits = torch.zeros((n, vocab), dtype=torch.float16, device=dev)
        self.answers = torch.zeros((n, most), dtype=torch.int64, device=dev)
        self.at = torch.zeros(1, dtype=torch.int64, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ws = L.beam_select_workspace(items, beams, vocab, beams)
        self.starts = torch.arange(n + 1, dtype=torch.int32, device=dev)
        self.one = L.KvBatch(self.starts, self.ready, self.seqs.pages, self.seqs.slots, n, 1, most, self.seqs.status)
        self.one_ws = L.kv_attention_workspace(self.layers[0].cache, self.one, heads_q)

    def forward(self, x, batch, ws):
        for layer in self.layers:
            L.kv_copy(layer.cache, self.moves, self.status)
            x = x + layer(x, batch, ws)
            x = (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True))).half()
        return x

    def prompt(self, prompts):
        """prompts: a list of tokens for each item, in the item's first sequence."""
        b, n = self.beams, self.n
        rows = [len(prompts[i // b]) if i % b == 0 else 0 for i in range(n)]
        start = torch.tensor([0] + rows, device="cuda").cumsum(0).to(torch.int32)
        self.seqs.kv_len.copy_(torch.tensor(rows, dtype=torch.int32))
        L.kv_reserve(self.pool, self.seqs, start, self.moves, ready=self.ready)
        batch = L.KvBatch(start, self.ready, self.seqs.pages, self.seqs.slots, sum(rows), max(rows), self.most, self.seqs.status)
        x = self.embedding[torch.tensor([t for p in prompts for t in p], device="cuda")]
        x = self.forward(x, batch, L.kv_attention_workspace(self.layers[0].cache, batch, self.layers[0].heads_q))
        last = x[start[1::b].long() - 1]
        self.logits.view(self.items, b, -1)[:, 0] = self.head(last)
        self.scores.fill_(float("-inf"))  # one beam an item to begin with
        self.scores.view(self.items, b)[:, 0] = 0.0

    def step(self, eos):
        L.beam_select(self.logits, self.scores, self.beams, ended=self.ended, eos=eos, ws=self.ws, status=self.status,
                      out=[self.scores, self.parent, self.token, self.ended])
        self.answers.copy_(self.answers[self.parent.clamp(min=0).long()])
        self.answers.scatter_(1, self.at.expand(self.n, 1), self.token.long()[:, None])
        self.at += 1
        L.kv_fork(self.pool, self.seqs, self.parent, self.moves, grow=1)
        L.kv_reserve(self.pool, self.seqs, self.starts, self.moves, ready=self.ready, more=True)
        x = self.forward(self.embedding[self.token.long()], self.one, self.one_ws)
        self.logits.copy_(self.head(x))

    def captured(self, eos):
        """-> a function that makes a step, from a graph; has made one."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(eos)  # a step of its own, which also sets up what a library sets up at first
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step(eos)
        return graph.replay


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("hidden", 2048), ("heads-q", 16), ("heads", 16), ("vocab", 32000), ("beams", 4), ("tokens", 48)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--prompts", type=lambda s: [int(x) for x in s.split(",")], default=[300, 17])
    a = p.parse_args(argv)
    torch.manual_seed(0)
    eos, most = 2, max(a.prompts) + a.tokens
    model = Decoder(a.layers, a.hidden, a.heads_q, a.heads, a.vocab, len(a.prompts), a.beams, most, max(sum(a.prompts), len(a.prompts) * a.beams))
    model.prompt([torch.randint(3, a.vocab, (n,)).tolist() for n in a.prompts])
    run = model.captured(eos)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(a.tokens - 1):
        run()
    end.record()
    end.synchronize()
    print(f"{a.tokens - 1} steps of {len(a.prompts)} x {a.beams} beams: {begin.elapsed_time(end) / (a.tokens - 1) * 1e3:.1f} us a step")
    answers = model.answers[:, :a.tokens].view(len(a.prompts), a.beams, -1)
    for i, s in enumerate(model.scores.view(len(a.prompts), a.beams).tolist()):
        print(f"item {i}: scores {[round(x, 3) for x in s]}, best {answers[i, 0, :12].tolist()} ...")
    held = int((model.pool.refs > 0).sum())
    alone = int((-(-model.seqs.kv_len // PAGE)).sum())
    print(f"pages held: {held}; sequences with pages of their own would hold {alone}")
    assert model.status.item() == 0 and model.seqs.status.item() == 0
    return model


if __name__ == "__main__":
    main()
