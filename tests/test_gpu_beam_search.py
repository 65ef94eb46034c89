"""The operators of a beam search together: selection, forks, pages and copies, append and attention over the cache, against beams that
share nothing.  What a cache holds depends on the tokens alone and attention on what it holds, so everything is equal bit for bit."""
import os
import random
import sys

import numpy as np
import pytest

from beam_util import LSE_ERROR, select

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def ints(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("items, beams, heads_q, heads, d, page, prompts, steps", [
    (2, 4, 4, 2, 64, 64, (70, 1), 80), (3, 3, 2, 2, 33, 32, (31, 64, 200), 70), (1, 8, 8, 1, 128, 128, (500,), 100), (2, 2, 1, 1, 100, 96, (5, 95), 75)])
def test_search(items, beams, heads_q, heads, d, page, prompts, steps):
    import torch

    import paper_2208_07339_amd as L
    g = torch.Generator(device="cuda")
    g.manual_seed(items * 100 + d)
    r = random.Random(3)
    n, vocab, most = items * beams, 300, max(prompts) + steps + 1
    per = -(-most // page)
    # a model that is nothing but tables: queries, keys and values of a token, and logits from what attention gives
    table = torch.randn(vocab, heads_q + 2 * heads, d, device="cuda", generator=g).half()
    out = torch.randn(heads_q * d, vocab, device="cuda", generator=g) * (heads_q * d) ** -0.5 * 6
    cos = torch.randn(most, d // 2, device="cuda", generator=g)
    sin = (1 - cos.square().clamp(max=1)).sqrt()
    # fewer pages than sequences that share nothing would need
    n_pages = items * per + n * 3
    cache = L.KvCache.allocate(n_pages, page, n, heads, d)
    pool, seqs, moves = L.KvPool.allocate(n_pages, page), L.KvSeqs.allocate(n, per), L.KvMoves.allocate(max(n, n_pages // 2), n)
    ready, status = ints(torch, [0] * n), ints(torch, [0])
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")

    def layer(c, batch, tokens):
        q, k, v = table[tokens].split([heads_q, heads, heads], 1)
        q = L.kv_append(c, batch, k.contiguous(), v.contiguous(), q=q.contiguous(), cos=cos, sin=sin)
        return q, L.kv_attention(c, batch, q)

    def logits_of(att):
        return (att.flatten(1).float() @ out).half()

    # the prompts, in each item's first sequence
    held = [[] for _ in range(n)]
    rows = [0] * n
    for i, m in enumerate(prompts):
        held[i * beams] = [r.randrange(vocab) for _ in range(m)]
        rows[i * beams] = m
    start = ints(torch, np.concatenate([[0], np.cumsum(rows)]).tolist())
    seqs.kv_len.copy_(ints(torch, rows))
    L.kv_reserve(pool, seqs, start, moves, ready=ready)
    batch = L.KvBatch(start, ready, seqs.pages, seqs.slots, sum(rows), max(rows), most, status)
    _, att = layer(cache, batch, torch.tensor(sum(held, []), device="cuda"))
    logits = torch.full((n, vocab), float("nan"), dtype=torch.float16, device="cuda")  # of beams that there are not: not read
    logits[::beams] = logits_of(att[start[1::beams].long() - 1])
    scores = torch.full((n,), float("-inf"), device="cuda")
    scores[::beams] = 0.0
    ended = ints(torch, [0] * n)
    one = L.KvBatch(starts, ready, seqs.pages, seqs.slots, n, 1, most, status)

    def alone(q):
        """A cache of sequences that share nothing, filled at once; its contents and what attention over it gives."""
        c = L.KvCache.allocate(n * per, page, n, heads, d)
        pages = torch.arange(n * per, dtype=torch.int32, device="cuda").view(n, per)
        lengths = [len(h) for h in held]
        b = L.KvBatch(ints(torch, np.concatenate([[0], np.cumsum(lengths)]).tolist()), ints(torch, lengths), pages, None, sum(lengths), max(lengths), most)
        _, k, v = table[torch.tensor(sum(held, []), device="cuda")].split([heads_q, heads, heads], 1)
        L.kv_append(c, b, k.contiguous(), v.contiguous(), cos=cos, sin=sin)
        return L.kv_read(c, b), L.kv_attention(c, L.KvBatch(starts, ints(torch, lengths), pages, None, n, 1, most), q)

    for step in range(steps):
        want = select(logits.cpu().numpy(), scores.cpu().numpy(), beams, beams, ended.tolist(), 7)
        s, parent, token, over = L.beam_select(logits, scores, beams, ended=ended, eos=7, status=status)
        assert np.array_equal(parent.cpu().numpy(), want[1]) and np.array_equal(token.cpu().numpy(), want[2])
        assert (np.abs(s.cpu().numpy() - want[0]) <= LSE_ERROR + 2.0 ** -24 * np.abs(want[0])).all()
        scores, ended = s.flatten(), over.flatten()
        held = [held[p] + [t] for p, t in zip(parent.flatten().tolist(), token.flatten().tolist())]
        L.kv_fork(pool, seqs, parent.flatten(), moves, grow=1)
        if step % 11 == 5:  # pages without gaps, now and then: the fork's copies first
            L.kv_copy(cache, moves, status)
            L.kv_compact(pool, seqs, moves)
            L.kv_copy(cache, moves, status)
            assert (pool.refs > 0).tolist() == sorted((pool.refs > 0).tolist(), reverse=True)
            L.kv_reserve(pool, seqs, starts, moves, ready=ready)
        else:
            L.kv_reserve(pool, seqs, starts, moves, ready=ready, more=True)
        assert ready.tolist() == seqs.kv_len.tolist() == [len(h) for h in held]
        L.kv_copy(cache, moves, status)
        q, att = layer(cache, one, token.flatten().long())
        logits = logits_of(att)
        if step % 6 == 0 or step == steps - 1:
            (k, v), same = alone(q)
            lengths = [len(h) for h in held]
            all_rows = L.KvBatch(ints(torch, np.concatenate([[0], np.cumsum(lengths)]).tolist()), seqs.kv_len, seqs.pages, seqs.slots, sum(lengths),
                                 max(lengths), most, status)
            got = L.kv_read(cache, all_rows)
            assert torch.equal(got[0], k) and torch.equal(got[1], v)
            assert torch.equal(att, same)
    assert status.item() == 0 and seqs.status.item() == 0
    # everything is given back
    L.kv_fork(pool, seqs, ints(torch, [-1] * n), moves)
    assert not pool.refs.any() and (seqs.pages == -1).all() and not seqs.kv_len.any()


def test_samples_are_shortened_after_a_fork():
    """Children may drop positions as llmint8_kv_batch_t says, down to 32 below their length, and go on from there with other tokens; the
    other children keep theirs."""
    import torch

    import paper_2208_07339_amd as L
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    heads, d, page, n, most = 2, 64, 64, 4, 400
    x = torch.randn(2, n, most, heads, d, device="cuda", generator=g).half()  # keys and values that sequence b has at a position
    x[:, 1:, :150] = x[:, :1, :150]
    for length in (150, 160, 191, 129):
        cache = L.KvCache.allocate(40, page, n, heads, d)
        pool, seqs, moves = L.KvPool.allocate(40, page), L.KvSeqs.allocate(n, 7), L.KvMoves.allocate(20, n)
        ready, status = ints(torch, [0] * n), ints(torch, [0])

        def put(rows, first):
            """Sequence b's positions first[b] .. + rows[b]."""
            start = ints(torch, np.concatenate([[0], np.cumsum(rows)]).tolist())
            seqs.kv_len.copy_(ints(torch, [f + m for f, m in zip(first, rows)]))
            L.kv_reserve(pool, seqs, start, moves, ready=ready, more=True)
            L.kv_copy(cache, moves, status)
            k, v = (torch.cat([x[w, b, f:f + m] for b, (f, m) in enumerate(zip(first, rows))]) for w in range(2))
            L.kv_append(cache, L.KvBatch(start, ready, seqs.pages, seqs.slots, sum(rows), max(rows), most, status), k, v)

        x[:, 1:, 150:length] = x[:, :1, 150:length] if length > 150 else 0
        put([length, 0, 0, 0], [0] * 4)
        L.kv_fork(pool, seqs, ints(torch, [0, 0, 0, 0]), moves)
        drop = [0, 1, 17, 32]
        old = [length - y for y in drop]
        want = x.clone()
        for b in range(n):
            want[:, b, :old[b]] = x[:, 0, :old[b]]
        new = torch.randn(2, n, most, heads, d, device="cuda", generator=g).half()
        x = want.clone()
        for b in range(n):
            x[:, b, old[b]:] = new[:, b, old[b]:]
        put([70, 70, 33, 100], old)
        total = [o + m for o, m in zip(old, [70, 70, 33, 100])]
        # the same sequences, each by itself
        pages = torch.arange(28, dtype=torch.int32, device="cuda").view(n, 7)
        start = ints(torch, np.concatenate([[0], np.cumsum(total)]).tolist())
        plain = L.KvCache.allocate(28, page, n, heads, d)
        b = L.KvBatch(start, ints(torch, total), pages, None, sum(total), max(total), most)
        k, v = (torch.cat([x[w, q, :total[q]] for q in range(n)]) for w in range(2))
        L.kv_append(plain, b, k, v)
        got = L.kv_read(cache, L.KvBatch(start, ready, seqs.pages, seqs.slots, sum(total), max(total), most, status))
        for y, z in zip(got, L.kv_read(plain, b)):
            assert torch.equal(y, z)
        assert status.item() == 0
        x[:, 1:, :150] = x[:, :1, :150]


def test_example():
    import torch

    import beam_search as E
    args = ["--layers", "2", "--hidden", "256", "--heads-q", "4", "--heads", "2", "--vocab", "500", "--prompts", "70,3,40", "--beams", "3", "--tokens", "40"]
    model = E.main(args)
    # the same search without a graph
    torch.manual_seed(0)
    prompts = [70, 3, 40]
    other = E.Decoder(2, 256, 4, 2, 500, 3, 3, max(prompts) + 40, sum(prompts))
    other.prompt([torch.randint(3, 500, (n,)).tolist() for n in prompts])
    for _ in range(40):
        other.step(2)
    assert torch.equal(model.answers, other.answers) and torch.equal(model.scores, other.scores)
    assert torch.equal(model.pool.refs, other.pool.refs) and torch.equal(model.seqs.pages, other.seqs.pages)
