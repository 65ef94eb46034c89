"""The example's decoder attention layer: prompts and captured steps against the operators' 64-bit implementation, fed with the
layer's own projections, and against the layer run at once."""
import os
import sys

import numpy as np
import pytest

from kv_util import Sequence, attention, rotate, table

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("heads_q, heads, d", [(4, 4, 64), (8, 2, 80)])
def test_layer(heads_q, heads, d):
    import torch

    import decoder_attention as E
    import paper_2208_07339_amd as L
    hidden, prompts, steps = heads_q * d, [70, 1, 33], 40
    most, n = max(prompts) + steps, len(prompts)
    rng = np.random.default_rng(0)
    cos, sin = table(most, d)

    def dev(a):
        return torch.from_numpy(a).cuda()

    def weight(h, o):
        return (rng.standard_normal((h, o)) * h ** -0.5).astype(np.float16)
    w_qkv, w_out = weight(hidden, (heads_q + 2 * heads) * d), weight(hidden, hidden)

    def layer():
        cache = L.KvCache.allocate(n * -(-most // 64), 64, n, heads, d)
        return E.Attention(dev(w_qkv), dev(w_out), heads_q, cache, n * most, dev(cos), dev(sin)), E.Sequences(n, cache, most)

    one, seqs = layer()
    held = [Sequence(heads, d) for _ in range(n)]
    plain = E.Linear(dev(w_qkv), n * most)

    def check(x, att, new):
        """The layer's attention for rows x; appends to `held`."""
        q, k, v = np.split(plain(dev(x)).cpu().numpy().reshape(len(x), -1, d), [heads_q, heads_q + heads], 1)
        row = 0
        for s, m in zip(held, new):
            r, pos = slice(row, row + m), np.arange(m) + s.x.shape[2]
            s.append(rotate(k[r], pos, cos, sin, False), v[r])
            want, tol = attention(rotate(q[r], pos, cos, sin, False), s.held(), pos, d ** -0.5)
            assert (np.abs(att[r] - want) <= tol).all()
            row += m

    x = [rng.standard_normal((m + steps, hidden)).astype(np.float16) for m in prompts]
    first = np.concatenate([y[:m] for y, m in zip(x, prompts)])
    seqs.prompt(one, dev(first), prompts)
    check(first, one.att[:sum(prompts)].cpu().numpy().astype(np.float64), prompts)
    token = torch.zeros((n, hidden), dtype=torch.float16, device="cuda")
    run = seqs.step(one, token)
    assert seqs.kv_len.tolist() == prompts
    for i in range(steps):
        now = np.stack([y[m + i] for y, m in zip(x, prompts)])
        token.copy_(dev(now))
        out = run().clone()
        check(now, one.att[:n].cpu().numpy().astype(np.float64), [1] * n)
        assert torch.equal(out, E.Linear(dev(w_out), n)(one.att[:n].reshape(n, -1)))
    assert seqs.kv_len.tolist() == [m + steps for m in prompts] and seqs.status.item() == 0


def test_example_runs():
    import decoder_attention as E
    E.main(["--hidden", "256", "--heads-q", "4", "--heads", "2", "--prompts", "100,1,40", "--tokens", "33"])
