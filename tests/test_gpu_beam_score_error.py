"""How far beam_select's scores may be off.  A sum of exponentials is made in fp32 where no comparison hangs on it: in units of 2^-24 of it,
the exponentials' arguments are off by (fp16: 1.25, fp32: 2.25) times sum p (max - x) <= log(vocab), an exponential by 2, the sum of 8 by
3, and 1 for the rest; two scores that are not further apart than twice that are compared by sums in 64 bits.  scores_out has that error and one
rounding to fp32 (2^-24 relative)."""
import numpy as np
import pytest

from beam_util import select
from test_gpu_beam_select import made

pytestmark = pytest.mark.gpu


def tolerance(vocab, f32, s):
    return 2.0 ** -24 * ((2.25 if f32 else 1.25) * np.log(vocab) + 6.0 + np.abs(s))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("spread", [0.0, 0.1, 1.0, 3.0, 12.0])
@pytest.mark.parametrize("items, beams, vocab, n_out", [(4, 4, 1, 1), (8, 4, 7, 4), (8, 4, 2049, 8), (30, 8, 8192, 4), (4, 3, 50257, 8), (40, 4, 50257, 4),
                                                        (70, 4, 30001, 4), (1, 2, 400001, 4)])
def test_scores(items, beams, vocab, n_out, spread, f32):
    import torch

    import paper_2208_07339_amd as L
    logits, scores = made(torch, vocab + items, items * beams, vocab, f32, spread)
    logits[::3] += 40.0   # (a distance to 0 that the arguments' rounding would show)
    logits[1::3] -= 900.0
    scores = scores * 0.05
    s, parent, token, _ = (t.cpu().numpy() for t in L.beam_select(logits, scores, beams, n_out))
    want = select(logits.cpu().numpy(), scores.cpu().numpy(), beams, n_out)
    assert np.array_equal(parent, want[1]) and np.array_equal(token, want[2])
    there = want[1] >= 0
    off = np.abs(s[there].astype(np.float64) - want[0][there])
    assert (off <= tolerance(vocab, f32, want[0][there])).all(), (off / tolerance(vocab, f32, want[0][there])).max()
