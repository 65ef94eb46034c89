"""beam_select where scores are below fp32's range: logits of a row that are further apart than the largest fp32 number, and beams whose
score is a large negative number over logits masked by the type's lowest value.  Scores are compared in 64 bits, where they are ordinary
numbers, so parents and tokens are those of the definition (beam_util.py); scores_out is -inf where fp32 has no other number for it."""
import numpy as np
import pytest

from beam_util import select
from test_gpu_beam_select import made

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def L(torch):
    import paper_2208_07339_amd as L
    return L


def check(torch, L, logits, scores, beams, n_out, ended=None, eos=-1):
    """-> whether some scores are below fp32's range."""
    e = None if ended is None else torch.tensor(ended, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    s, parent, token, over = (t.cpu().numpy() for t in L.beam_select(logits, scores, beams, n_out, ended=e, eos=eos, status=status))
    want = select(logits.cpu().numpy(), scores.cpu().numpy(), beams, n_out, ended, eos)
    assert np.array_equal(parent, want[1])
    assert np.array_equal(token, want[2])
    assert np.array_equal(over, want[3])
    there = want[1] >= 0
    with np.errstate(over="ignore"):
        below = there & np.isneginf(want[0].astype(np.float32))
    assert np.array_equal(np.isneginf(s), ~there | below)
    near = there & ~below
    # (a sum's error: a few units of 2^-24, as beam_select's kernels derive it for fp32 logits; and one rounding to fp32)
    tolerance = 2.0 ** -24 * (2.25 * np.log(logits.shape[1]) + 6.0 + np.abs(want[0][near]))
    assert (np.abs(s[near].astype(np.float64) - want[0][near]) <= tolerance).all()
    assert status.item() == 0
    return bool(below.any())


# candidates: beams x pieces of 4 096 logits x n_out: up to 128 of them, 129 to 512, more
@pytest.mark.parametrize("items, beams, vocab", [(1, 8, 10000), (3, 4, 50257), (2, 3, 9000), (1, 1, 70000), (2, 32, 600), (1, 16, 4097)])
@pytest.mark.parametrize("n_out", [4, 8, 16, 32])
def test_logits_further_apart_than_the_largest_number(torch, L, items, beams, vocab, n_out):
    logits = torch.full((items * beams, vocab), -2e38, device="cuda")
    logits[torch.arange(items * beams), torch.arange(items * beams) * 7919 % vocab] = 2e38
    scores = -1.0 - torch.arange(items * beams, device="cuda") % 5 * 0.25
    below = check(torch, L, logits, scores, beams, n_out)
    assert below == (n_out > beams)
    # some tokens between them
    logits[:, ::vocab // 5] = 1.5e38
    logits[:, 3::vocab // 3] = -1.9e38
    check(torch, L, logits, scores, beams, n_out)


@pytest.mark.parametrize("score", [LOWEST, -1e30, -3e38])
@pytest.mark.parametrize("items, beams, vocab", [(1, 4, 50257), (2, 8, 10000), (5, 3, 20000), (1, 32, 5000), (2, 2, 40)])
@pytest.mark.parametrize("n_out", [1, 4, 8, 16, 32])
def test_scores_and_masks_of_the_lowest_value(torch, L, items, beams, vocab, n_out, score):
    """Every beam has one token that may follow, or two; the others are masked."""
    logits, _ = made(torch, vocab + n_out, items * beams, vocab, True)
    allowed = torch.zeros(items * beams, vocab, dtype=torch.bool, device="cuda")
    allowed[torch.arange(items * beams), torch.arange(items * beams) * 7919 % vocab] = True
    allowed[::3, vocab // 2] = True
    logits = torch.where(allowed, logits, LOWEST)
    scores = torch.full((items * beams,), score, device="cuda")
    check(torch, L, logits, scores, beams, n_out)
    # one beam that has an ordinary score, and one that has ended
    scores[beams - 1] = -2.0
    check(torch, L, logits, scores, beams, n_out)
    ended = [0] * (items * beams)
    ended[0] = 1
    check(torch, L, logits, scores, beams, n_out, ended, eos=5)


def test_beams_of_the_lowest_value_beside_those_that_there_are_not(torch, L):
    logits, _ = made(torch, 3, 16, 30000, True)
    logits[:, 2:] = LOWEST
    scores = torch.full((16,), LOWEST, device="cuda")
    scores[1::4] = float("-inf")
    logits[2, 5:] = float("-inf")
    logits[6] = float("-inf")
    for n_out in (4, 12, 20, 32):
        check(torch, L, logits, scores, 4, n_out)
