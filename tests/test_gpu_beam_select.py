"""beam_select against its definition in 64 bits (beam_util.py): parents and tokens equal, scores to the error of their sums (LSE_ERROR) and
one rounding to fp32 (half a step, 2^-24 relative)."""
import numpy as np
import pytest

from beam_util import LSE_ERROR, select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def L(torch):
    import paper_2208_07339_amd as L
    return L


def agree(got, want, status=None):
    s, parent, token, ended = (t.cpu().numpy() for t in got)
    assert np.array_equal(parent, want[1])
    assert np.array_equal(token, want[2])
    assert np.array_equal(ended, want[3])
    there = want[1] >= 0
    assert np.array_equal(np.isneginf(s), ~there)
    off = np.abs(s[there].astype(np.float64) - want[0][there])
    assert (off <= LSE_ERROR + 2.0 ** -24 * np.abs(want[0][there])).all(), off.max()
    if status is not None:
        assert status.item() == (1 if want[4] else 0)


def check(torch, L, logits, scores, beams, n_out, ended=None, eos=-1):
    """logits, scores: device tensors; ended: a list or None."""
    e = None if ended is None else torch.tensor(ended, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = L.beam_select(logits, scores, beams, n_out, ended=e, eos=eos, status=status)
    want = select(logits.cpu().numpy(), scores.cpu().numpy(), beams, n_out, ended, eos)
    agree(got, want, status)
    return got, want


def made(torch, seed, rows, vocab, f32, spread=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, vocab, device="cuda", generator=g) * spread
    return x if f32 else x.half(), torch.randn(rows, device="cuda", generator=g) * 2 - 15


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("items, beams, vocab, n_out", [
    (1, 1, 1, 1), (2, 3, 1, 3), (1, 4, 2, 8), (3, 2, 7, 5), (1, 4, 8, 4), (2, 5, 9, 32), (1, 32, 33, 32), (4, 4, 511, 4), (3, 4, 512, 8), (2, 3, 513, 1),
    (2, 4, 2047, 4), (5, 4, 2048, 10), (1, 4, 2049, 4), (1, 2, 4095, 32), (9, 16, 5000, 32), (1, 4, 50257, 4), (16, 8, 32003, 16), (70, 4, 8191, 4),
    (130, 8, 8192, 8), (130, 8, 8193, 8), (300, 4, 4097, 8), (64, 8, 16385, 8), (1, 1, 200000, 32), (2, 32, 70001, 32), (40, 4, 120001, 4)])
def test_sizes(torch, L, items, beams, vocab, n_out, f32):
    logits, scores = made(torch, items * vocab + n_out, items * beams, vocab, f32)
    check(torch, L, logits, scores, beams, n_out)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab", [5, 700, 2048, 6000, 40001])
def test_masks_ends_and_beams_that_there_are_not(torch, L, vocab, f32):
    items, beams = 6, 4
    logits, scores = made(torch, vocab, items * beams, vocab, f32)
    low = torch.finfo(logits.dtype).min
    logits[0, vocab // 2:] = float("-inf")
    logits[1] = float("-inf")                    # no token may follow
    logits[2, 1:] = float("-inf")                # one may
    logits[4, 1:] = low                          # masked by the lowest value: far below, but there
    logits[5] = low                              # all alike
    scores[8:11] = float("-inf")
    ended = [0] * 12 + [1, 0, 1, 0] + [1] * 4 + [0, 0, 1, 0]
    scores[22] = float("-inf")                   # ended, and there is no such beam
    logits[12] = float("nan")                    # an ended beam's logits are not looked at
    for n_out in (1, 4, 8, 32):
        _, want = check(torch, L, logits, scores, beams, n_out, ended, eos=min(2, vocab - 1))
        assert not want[4]
    assert (want[1][4] >= 0).sum() == 4          # nothing but ended beams: one continuation each


@pytest.mark.parametrize("f32", [False, True])
def test_what_is_not_finite(torch, L, f32):
    for vocab in (3, 3000, 30000):
        logits, scores = made(torch, vocab, 24, vocab, f32)
        logits[1, vocab - 1] = float("nan")
        logits[2, 0] = float("inf")
        logits[4, vocab // 2] = float("inf")
        logits[4, 1] = float("nan")
        logits[5] = float("nan")
        logits[6] = float("inf")
        scores[8], scores[9] = float("nan"), float("inf")
        _, want = check(torch, L, logits, scores, 4, 6)
        assert want[4]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab", [300, 2048, 20000, 100003])
@pytest.mark.parametrize("items", [1, 150])
def test_orders_that_leave_many_candidates(torch, L, vocab, items, f32):
    """Equal logits, rising and falling ones, large ones side by side or a piece apart: ties go to the lower token."""
    if items * 3 * vocab > 10_000_000:
        items = 30
    t = torch.arange(vocab, device="cuda")
    ramp = t / vocab * 8
    piece = (t // 64 % 3 == 1) * 5.0
    for x in (torch.zeros(vocab, device="cuda"), ramp, ramp.flip(0), ramp.half().float(), piece, (t >= vocab - 100) * 3.0, (t % 2048 < 30) * 4.0 + ramp * 0.01,
              torch.where(t % 7 == 0, 1.0, float("-inf")), (t // 8 % 2) * 1.0):
        logits = x.repeat(3 * items, 1).to(torch.float32 if f32 else torch.float16).contiguous()
        logits[1::3] += 0.25
        scores = torch.zeros(3 * items, device="cuda")
        scores[2::3] = -0.125
        for n_out in (3, 32):
            check(torch, L, logits, scores, 3, n_out)


@pytest.mark.parametrize("f32", [False, True])
def test_zeros_of_either_sign_and_the_smallest_numbers(torch, L, f32):
    """-0 and 0 are equal; denormal numbers are not."""
    dtype = torch.float32 if f32 else torch.float16
    for vocab in (9, 3000, 40000):
        t = torch.arange(vocab, device="cuda")
        tiny = torch.finfo(dtype).smallest_normal / 4
        for x in (torch.where(t % 2 == 0, -0.0, 0.0), torch.where(t % 3 == 1, 0.0, -0.0), torch.where(t % 5 == 4, tiny, -0.0), (t % 7 - 6) * tiny):
            logits = x.to(dtype).repeat(4, 1)
            check(torch, L, logits, torch.tensor([-1.0, -1.0, -2.0, -0.5], device="cuda"), 2, 5)


def test_beams_that_are_alike(torch, L):
    """Equal rows with equal scores: the lower beam first.  As many candidates as there are, all of one score."""
    for beams, vocab, n_out in ((4, 5000, 8), (32, 600, 32), (32, 40000, 32), (2, 9, 20)):
        logits, _ = made(torch, beams, 1, vocab, False)
        for rows in (logits, torch.zeros_like(logits)):
            check(torch, L, rows.repeat(2 * beams, 1), torch.full((2 * beams,), -3.0, device="cuda"), beams, n_out)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab", [50, 3000, 50257])
def test_scores_that_32_bits_cannot_tell_apart(torch, L, vocab, f32):
    """The beams' logits are alike but for tokens that weigh next to nothing, and their scores a few units of fp32's last place apart: which
    is the larger is known in 64 bits only."""
    beams, items = 4, 40
    base, _ = made(torch, vocab, items, vocab, f32)
    logits = base.repeat_interleave(beams, 0).contiguous()
    top = logits.amax(1)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for b in range(items * beams):
        # some tokens e^-9 .. e^-16 of the largest: the sums differ by about 1e-6
        some = torch.randint(0, vocab, (3,), device="cuda", generator=g)
        logits[b, some] = (top[b] - 9 - 7 * torch.rand(3, device="cuda", generator=g)).to(logits.dtype)
    step = 2.0 ** -23
    scores = -1.0 - step * torch.randint(0, 20, (items * beams,), device="cuda", generator=g).float()
    check(torch, L, logits, scores, beams, 4)
    check(torch, L, logits, scores, beams, 11)


def test_rows_of_wider_ones(torch, L):
    for dtype in (torch.float16, torch.float32):
        for vocab, width, first in ((1000, 1001, 1), (5000, 5011, 3), (50257, 50304, 0)):
            wide = torch.full((12, width), float("nan"), dtype=dtype, device="cuda")  # what is beside the rows counts for nothing
            logits, scores = made(torch, vocab, 12, vocab, dtype == torch.float32)
            wide[:, first:first + vocab] = logits
            got = L.beam_select(wide[:, first:first + vocab], scores, 4, 6)
            agree(got, select(logits.cpu().numpy(), scores.cpu().numpy(), 4, 6))


def test_in_place_and_without_what_may_be_left_out(torch, L):
    logits, scores = made(torch, 9, 40, 3000, False)
    ended = torch.zeros(40, dtype=torch.int32, device="cuda")
    ended[5::7] = 1
    want = select(logits.cpu().numpy(), scores.cpu().numpy(), 4, 4, ended.tolist(), 17)
    parent, token = (torch.empty((10, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    got = L.beam_select(logits, scores, 4, ended=ended, eos=17, out=(scores, parent, token, ended))
    agree([t.view(10, 4) for t in got], want)
    logits, scores = made(torch, 10, 40, 3000, False)
    out = [torch.full((10, 2), -5.0, device="cuda"), *(torch.full((10, 2), -5, dtype=torch.int32, device="cuda") for _ in range(2)), None]
    L.beam_select(logits, scores, 4, 2, out=out)
    want = select(logits.cpu().numpy(), scores.cpu().numpy(), 4, 2)
    agree(out[:3] + [torch.from_numpy(want[3])], want)


def test_ends_without_ended_beams(torch, L):
    logits, scores = made(torch, 4, 8, 500, True)
    logits[:, 7] += 12.0
    got, want = check(torch, L, logits, scores, 4, 4, eos=7)
    assert want[3].sum() >= 2


def test_more_than_2_31_logits(torch, L):
    vocab, rows = 2 ** 21 + 1, 1040  # 4.4 GB of fp16
    logits = torch.zeros((rows, vocab), dtype=torch.float16, device="cuda")
    logits[rows - 1, vocab - 1], logits[rows - 1, vocab - 5], logits[rows - 3, 3] = 20.0, 19.0, 18.0
    scores = torch.zeros(rows, device="cuda")
    s, parent, token, _ = L.beam_select(logits, scores, 4, 3)
    # 18 - log(2^21 + e^18) = -0.03; 20 - log(2^21 + e^20 + e^19) = -0.32, and one less
    assert parent[-1].tolist() == [rows - 3, rows - 1, rows - 1] and token[-1].tolist() == [3, vocab - 1, vocab - 5]
    lse = [np.log(vocab - 2 + np.exp(20.0) + np.exp(19.0)), np.log(vocab - 1 + np.exp(18.0))]
    want = np.array([18.0 - lse[1], 20.0 - lse[0], 19.0 - lse[0]])
    assert (np.abs(s[-1].double().cpu().numpy() - want) <= LSE_ERROR + 2.0 ** -24 * np.abs(want)).all()
    assert parent[0].tolist() == [0, 0, 0] and token[0].tolist() == [0, 1, 2]


def test_the_largest_vocabulary(torch, L):
    vocab = 2 ** 27  # LLMINT8_BEAM_MAX_VOCAB
    logits = torch.zeros((2, vocab), dtype=torch.float16, device="cuda")
    logits[1, vocab - 1], logits[0, vocab - 2] = 25.0, 24.0
    s, parent, token, _ = L.beam_select(logits, torch.zeros(2, device="cuda"), 2, 3)
    assert parent.tolist() == [[1, 0, 0]] and token.tolist() == [[vocab - 1, vocab - 2, 0]]
    lse = [np.log(vocab - 1 + np.exp(24.0)), np.log(vocab - 1 + np.exp(25.0))]
    want = np.array([25.0 - lse[1], 24.0 - lse[0], -lse[0]])
    assert (np.abs(s[0].double().cpu().numpy() - want) <= LSE_ERROR + 2.0 ** -24 * np.abs(want)).all()


def test_streams_and_replays(torch, L):
    """Two captured calls that share a workspace, replayed in turn with eager work between."""
    calls = []
    ws = L.beam_select_workspace(20, 4, 50257, 8)
    side = torch.cuda.Stream()
    for seed in range(2):
        logits, scores = made(torch, seed, 80, 50257, False)
        out = (torch.zeros((20, 8), device="cuda"), *(torch.zeros((20, 8), dtype=torch.int32, device="cuda") for _ in range(3)))
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            L.beam_select(logits, scores, 4, 8, ws=ws, out=out)
        calls.append((logits, scores, out, graph))
    for turn in range(4):
        for k, (logits, scores, out, graph) in enumerate(calls):
            new, s = made(torch, 100 + 10 * turn + k, 80, 50257, False)
            logits.copy_(new), scores.copy_(s)
            graph.replay()
            agree(out, select(new.cpu().numpy(), s.cpu().numpy(), 4, 8))
        with torch.cuda.stream(side):
            got = L.beam_select(calls[0][0], calls[0][1], 4, 8)
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, calls[0][2]))


def test_refusals(torch, L):
    logits, scores = made(torch, 0, 8, 100, False)
    with pytest.raises(L.Llmint8Error):
        L.beam_select(logits, scores, 4, 33)
    with pytest.raises(L.Llmint8Error):
        L.beam_select(logits, scores, 4, 4, ws=L.Workspace(torch.empty(64, dtype=torch.uint8, device="cuda")))
    with pytest.raises(L.Llmint8Error):
        L.beam_select(logits, scores, 4, 4, ended=torch.zeros(8, dtype=torch.int32, device="cuda"))
    for bad in (dict(logits=logits.double()), dict(logits=logits.t()), dict(scores=scores[:7]), dict(scores=scores.double()),
                dict(ended=torch.zeros(8, dtype=torch.int64, device="cuda"), eos=1), dict(beams=3)):
        with pytest.raises(AssertionError):
            L.beam_select(**{**dict(logits=logits, scores=scores, beams=4), **bad})
