"""Attention where the work is cut up in other ways: windows over long axes, whose parts are fewer than the workspace is for, prompts
of several sizes over themselves and behind others, and a captured prompt of wide heads."""
import numpy as np
import pytest

from kv_util import Device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [1, 50, 1000, 4500])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_windows_over_long_axes(new, window):
    rng = np.random.default_rng(window + new)
    dev = Device(1, 2, 64, page=64, most=5000, seed=new)
    dev.append([4970], rng)
    dev.check_attention([new], rng, group=4, window=window)
    dev.check_attention([new], rng, group=4)


@pytest.mark.parametrize("heads, new, past", [(8, 1100, 0), (1, 1100, 0), (4, 700, 1500), (1, 130, 4200)])
def test_prompts(heads, new, past):
    rng = np.random.default_rng(new)
    dev = Device(1, heads, 32, page=128, most=new + past, seed=3)
    if past:
        dev.append([past], rng)
    dev.append([new], rng)
    dev.check_attention([new], rng)
    dev.check_attention([new], rng, window=333)


def test_captured_prompt_of_wide_heads():
    import torch

    rng = np.random.default_rng(5)
    dev = Device(2, 2, 128, page=64, most=800, seed=5)
    dev.append([790, 300], rng)
    dev.check_attention([700, 290], rng, group=8)  # (outside first: modules are loaded)
    q = dev.dev(rng.standard_normal((990, 16, 128)).astype(np.float16))
    batch = dev.batch([700, 290], dev.lengths())
    ws, out = dev.L.kv_attention_workspace(dev.cache, batch, 16), torch.empty_like(q)
    want = dev.L.kv_attention(dev.cache, batch, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dev.L.kv_attention(dev.cache, batch, q, ws=ws, out=out)
    for i in range(3):
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("d", [32, 40, 64, 96, 128])
@pytest.mark.parametrize("new, past, heads", [(1500, 0, 16), (1535, 0, 16), (1536, 0, 16), (900, 700, 24)])
def test_tiles_of_two_halves(d, new, past, heads):
    """Rows whose tiles' blocks two halves of a workgroup share: numbers of blocks of all remainders, windows, everything seen."""
    rng = np.random.default_rng(d)
    dev = Device(1, heads, d, page=128, most=new + past, seed=d)
    if past:
        dev.append([past], rng)
    dev.append([new], rng)
    dev.check_attention([new], rng)
    if d == 64:
        dev.check_attention([new], rng, window=700)
        dev.check_attention([new], rng, causal=False)
        dev.check_attention([new], rng, lengths=[new + past - 32])


def test_two_halves_and_ragged_sequences():
    rng = np.random.default_rng(8)
    dev = Device(4, 16, 64, page=64, most=1600, seed=8)
    dev.append([1500, 90, 33, 7], rng)
    dev.check_attention([1400, 90, 20, 7], rng)
    dev.check_attention([1400, 90, 20, 7], rng, idle=(1,))
