"""Attention of batches in which one sequence has many rows and the others one: tiles that are there among many that are not."""
import numpy as np
import pytest

from kv_util import Device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads, group, new, lengths, window, tile", [
    (8, 1, [100] + [1] * 63, [300] * 64, 0, 32), (3, 2, [1] * 20 + [90, 1, 1, 47], [200] * 24, 0, 32), (8, 4, [1] * 30 + [64, 1], [500] * 32, 200, 32),
    (2, 1, [1, 300, 1, 1], [1500, 1300, 2, 1900], 0, 32), (1, 8, [70, 1, 0, 1, 2], [4000, 4100, 50, 1, 900], 0, 32),
    (8, 1, [1] * 100 + [2048] + [1] * 27, [130] * 100 + [2048] + [130] * 27, 128, 128)])
def test_one_prompt_among_single_rows(heads, group, new, lengths, window, tile):
    rng = np.random.default_rng(len(new))
    dev = Device(len(new), heads, 32, page=96, most=max(lengths), seed=len(new))
    dev.append(lengths, rng)
    assert dev.L.debug_kv_plan_for(dev.cache, dev.batch(new, lengths), heads * group, window).tile == tile
    dev.check_attention(new, rng, group=group, window=window)
    dev.check_attention(new, rng, group=group, window=window, idle=(0, len(new) - 1))
    assert int(dev.status) == 0


@pytest.mark.parametrize("heads, group, new, lengths", [
    (1, 48, [30], [400]), (1, 48, [7, 3, 5], [1000, 90, 2000]), (2, 8, [100], [3000]), (3, 1, [700], [900]), (9, 1, [200], [200]), (12, 1, [300, 40], [300, 250]),
    (17, 1, [90], [130])])
def test_few_parts(heads, group, new, lengths):
    """Numbers of heads and parts that are no multiple of eight, with many tiles."""
    rng = np.random.default_rng(heads)
    dev = Device(len(new), heads, 64, page=64, most=max(lengths), seed=heads)
    dev.append(lengths, rng)
    assert dev.L.debug_kv_plan_for(dev.cache, dev.batch(new, lengths), heads * group).tile == 32
    dev.check_attention(new, rng, group=group)
    dev.check_attention(new, rng, group=group, causal=False)
    dev.check_attention(new, rng, group=group, window=60)
    assert int(dev.status) == 0
