"""Attention where a page does not exist: its positions are left out, whatever the cache's unwritten constants hold."""
import numpy as np
import pytest

from kv_util import Device, attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("garbage", [np.inf, -np.inf, np.nan, 65504.0])
@pytest.mark.parametrize("heads, new, length, missing", [(1, 1, 160, 1), (1, 40, 160, 0), (2, 3, 4200, 70), (16, 1500, 1500, 0),
                                                         (16, 1500, 1500, 33)])
def test_constants_of_unwritten_pages_do_not_count(heads, new, length, missing, garbage, causal):
    """One row, some, and as many as are a prompt's; page 0 of the cache, which no sequence has, holds garbage."""
    rng = np.random.default_rng(length + missing)
    dev = Device(1, heads, 32, page=32, most=length, seed=1)
    dev.pages_np = np.arange(1, dev.pages_np.shape[1] + 1, dtype=np.int32)[None]
    dev.pages = dev.dev(dev.pages_np)
    dev.cache.consts.fill_(garbage)
    dev.append([length], rng)
    pages = dev.pages_np.copy()
    pages[0, missing] = dev.cache.codes.shape[0]
    q = rng.standard_normal((new, heads, 32)).astype(np.float16)
    got = dev.L.kv_attention(dev.cache, dev.batch((new,), (length,), pages=dev.dev(pages)), dev.dev(q), causal=causal)
    assert int(dev.status) == dev.L.KV_BAD_PAGE
    gone = np.arange(32 * missing, 32 * missing + 32)
    pos = np.arange(length - new, length)
    want, tol = attention(q, np.delete(dev.seq[0].held(), gone, 2), pos - (gone <= pos[:, None]).sum(1), 32 ** -0.5, causal)
    assert (np.abs(got.cpu().numpy() - want) <= tol).all()
