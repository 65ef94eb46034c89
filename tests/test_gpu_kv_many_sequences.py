"""More sequences than a wave looks at together, of which one cannot be and has no rows: it is told of all the same."""
import numpy as np
import pytest

from kv_util import Device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["length", "slot", "rows"])
@pytest.mark.parametrize("seqs, new", [(65, 129), (129, 129), (65, 1)])
def test_a_sequence_without_rows_that_cannot_be(seqs, new, what):
    rng = np.random.default_rng(seqs)
    n = [new] * (seqs - 1) + [0]
    dev = Device(seqs, 16, 32, page=32, most=160, seed=seqs)
    dev.append(n, rng)
    assert int(dev.status) == 0
    told, kw = dev.lengths(), {}
    q = rng.standard_normal((sum(n), 16, 32)).astype(np.float16)
    want = dev.check_attention(n, rng, q=q)
    if what == "length":
        told[-1] = -1
    elif what == "slot":
        kw["slots"] = dev.dev(np.array([*dev.slots_np[:-1], seqs + 2], np.int32))
    else:
        kw["row_start"] = dev.dev(np.cumsum([0, *n[:-1], 5]).astype(np.int32))
    batch = dev.batch(n, told, max_rows=new, max_len=160, **kw)
    assert dev.L.debug_kv_plan_for(dev.cache, batch, 16).tile == (128 if new > 1 else 32)
    kv = dev.dev(np.zeros((sum(n), 16, 32), np.float16))

    def attend():
        assert dev.torch.equal(dev.L.kv_attention(dev.cache, batch, dev.dev(q)), want)
    for call in (attend, lambda: dev.L.kv_read(dev.cache, batch), lambda: dev.L.kv_append(dev.cache, batch, kv, kv)):
        dev.status.zero_()
        call()
        assert int(dev.status) == dev.L.KV_BAD_BATCH
