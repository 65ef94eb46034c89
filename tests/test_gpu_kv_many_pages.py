"""kv_reserve where a call gives out, or looks at, thousands of pages: more than it lists at once (2 048), in several rounds (of 2 048 pages
behind the sequences' first ones)."""
import random

import pytest

from kv_pages_util import NO_PAGE
from test_gpu_kv_served import Served

pytestmark = pytest.mark.gpu


def idle(torch, L, n, stride, n_pages, page):
    return Served(torch, L, [[-1] * stride] * n, [0] * n_pages, [0] * n, list(range(n)), page)


@pytest.mark.parametrize("n, each, page, seed", [(40, 100, 32, 0), (7, 900, 64, 1), (300, 23, 96, 2), (2048, 4, 32, 3), (1, 5000, 32, 4), (33, 63, 32, 5),
                                                 (20, 1024, 32, 6)])
def test_prompts(n, each, page, seed):
    import torch

    import paper_2208_07339_amd as L
    r = random.Random(seed)
    stride = each + 3
    s = idle(torch, L, n, stride, 2 * n * stride + 9, page)
    # prompts of about so many pages, some of them none
    rows = [r.randint((each - 1) * page - 40, each * page) if n < 3 or r.random() < 0.95 else 0 for _ in range(n)]
    s.set_len(rows)
    s.reserve(rows)
    s.check()
    # written anew, by those that hold their pages alone: all are looked at, none is given
    s.reserve([x - 1 if x else 0 for x in rows])
    s.check()
    # half of them go on from others, shortened, over pages that they share; the rest get a page or two more
    parent = [r.randrange(n) if r.random() < 0.5 else b for b in range(n)]
    s.fork(parent)
    s.check()
    lengths, rows = [], []
    for b, x in enumerate(s.book.kv_len):
        if parent[b] != b or n == 1:
            old = r.randint(0, x) // 4
            y = r.randint(0, max(0, x - old) + 2 * page)
        else:
            old, y = x, r.randint(0, 2 * page)
        lengths.append(min(old + y, stride * page)), rows.append(min(y, stride * page - old))
    s.set_len(lengths)
    s.reserve(rows)
    s.check()
    assert s.book.refs == s.book.counted() and not s.book.status


@pytest.mark.parametrize("n, each, page, seed", [(40, 100, 32, 0), (6, 1100, 64, 1), (700, 9, 32, 2)])
def test_too_few_pages(n, each, page, seed):
    """The pool runs out among sequences, in whatever round, also where shared pages are to be replaced."""
    import torch

    import paper_2208_07339_amd as L
    r = random.Random(seed)
    stride = each + 1
    for share in (0.0, 0.2, 0.51, 0.9):
        s = idle(torch, L, n, stride, each + 3 + int(share * n * each), page)
        s.set_len([each * page - 5] + [0] * (n - 1))
        s.reserve([each * page - 5] + [0] * (n - 1))
        s.check()
        s.fork([0 if r.random() < 0.5 else -1 for _ in range(n)])
        lengths, rows = [], []
        for x in s.book.kv_len:
            old = r.randint(0, x) // 2
            y = r.randint(1, each * page - old)
            lengths.append(old + y), rows.append(y)
        s.set_len(lengths)
        s.reserve(rows)
        s.check()
        assert s.book.refs == s.book.counted() and (s.book.status == NO_PAGE or share > 0.5 and s.book.status == 0)
