"""Beam search over the 8-bit key/value cache, at the sizes a serving program has: what work on its speed is measured on.

beam_select picks, for each item of a batch, the best continuations of its beams from their logits.  kv_fork makes every
sequence one that goes on from a parent (a beam from another, a sample from a prompt; without a parent it ends), kv_reserve
gives sequences the pages that their next tokens need, pages of their own where they would write what others hold, kv_compact
moves the pages in use to the front of the pool, and kv_copy moves a layer's data as these three say.

Pages, as users of the cache see them: refs[p] is the number of table entries that name page p, entries below 0 name none, the
lowest free pages are given first.  Blocks of 32 positions of a page are full or not held there; the positions behind the last
full block, and the 32 before them, are in a ring of 64 positions (position p of a sequence at place p % 64 of its slot).
"""
import random

import torch

own = False

BLOCK, RING = 32, 64
MAX_LOGITS = 64 * 8 * 131072 * 2  # bytes of logits of the largest listed case
MAX_MOVED = 110e6                 # bytes that a case copies at most, about
MAX_CACHE = 2.2e9                 # bytes of codes of a case
MAX_TABLE = 256 * 1024            # entries of its tables

# key/value heads, width of a head
LAYOUTS = [(12, 64), (32, 80), (32, 128), (40, 128), (8, 128), (8, 128), (1, 128), (2, 256)]


def _select(name, items, beams, vocab, out, f32=False, first=False, ended=0):
    return {"name": name, "call": "select", "items": items, "beams": beams, "vocab": vocab, "out": out, "f32": f32,
            "first": first, "ended": ended}


def _reorder(name, layout, items, beams, live, lengths, close=False, page=64, layers=2):
    return {"name": name, "call": "reorder", "items": items, "beams": beams, "live": live, "len_lo": lengths[0], "len_hi": lengths[1],
            "close": close, "heads": layout[0], "d": layout[1], "page": page, "layers": layers}


def _turnover(name, layout, seqs, length, ends, compact, page=64, layers=1):
    return {"name": name, "call": "turnover", "seqs": seqs, "length": length, "ends": ends, "compact": compact, "heads": layout[0],
            "d": layout[1], "page": page, "layers": layers}


def listed():
    return [
        # one user's four beams: launches and dependent loads are all there is
        _select("select_one_user", 1, 4, 50257, 4),
        # a few users, logits that a program has worked on in fp32, twice the beams picked so that ended ones can be set aside
        _select("select_doubled", 3, 5, 32003, 10, f32=True, ended=20),
        # a serving batch in the middle of its answers, some beams at their end
        _select("select_batch", 64, 4, 50257, 8, ended=10),
        # the first step behind the prompts: one beam of each user lives, the others' logits count for nothing
        _select("select_first", 48, 8, 65024, 8, first=True),
        # the largest batch and vocabulary
        _select("select_large", 64, 8, 131072, 8),
        # one user's beams after a step: two of four go on, twice
        _reorder("reorder_one_user", (40, 128), 1, 4, 2, (1000, 1000)),
        # a serving batch after a step
        _reorder("reorder_batch", (8, 128), 32, 4, 2, (200, 4100)),
        # the same when a block of 32 tokens gets full, so that beams that shared its page need pages of their own
        _reorder("reorder_close", (32, 80), 32, 4, 2, (200, 4100), close=True, page=96),
        # eight samples from each of sixteen prompts
        _reorder("reorder_samples", (40, 128), 16, 8, 1, (500, 3000), layers=1),
        # beams over documents of 100 000 tokens: long tables
        _reorder("reorder_long", (8, 128), 2, 8, 3, (100003, 131071), close=True, layers=4),
        # twenty of two hundred sequences end and as many prompts come
        _turnover("admit", (8, 128), 200, 1500, 20, False, page=32),
        # the oldest sequences end, the pool is kept without gaps, others come
        _turnover("compact", (40, 128), 48, 2100, 3, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    call = rng.choice(["select", "select", "reorder", "reorder", "turnover"])
    while True:
        if call == "select":
            beams, out = rng.choice([1, 2, 3, 4, 4, 5, 8, 10, 16]), rng.choice([1, 2, 4, 8, 16])
            c = _select("", _log_int(rng, 1, 256), beams, _log_int(rng, 1000, 160000), rng.choice([beams, beams, 2 * beams, out]),
                        rng.random() < 0.3, rng.random() < 0.15, rng.choice([0, 0, 10, 40]))
            if c["items"] * beams * c["vocab"] * (4 if c["f32"] else 2) > MAX_LOGITS:
                continue
        else:
            layout = rng.choice(LAYOUTS)
            page, layers = rng.choice([32, 64, 64, 96, 128, 256]), rng.choice([1, 1, 2, 4])
            if call == "reorder":
                beams, hi = rng.choice([2, 3, 4, 4, 5, 8, 16]), _log_int(rng, 20, 131072)
                c = _reorder("", layout, _log_int(rng, 1, 128), beams, rng.randint(1, beams), (max(1, hi // rng.choice([1, 2, 10])), hi),
                             rng.random() < 0.5, page, layers)
            else:
                seqs = _log_int(rng, 2, 512)
                c = _turnover("", layout, seqs, _log_int(rng, 20, 32768), rng.randint(1, max(1, seqs // 4)), rng.random() < 0.6, page, layers)
            s = _sizes(c)
            if s["codes"] * layers > MAX_CACHE or s["seqs"] * s["stride"] > MAX_TABLE or s["seqs"] > 1024 or s["moved"] > MAX_MOVED:
                continue
        del c["name"]
        return c


def _padded(d):
    return -(-d // 32) * 32


def _lengths(case):
    """reorder: an item's tokens, the one that comes next included, and the parents of its beams: by the case alone.  A beam that
    goes on is its own parent, the others go on from one of those."""
    r = random.Random("%(items)d %(beams)d %(live)d %(len_lo)d %(len_hi)d" % case)
    length, parent, beams = [], [], case["beams"]
    for i in range(case["items"]):
        n = r.randint(case["len_lo"], case["len_hi"])
        length.append(-(-n // BLOCK) * BLOCK if case["close"] else n + (n % BLOCK == 0))
        alive = r.sample(range(beams), case["live"])
        parent += [i * beams + (b if b in alive else r.choice(alive)) for b in range(beams)]
    return length, parent


def _sizes(case):
    """Numbers that follow from the case: sequences, width of the tables, pages, bytes of a layer's codes, and bytes that a pass
    copies (reads and writes) in all layers."""
    page, h, d = case["page"], case["heads"], case["d"]
    per = page // BLOCK
    block = h * (2 * BLOCK * _padded(d) + 4)
    moved = 0
    if case["call"] == "reorder":
        length, parent = _lengths(case)
        seqs, beams = len(parent), case["beams"]
        most = -(-max(length) // page)
        copies = sum(p != b for b, p in enumerate(parent))
        # an item's beams share all pages but the last two
        used = sum(max(0, -(-n // page) - 2) + beams * min(2, -(-n // page)) for n in length)
        n_pages = used + copies + 7
        for b, p in enumerate(parent):
            n = length[b // beams]
            if p != b:
                rows = n - max(0, n // BLOCK - 1) * BLOCK
                kept = (n // BLOCK - 1) % per if case["close"] else 0
                moved += 2 * (rows * h * d * 4 + kept * block)
    else:
        seqs, most = case["seqs"], -(-case["length"] // page)
        n_pages = seqs * most + 5
        if case["compact"]:
            moved = 2 * per * block * most * min(case["ends"], seqs - case["ends"])
    return {"seqs": seqs, "stride": most + most // 4 + 1, "pages": n_pages, "codes": n_pages * per * block,
            "moved": moved * case["layers"]}


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return _prepare_select(case, g) if case["call"] == "select" else _prepare_cache(case, g)


def _prepare_select(case, g):
    items, beams, vocab, out = case["items"], case["beams"], case["vocab"], case["out"]
    # what a vocabulary's logits look like: most far below a few, alike in the beams of an item
    x = torch.empty((items, beams, vocab), device="cuda").normal_(generator=g).mul_(1.2)
    x += torch.empty((items, 1, vocab), device="cuda").normal_(generator=g).mul_(2.0)
    x += torch.empty((1, 1, vocab), device="cuda").normal_(generator=g)
    x = x.view(items * beams, vocab)
    x.masked_fill_(torch.rand(vocab, device="cuda", generator=g) < 0.01, float("-inf"))  # tokens that may not come
    logits = x if case["f32"] else x.half()
    scores = -20.0 + 1.5 * torch.randn(items * beams, device="cuda", generator=g)
    if case["first"]:
        scores.view(items, beams)[:, 1:] = float("-inf")
    ended = (torch.rand(items * beams, device="cuda", generator=g) * 100 < case["ended"]).int()
    ended.view(items, beams)[:, 0] = 0  # (an item with nothing but ended beams is done)
    s = {"case": case, "logits": logits, "scores": scores, "ended": ended, "eos": 2}
    if own:
        import paper_2208_07339_amd as L
        s["ws"] = L.beam_select_workspace(items, beams, vocab, out)
        s["out"] = (torch.zeros((items, out), device="cuda"), *(torch.zeros((items, out), dtype=torch.int32, device="cuda") for _ in range(3)))
    return s


def _prepare_cache(case, g):
    z = _sizes(case)
    seqs, stride, n_pages, page = z["seqs"], z["stride"], z["pages"], case["page"]
    h, d, per, layers = case["heads"], case["d"], page // BLOCK, case["layers"]
    reorder = case["call"] == "reorder"
    pages = torch.full((seqs, stride), -1, dtype=torch.int32, device="cuda")
    if reorder:
        length, parent = _lengths(case)
        beams = case["beams"]
        order = torch.randperm(n_pages, device="cuda", generator=g).int()
        at = 0
        for i, n in enumerate(length):
            most = -(-n // page)
            both, each = max(0, most - 2), min(2, most)
            rows = pages[i * beams:(i + 1) * beams]
            rows[:, :both] = order[at:at + both]
            at += both
            rows[:, both:most] = order[at:at + beams * each].view(beams, each)
            at += beams * each
        kv_len = _ints([n for n in length for _ in range(beams)])
        row_start = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    else:
        n, ends, most = case["length"], case["ends"], -(-case["length"] // page)
        # the pages in use are the first ones, in whatever order
        pages[:, :most] = torch.randperm(seqs * most, device="cuda", generator=g).int().view(seqs, most)
        parent = list(range(ends, seqs)) + [-1] * ends
        kv_len = _ints([n] * seqs)
        row_start = _ints([0] * (seqs - ends) + [n * i for i in range(ends + 1)])  # the new ones' prompts
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs.index_add_(0, pages.clamp(min=0).flatten().long(), (pages >= 0).int().flatten())
    s = {"case": case, "pages": pages, "kv_len": kv_len, "refs": refs, "row_start": row_start, "parent": _ints(parent),
         "slots": torch.randperm(seqs, device="cuda", generator=g).int(), "layers": []}
    for _ in range(layers):
        codes = torch.randint(-127, 128, (n_pages, h, per, 2, BLOCK * _padded(d)), dtype=torch.int8, device="cuda", generator=g)
        consts = torch.rand((n_pages, h, per, 2), device="cuda", generator=g).half()
        ring = torch.empty((seqs, h, 2, RING, d), dtype=torch.float16, device="cuda").normal_(generator=g)
        s["layers"].append((codes, consts, ring))
    if own:
        import paper_2208_07339_amd as L
        s["pool"] = L.KvPool(refs, page)
        s["seqs"] = L.KvSeqs(pages, kv_len, s["slots"])
        s["moves"] = L.KvMoves.allocate(max(seqs, n_pages), seqs)
        s["caches"] = [L.KvCache(*layer, page, d) for layer in s["layers"]]
    return s


def _held(state):
    """What a pass over the cache leaves: 16-bit values as their bits, which copies keep."""
    layers = [[codes, consts.view(torch.int16), ring.view(torch.int16)] for codes, consts, ring in state["layers"]]
    return {"pages": state["pages"], "refs": state["refs"], "kv_len": state["kv_len"], "slots": state["slots"], "layers": layers}


def run(state):
    case = state["case"]
    if not own:
        return {"select": _plain_select, "reorder": _plain_reorder, "turnover": _plain_turnover}[case["call"]](state)
    import paper_2208_07339_amd as L
    if case["call"] == "select":
        scores, parent, token, ended = state["out"]
        L.beam_select(state["logits"], state["scores"], case["beams"], case["out"], ended=state["ended"], eos=state["eos"],
                      ws=state["ws"], out=state["out"])
        return {"scores": scores, "parent": parent, "token": token, "ended": ended}
    pool, seqs, moves = state["pool"], state["seqs"], state["moves"]
    L.kv_fork(pool, seqs, state["parent"], moves)
    if case["call"] == "turnover":
        if case["compact"]:
            L.kv_compact(pool, seqs, moves)
            for cache in state["caches"]:
                L.kv_copy(cache, moves)
        state["kv_len"][case["seqs"] - case["ends"]:] = case["length"]
        L.kv_reserve(pool, seqs, state["row_start"], moves)
    else:
        L.kv_reserve(pool, seqs, state["row_start"], moves, more=True)
        for cache in state["caches"]:
            L.kv_copy(cache, moves)
    return _held(state)


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _plain_select(state):
    case, eos = state["case"], state["eos"]
    items, beams, vocab, n = case["items"], case["beams"], case["vocab"], case["out"]
    x = state["logits"].double()  # in 64 bits: which of two scores is the larger hangs on their last bits
    cum = state["scores"].double()[:, None]
    top = x.amax(1, keepdim=True)
    x = x - top
    x = cum + (x - x.exp().sum(1, keepdim=True).log())
    done = state["ended"][:, None] > 0
    x.masked_fill_(done, float("-inf"))
    x[:, eos] = torch.where(done, cum, x[:, eos:eos + 1])[:, 0]
    x = x.view(items, beams * vocab)
    place = torch.arange(beams * vocab, device="cuda")
    best, at = [], []
    for _ in range(n):
        m = x.amax(1, keepdim=True)
        i = torch.where(x == m, place, beams * vocab).amin(1, keepdim=True)
        x.scatter_(1, i, float("-inf"))
        best.append(m)
        at.append(i)
    best, at = torch.cat(best, 1), torch.cat(at, 1)
    parent = torch.arange(items, device="cuda")[:, None] * beams + at // vocab
    token = at % vocab
    ended = (state["ended"][parent] > 0) | (token == eos)
    return {"scores": best.float(), "parent": parent.int(), "token": token.int(), "ended": ended.int()}


def _rank(flags):
    """How many are set before each place."""
    return flags.long().cumsum(0) - flags.long()


def _listed_where(flags, values):
    """The values where flags are set, in front, in order."""
    n = len(flags)
    out = torch.zeros(n + 1, dtype=torch.long, device="cuda")
    out[torch.where(flags, _rank(flags), n)] = values
    return out[:n]


def _plain_fork(state):
    """-> source and destination slots and the length of sequences whose ring is copied; slots behind the last stand for themselves."""
    n = len(state["parent"])
    me = torch.arange(n, device="cuda")
    parent, length = state["parent"].long(), state["kv_len"].long()
    alive, src = parent >= 0, parent.clamp(min=0)
    children = torch.zeros(n, dtype=torch.long, device="cuda").index_add_(0, src, alive.long())
    pages = state["pages"].long()
    state["refs"].index_add_(0, pages.clamp(min=0).flatten(), torch.where(pages >= 0, children[:, None] - 1, 0).int().flatten())
    state["pages"].copy_(torch.where(alive[:, None], pages[src], -1))
    first = torch.full((n,), n, device="cuda").scatter_reduce_(0, src, torch.where(alive, me, n), "amin")
    heir = alive & (first[src] == me)
    slots = state["slots"].long()
    spare = _listed_where(children == 0, slots)
    extra = alive & ~heir
    turn = torch.where(extra, _rank(extra), extra.sum() + _rank(~alive))
    new = torch.where(heir, slots[src], spare[turn.clamp(max=n - 1)])
    state["slots"].copy_(new)
    state["kv_len"].copy_(torch.where(alive, length[src], 0))
    to = _listed_where(extra, new)
    nothing = me >= extra.sum()
    return torch.where(nothing, new, _listed_where(extra, slots[src])), torch.where(nothing, new, to), torch.where(nothing, 0, _listed_where(extra, length[src]))


def _given(free, need):
    """The lowest free pages to the places that need one, in order."""
    pages = _listed_where(free, torch.arange(len(free), device="cuda"))
    return pages[_rank(need).clamp(max=len(free) - 1)]


def _plain_reserve(state):
    """-> pages to copy: source, destination and blocks of each sequence (source = destination where there is nothing to copy)."""
    page = state["case"]["page"]
    per = page // BLOCK
    pages, refs, length = state["pages"].long(), state["refs"], state["kv_len"].long()
    old = length - state["row_start"].long().diff()
    n, stride = pages.shape
    b, j = torch.arange(n, device="cuda"), torch.arange(stride, device="cuda")
    first = (old // page)[:, None]
    due = (j >= first) & (j < (-(-length // page))[:, None]) & (old < length)[:, None]
    missing = due & (pages < 0)
    closing = torch.maximum(j * per, (old // BLOCK)[:, None]) < torch.minimum((j + 1) * per, (length // BLOCK)[:, None])
    shared = due & ~missing & closing & (refs[pages.clamp(min=0)] > 1)
    here = shared & (j == first)
    at = torch.where(here, pages, len(refs)).flatten()  # (a page behind the last stands for none)
    want = torch.zeros(len(refs) + 1, dtype=torch.long, device="cuda").index_add_(0, at, torch.ones_like(at))
    who = b[:, None].expand(n, stride)
    last = torch.full((len(refs) + 1,), -1, device="cuda").scatter_reduce_(0, at, who.flatten(), "amax")
    at = at.view(n, stride)
    keeps = here & (want[at] >= torch.nn.functional.pad(refs, (0, 1))[at]) & (last[at] == who)
    shared &= ~keeps
    need = missing | shared
    new = torch.where(need, _given(refs == 0, need.flatten()).view(n, stride), pages)
    refs.index_add_(0, pages.clamp(min=0).flatten(), -shared.flatten().int())
    refs.index_add_(0, new.clamp(min=0).flatten(), need.flatten().int())
    state["pages"].copy_(new)
    f = first.clamp(max=stride - 1)
    to = new.gather(1, f)[:, 0].clamp(min=0)
    copied = (here & shared).any(1)
    return torch.where(copied, pages.gather(1, f)[:, 0], to), to, torch.where(copied, old // BLOCK - first[:, 0] * per, 0)


def _plain_rings(state, src, dst, length):
    place = torch.arange(RING, device="cuda")
    lo = ((length // BLOCK - 1) * BLOCK).clamp(min=0)[:, None]
    position = lo + (place - lo) % RING  # of each place of the ring
    held = (position < length[:, None])[:, None, None, :, None]
    for _, _, ring in state["layers"]:
        ring[dst] = torch.where(held, ring[src], ring[dst])


def _plain_reorder(state):
    case = state["case"]
    copies = sum(p != b for b, p in enumerate(_lengths(case)[1]))
    src, dst, length = _plain_fork(state)
    _plain_rings(state, src[:copies], dst[:copies], length[:copies])
    src, dst, blocks = _plain_reserve(state)
    if case["close"] and case["page"] > BLOCK:
        at = torch.argsort((src == dst).int(), stable=True)[:copies]  # the sequences that copy, then others
        src, dst, keep = src[at], dst[at], (torch.arange(case["page"] // BLOCK, device="cuda") < blocks[at, None])
        for codes, consts, _ in state["layers"]:
            codes[dst] = torch.where(keep[:, None, :, None, None], codes[src], codes[dst])
            consts[dst] = torch.where(keep[:, None, :, None], consts[src], consts[dst])
    return _held(state)


def _plain_compact(state, most):
    """-> pages to move, `most`: source and destination; the first again behind the last."""
    refs = state["refs"]
    p, used = torch.arange(len(refs), device="cuda"), refs > 0
    n = used.sum()
    moved, gaps = used & (p >= n), ~used & (p < n)
    to = torch.where(moved, _given(gaps, moved), p)
    new = torch.zeros_like(refs).index_add_(0, to, refs)
    refs.copy_(new)
    pages = state["pages"].long()
    state["pages"].copy_(torch.where(pages >= 0, to[pages.clamp(min=0)], -1))
    k = torch.arange(most, device="cuda")
    src = _listed_where(moved, p)[torch.where(k < moved.sum(), k, 0)]
    return src, to[src]


def _plain_turnover(state):
    case = state["case"]
    _plain_fork(state)
    if case["compact"]:
        page = -(-case["length"] // case["page"])
        src, dst = _plain_compact(state, page * min(case["ends"], case["seqs"] - case["ends"]))
        for codes, consts, _ in state["layers"]:
            codes[dst], consts[dst] = codes[src], consts[src]
    state["kv_len"][case["seqs"] - case["ends"]:] = case["length"]
    _plain_reserve(state)
    return _held(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    if case["call"] == "select":
        rows = case["items"] * (1 if case["first"] else case["beams"] - case["ended"] / 100 * (case["beams"] - 1))
        n = rows * case["vocab"]
        return {"bytes": n * (4 if case["f32"] else 2) + 16 * case["items"] * case["out"] + 8 * case["items"] * case["beams"], "flops": 4 * n}
    z = _sizes(case)
    tables = 8 * z["seqs"] * z["stride"] + 8 * z["pages"] + 32 * z["seqs"]  # tables and counts read and written once
    return {"bytes": tables + z["moved"], "flops": 0}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["call"] != "select":
        return None  # nothing but whole numbers and copies
    s = prepare(case, seed)
    best = []
    for item in range(case["items"]):
        found = []
        for b in range(item * case["beams"], (item + 1) * case["beams"]):
            if s["ended"][b]:
                found.append(s["scores"][b:b + 1].double())
            else:
                x = s["logits"][b].double()
                x = torch.topk(x, min(case["out"], case["vocab"])).values - torch.logsumexp(x, 0)
                found.append(s["scores"][b].double() + x)
        best.append(torch.sort(torch.cat(found), descending=True).values[:case["out"]])
    return {"scores": torch.stack(best), "parent": None, "token": None, "ended": None}
