"""The 8-bit key/value cache and its attention, at the sizes a serving program has: what work on their speed is measured on.

Three operators: kv_append (position rotation of queries and keys, keys and values into the paged cache), kv_attention (over
that cache: rows of a prompt, or one row a sequence), and kv_read (the cached values as fp16), which a pass of kv_append runs
too, so that what came into the cache is seen.  Heads and widths are those of the GPT-3-family layers of the benchmark (width
4 096: 32 heads of 128; 5 120: 40; 12 288: 96; 2 560: 32 of 80; 768: 12 of 64), and layouts that share keys between heads.

The cache, as its users see it: pages of page tokens; blocks of 32 tokens and one head that are full hold codes of absmax
quantisation with one constant for keys and one for values; the tokens behind the last full block are fp16 in a ring of 64
positions (position p of a sequence at place p % 64).  Codes are tiles of 32 x 32 in the order of the matrix units, see
_tiles().
"""
import random

import torch

own = False

BLOCK, RING = 32, 64
MAX_SCORES = 8192 * 8192 * 40   # query heads x rows x tokens of the largest listed case
MAX_CACHE = 131072 * 8 * 128 * 2  # tokens x heads x width that a listed case holds at most

# query heads, key/value heads, width of a head
LAYOUTS = [(12, 12, 64), (32, 32, 80), (32, 32, 128), (40, 40, 128), (96, 96, 128), (32, 8, 128), (64, 8, 128), (40, 8, 128),
           (48, 1, 128), (16, 2, 256)]


def _attend(name, layout, seqs, new, past, window=0, page=64):
    hq, h, d = layout
    return {"name": name, "call": "attend", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "heads_q": hq, "heads": h, "d": d, "page": page, "window": window}


def _append(name, layout, seqs, new, past, rot, pairs=False, fused=True, page=64):
    hq, h, d = layout
    return {"name": name, "call": "append", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0],
            "past_hi": past[1], "heads_q": hq, "heads": h, "d": d, "page": page, "rot": rot, "pairs": pairs, "fused": fused}


def listed():
    return [
        # a small model answering one user, early in the answer: launches and host work are all there is
        _attend("step_small", (12, 12, 64), 1, (1, 1), (75, 75)),
        # the 13B layer generating for one user in the middle of a long conversation: one row, a long axis
        _attend("step_one_user", (40, 40, 128), 1, (1, 1), (4000, 4000)),
        # a serving batch, keys shared by four query heads, lengths as they come
        _attend("step_batch", (32, 8, 128), 64, (1, 1), (200, 4100)),
        # two users with documents of 100 000 tokens and more, keys shared by eight query heads
        _attend("step_long", (64, 8, 128), 2, (1, 1), (100003, 131071)),
        # a few drafted tokens checked at once, one key head for all 48 query heads: more rows than a tile has
        _attend("step_drafted", (48, 1, 128), 8, (3, 7), (1000, 9000)),
        # a prompt through the 6.7B layer: the benchmark's token count
        _attend("prompt", (32, 32, 128), 1, (2048, 2048), (0, 0)),
        # prompts of any length together, heads of 80, attention to the last 1 000 tokens only
        _attend("prompt_ragged_window", (32, 32, 80), 7, (33, 1900), (0, 700), window=1000, page=96),
        # the next piece of a long document behind 20 000 tokens that the cache holds
        _attend("prompt_piece", (32, 8, 128), 1, (1024, 1024), (20011, 20011), page=256),
        # a long prompt through the 13B layer: the largest call
        _attend("prompt_long", (40, 40, 128), 1, (8192, 8192), (0, 0)),
        # one token of each user of a serving batch into the cache, from the joint projection's output
        _append("append_step", (40, 40, 128), 96, (1, 1), (30, 3000), 128),
        # prompts of any length, heads of 80 of which 32 features are rotated in neighbouring pairs
        _append("append_ragged", (32, 32, 80), 5, (17, 1000), (0, 0), 32, pairs=True, fused=False, page=96),
        # a long prompt through the 13B layer
        _append("append_prompt", (40, 40, 128), 1, (8192, 8192), (0, 0), 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    call = rng.choice(["attend", "attend", "append"])
    while True:
        layout = hq, h, d = rng.choice(LAYOUTS)
        page = rng.choice([32, 64, 64, 96, 128, 256])
        step = rng.random() < 0.5
        if call == "append":
            seqs = _log_int(rng, 1, 128)
            hi = 1 if step else _log_int(rng, 2, 8192)
            lo = hi if rng.random() < 0.5 else max(1, hi // rng.randint(1, 20))
            past = _log_int(rng, 1, 4096) if step else rng.choice([0, 0, 32 * _log_int(rng, 1, 64)])
            if seqs * hi * (hq + 2 * h) * d > 8192 * 120 * 128 or seqs * (past + hi) * h * d > MAX_CACHE:
                continue
            rot = rng.choice([d, d, d // 2, 32, 0])
            c = _append("", layout, seqs, (lo, hi), (past if not step else 1 + past // 4, past), rot, rng.random() < 0.3,
                        rng.random() < 0.7, page)
            if c["past_lo"] > c["past_hi"]:
                c["past_lo"] = c["past_hi"]
        else:
            seqs = _log_int(rng, 1, 128) if step else _log_int(rng, 1, 16)
            hi = rng.choice([1, 1, 1, _log_int(rng, 1, 8)]) if step else _log_int(rng, 9, 8192)
            lo = hi if rng.random() < 0.5 else max(1, hi // rng.randint(1, 20))
            past = _log_int(rng, 1, 131072) if step else rng.choice([0, _log_int(rng, 1, 32768)])
            first = past if rng.random() < 0.3 else past // rng.randint(1, 10)
            if seqs * (past + hi) * h * d > MAX_CACHE or seqs * hq * hi * (past + hi) > MAX_SCORES:
                continue
            window = rng.choice([0, 0, 0, _log_int(rng, 16, 8192)])
            c = _attend("", layout, seqs, (lo, hi), (first, past), window, page)
        del c["name"]
        return c


def _lengths(case):
    """Tokens of each sequence before the call, and new ones: by the case alone."""
    r = random.Random("%(seqs)d %(new_lo)d %(new_hi)d %(past_lo)d %(past_hi)d" % case)
    past = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    # A pass of kv_append can be made again on its state unless it leaves the block that it began in by more than one block,
    # where it needs the ring's old values and overwrites them: a prompt begins a block here.
    if case["call"] == "append" and case["new_hi"] > 1:
        past = [p // BLOCK * BLOCK for p in past]
    return past, new


def _padded(d):
    return -(-d // 32) * 32


def _tiles(x, values):
    """Codes [n, heads, 32 tokens, d] as tiles [n, heads, 32 * padded d].  Keys: 32 features at a time, the first 16 of each
    token, then the other 16.  Values: 32 features at a time; half h of a tile holds, feature by feature, tokens 8 j + 4 h + e
    (j, e = 0 .. 3)."""
    n, heads, _, d = x.shape
    x = torch.nn.functional.pad(x, (0, _padded(d) - d))
    if values:
        x = x.reshape(n, heads, 4, 2, 4, -1, 32).permute(0, 1, 5, 3, 6, 2, 4)
    else:
        x = x.reshape(n, heads, 32, -1, 2, 16).permute(0, 1, 3, 4, 2, 5)
    return x.reshape(n, heads, -1)


def _from_tiles(t, d, values):
    """The inverse of _tiles for t [..., 32 * padded d]: [..., 32, d]."""
    head = t.shape[:-1]
    k = len(head)
    if values:
        x = t.reshape(*head, -1, 2, 32, 4, 4).permute(*range(k), k + 3, k + 1, k + 4, k, k + 2)
    else:
        x = t.reshape(*head, -1, 2, 32, 16).permute(*range(k), k + 2, k, k + 1, k + 3)
    return x.reshape(*head, 32, -1)[..., :d]


def _states(g, shape, large):
    """N(0, 1), the features of `large` many times as large."""
    x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g)
    return (x * large).half()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    s = [0]
    for x in n:
        s.append(s[-1] + x)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hq, h, d, page = case["heads_q"], case["heads"], case["d"], case["page"]
    past, new = _lengths(case)
    total = [p + n for p, n in zip(past, new)]
    attend = case["call"] == "attend"
    held = total if attend else past  # what the cache holds before the call
    per = [-(-t // page) for t in total]
    first, n_pages, seqs = _starts(per), sum(per) + 3, len(past)
    order = torch.randperm(n_pages, device="cuda", generator=g).int()
    pages = torch.zeros((seqs, max(per)), dtype=torch.int32, device="cuda")
    for b in range(seqs):
        pages[b, :per[b]] = order[first[b]:first[b + 1]]
    slots = torch.randperm(seqs + 1, device="cuda", generator=g)[:seqs].int()
    # three features of each head's keys are larger than the others
    large = torch.ones((h, 1, d), device="cuda")
    large.scatter_(2, torch.randint(0, d, (h, 1, 3), device="cuda", generator=g), 6.0)
    codes = torch.zeros((n_pages, h, page // BLOCK, 2, 32 * _padded(d)), dtype=torch.int8, device="cuda")
    consts = torch.zeros((n_pages, h, page // BLOCK, 2), dtype=torch.float16, device="cuda")
    ring = torch.zeros((seqs + 1, h, 2, RING, d), dtype=torch.float16, device="cuda")
    full = [n // BLOCK for n in held]
    if sum(full):
        b = torch.repeat_interleave(torch.arange(seqs, device="cuda"), torch.tensor(full, device="cuda"))
        i = torch.cat([torch.arange(n, device="cuda") for n in full])
        at, sub = pages[b, i // (page // BLOCK)].long(), i % (page // BLOCK)
        for kv in range(2):
            for s in range(0, len(i), 4096):  # some at a time: their fp32 values are many times what the cache holds
                e = min(len(i), s + 4096)
                x = _states(g, (e - s, h, 32, d), large if kv == 0 else 1.0).float()
                c = x.abs().amax((2, 3))
                codes[at[s:e], :, sub[s:e], kv] = _tiles((127.0 * x / c[:, :, None, None]).round_().to(torch.int8), kv == 1)
                consts[at[s:e], :, sub[s:e], kv] = c.half()
    for slot, n in zip(slots.tolist(), held):
        if n % BLOCK:
            p = (torch.arange(n // BLOCK * BLOCK, n, device="cuda") % RING)
            x = _states(g, (2, h, len(p), d), 1.0)
            x[0] = (x[0].float() * large).half()
            ring[slot][:, :, p] = x.transpose(0, 1)
    s = {"case": case, "past": past, "new": new, "codes": codes, "consts": consts, "ring": ring, "pages": pages,
         "slots": slots, "row_start": _ints(_starts(new)), "kv_len": _ints(total), "scale": d ** -0.5}
    rows = sum(new)
    if attend:
        s["q"] = _states(g, (rows, hq, d), 1.0)
    else:
        x = _states(g, (rows, hq + 2 * h, d), 1.0)
        x[:, hq:hq + h] = (x[:, hq:hq + h].float() * large[:, 0]).half()
        s["q"], s["k"], s["v"] = x.split([hq, h, h], 1)
        if not case["fused"]:
            s["q"], s["k"], s["v"] = (t.contiguous() for t in (s["q"], s["k"], s["v"]))
        rot = case["rot"]
        if rot:
            angle = torch.outer(torch.arange(max(total), device="cuda", dtype=torch.float64),
                                10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        # what is read back: the new tokens, and those that were in the block with the first of them
        s["back"] = [t - p // BLOCK * BLOCK for t, p in zip(total, past)]
        s["back_start"] = _ints(_starts(s["back"]))
    if own:  # the handles around these tensors, and the buffers that a program keeps from layer to layer
        import paper_2208_07339_amd as L
        s["cache"] = L.KvCache(codes, consts, ring, page, d)
        s["batch"] = L.KvBatch(s["row_start"], s["kv_len"], pages, slots, rows, max(new), max(total))
        if attend:
            s["ws"] = L.kv_attention_workspace(s["cache"], s["batch"], hq)
            s["out"] = torch.zeros((rows, hq, d), dtype=torch.float16, device="cuda")
        else:
            s["back_batch"] = L.KvBatch(s["back_start"], s["kv_len"], pages, slots, sum(s["back"]), max(s["back"]), max(total))
            s["q_out"] = torch.zeros((rows, hq, d), dtype=torch.float16, device="cuda")
            s["k_back"], s["v_back"] = (torch.zeros((sum(s["back"]), h, d), dtype=torch.float16, device="cuda") for _ in range(2))
    return s


def run(state):
    append = state["case"]["call"] == "append"
    if not own:
        return _plain_append(state) if append else _plain_attend(state)
    import paper_2208_07339_amd as L
    case = state["case"]
    if append:
        L.kv_append(state["cache"], state["batch"], state["k"], state["v"], q=state["q"], q_out=state["q_out"],
                    cos=state.get("cos"), sin=state.get("sin"), pairs=case["pairs"])
        L.kv_read(state["cache"], state["back_batch"], state["k_back"], state["v_back"])
        return {"q": state["q_out"], "k": state["k_back"], "v": state["v_back"]}
    L.kv_attention(state["cache"], state["batch"], state["q"], scale=state["scale"], window=case["window"], ws=state["ws"],
                   out=state["out"])
    return {"out": state["out"]}


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _rows_of(state):
    """Sequence and position of each new row."""
    n = sum(state["new"])
    start, length = state["row_start"].long(), state["kv_len"].long()
    b = torch.repeat_interleave(torch.arange(len(state["new"]), device="cuda"), start.diff(), output_size=n)
    return b, torch.arange(n, device="cuda") - start[b + 1] + length[b]


def _rotated(x, pos, state):
    rot, pairs = state["case"]["rot"], state["case"]["pairs"]
    if not rot:
        return x
    c, s = state["cos"][pos][:, None], state["sin"][pos][:, None]
    y = x.float()
    turned = y[..., :rot]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if pairs else turned.chunk(2, -1)
    first, second = a * c - b * s, b * c + a * s
    turned = torch.stack((first, second), -1).flatten(-2) if pairs else torch.cat((first, second), -1)
    return torch.cat((turned, y[..., rot:]), -1).half()


def _plain_append(state):
    case, page = state["case"], state["case"]["page"]
    past, new = state["past"], state["new"]
    seqs, d = len(new), case["d"]
    b, pos = _rows_of(state)
    q = _rotated(state["q"], pos, state)
    kv = torch.stack((_rotated(state["k"], pos, state), state["v"]), 1)  # [rows, 2, heads, d]
    # the blocks that hold new tokens, and those of their tokens that were there
    touched = [-(-(p + n) // BLOCK) - p // BLOCK for p, n in zip(past, new)]
    length, start = state["kv_len"].long(), state["row_start"].long()
    before = length - start.diff()
    count = -(-length // BLOCK) - before // BLOCK
    s = torch.repeat_interleave(torch.arange(seqs, device="cuda"), count, output_size=sum(touched))
    blk = torch.arange(sum(touched), device="cuda") - (count.cumsum(0) - count)[s] + before[s] // BLOCK
    p = blk[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    s2, is_new, there = s[:, None].expand_as(p), p >= before[s][:, None], p < length[s][:, None]
    row = (start[s2] + p - before[s2]).clamp(0, len(b) - 1)
    slot = state["slots"].long()
    x = torch.where(is_new[..., None, None, None], kv[row], state["ring"][slot[s2], :, :, p % RING].transpose(2, 3))
    x = torch.where(there[..., None, None, None], x, 0).permute(0, 2, 3, 1, 4)  # [blocks, 2, heads, 32, d]
    # full blocks: codes
    y = x.float()
    c = y.abs().amax((3, 4), keepdim=True)
    code = torch.where(c > 0, 127.0 * y / torch.where(c > 0, c, 1.0), 0.0).round()
    full = there[:, -1]
    value = torch.where(full[:, None, None, None, None], (code * c / 127.0).half(), x)
    # into the cache
    at, sub = state["pages"][s, blk // (page // BLOCK)].long(), blk % (page // BLOCK)
    keep = full[:, None, None]
    int8 = code.to(torch.int8)
    state["codes"][at, :, sub, 0] = torch.where(keep, _tiles(int8[:, 0], False), state["codes"][at, :, sub, 0])
    state["codes"][at, :, sub, 1] = torch.where(keep, _tiles(int8[:, 1], True), state["codes"][at, :, sub, 1])
    state["consts"][at, :, sub] = torch.where(keep, c[:, :, :, 0, 0].transpose(1, 2).half(), state["consts"][at, :, sub])
    last = pos >= length[b] // BLOCK * BLOCK - BLOCK
    lr = torch.where(last, torch.arange(len(b), device="cuda"), start[b + 1] - 1)  # a row that stays out: its sequence's last
    state["ring"][slot[b[lr]], :, :, pos[lr] % RING] = kv[lr].transpose(1, 2)
    # and read again
    n = sum(state["back"])
    back = state["back_start"].long()
    r = torch.repeat_interleave(torch.arange(seqs, device="cuda"), back.diff(), output_size=n)
    i = torch.arange(n, device="cuda") - back[r]
    block = (count.cumsum(0) - count)[r] + i // BLOCK
    return {"q": q if case["rot"] else q.clone(), "k": value[block, 0, :, i % BLOCK], "v": value[block, 1, :, i % BLOCK]}


def _plain_cache(state):
    """Keys and values of all sequences in 32 bits, [2, seqs, heads, tokens, d]; what no sequence has is zero."""
    d, pages, length = state["case"]["d"], state["pages"].long(), state["kv_len"].long()
    seqs, slots = len(length), state["slots"].long()
    codes, c = state["codes"][pages], state["consts"][pages].float() / 127.0  # [seqs, pages, heads, blocks, 2, ...]
    full = length // BLOCK * BLOCK
    p = full[:, None] + torch.arange(BLOCK, device="cuda")
    got = []
    for kv in range(2):
        x = _from_tiles(codes[..., kv, :], d, kv == 1).float() * c[..., kv, None, None]
        x = x.permute(0, 2, 1, 3, 4, 5).reshape(seqs, x.shape[2], -1, d)
        x = torch.nn.functional.pad(x, (0, 0, 0, BLOCK))
        t = torch.arange(x.shape[2], device="cuda")
        x = torch.where((t < full[:, None])[:, None, :, None], x, 0.0)
        tail = state["ring"][slots[:, None], :, kv, p % RING].float()  # [seqs, 32, heads, d]
        x[torch.arange(seqs, device="cuda")[:, None], :, p] = torch.where((p < length[:, None])[..., None, None], tail, 0.0)
        got.append(x)
    return got


def _plain_attend(state):
    case, length = state["case"], state["kv_len"].long()
    hq, h, d, window = case["heads_q"], case["heads"], case["d"], case["window"]
    seqs, most = len(length), max(state["new"])
    b, pos = _rows_of(state)
    i = torch.arange(len(b), device="cuda") - state["row_start"].long()[b]
    q = torch.zeros((seqs, most, hq, d), device="cuda")
    q[b, i] = state["q"].float()
    at = torch.full((seqs, most), -1, device="cuda")
    at[b, i] = pos
    k, v = _plain_cache(state)
    q = q.view(seqs, most, h, hq // h, d).permute(0, 2, 3, 1, 4).reshape(seqs, h, -1, d)  # heads that share keys: as rows
    score = (q @ k.transpose(2, 3)).mul_(state["scale"])
    t = torch.arange(k.shape[2], device="cuda")
    hidden = t > at[..., None]
    if window:
        hidden |= t <= at[..., None] - window
    score.view(seqs, h, hq // h, most, -1).masked_fill_(hidden[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True).clamp_(min=-1e30)
    score.sub_(top).exp_()
    out = (score @ v) / score.sum(-1, keepdim=True).clamp_(min=1e-30)
    out = out.view(seqs, h, hq // h, most, d).permute(0, 3, 1, 2, 4).reshape(seqs, most, hq, d)
    return {"out": out[b, i].half()}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    hq, h, d = case["heads_q"], case["heads"], case["d"]
    past, new = _lengths(case)
    rows = sum(new)

    def cached(lo, hi, closed):
        """Bytes of keys and values of positions lo .. hi - 1, those below `closed` as codes."""
        n8 = max(0, min(hi, closed) - lo)
        return 2 * h * d * n8 + 4 * h * -(-n8 // BLOCK) + 4 * h * d * (max(0, hi - lo) - n8)

    moved, flops = 4 * rows * hq * d, 0
    for p, n in zip(past, new):
        t = p + n
        closed = t // BLOCK * BLOCK
        if case["call"] == "attend":
            w = case["window"] or t
            seen = sum(min(x, w) for x in (p + 1, t)) * n / 2 if w >= t or p + 1 >= w else sum(min(x, w) for x in range(p + 1, t + 1))
            flops += 4 * hq * d * seen
            moved += cached(max(0, p + 1 - w), t, closed)
        else:
            f = p // BLOCK * BLOCK
            moved += 4 * h * d * n                                # the new keys and values
            moved += 4 * h * d * (p - f)                          # tokens that were in the block
            moved += cached(f, closed, closed) + 4 * h * d * min(n, t - max(0, closed - BLOCK))  # written
            moved += cached(f, t, closed) + 4 * h * d * (t - f)   # read again
            flops += (3 * case["rot"] * (hq + h) + 4 * h * d) * n
    if case["call"] == "append" and case["rot"]:
        moved += 4 * case["rot"] * (max(p + n for p, n in zip(past, new)) - min(past) if max(new) > 1 else len(set(past)))
    return {"bytes": moved, "flops": flops}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------

def _exact_block(state, b, j, kv):
    """Values of full block j of sequence b as held: [heads, 32, d] in 64 bits, element by element from the tiles."""
    page, d = state["case"]["page"], state["case"]["d"]
    at, sub = int(state["pages"][b, j * BLOCK // page]), j % (page // BLOCK)
    return _exact_values(state["codes"][at, :, sub, kv], state["consts"][at, :, sub, kv], d, kv)


def _exact_values(tiles, consts, d, kv):
    token = torch.arange(BLOCK, device="cuda")[:, None]
    f = torch.arange(d, device="cuda")[None]
    if kv:
        byte = f // 32 * 1024 + token // 4 % 2 * 512 + f % 32 * 16 + token // 8 * 4 + token % 4
    else:
        byte = f // 32 * 1024 + f // 16 % 2 * 512 + token * 16 + f % 16
    return tiles[..., byte].double() * consts.double()[..., None, None] / 127.0


def _exact_attend(state):
    case = state["case"]
    hq, h, d, page, window = case["heads_q"], case["heads"], case["d"], case["page"], case["window"]
    out, row = [], 0
    for b, (p, n) in enumerate(zip(state["past"], state["new"])):
        t, g = p + n, hq // h
        q = state["q"][row:row + n].double()
        row += n
        pos = torch.arange(p, t, device="cuda").repeat_interleave(g)
        result = torch.empty((n, hq, d), dtype=torch.float64, device="cuda")
        closed = t // BLOCK
        j = torch.arange(closed, device="cuda")
        at, sub = state["pages"][b].long()[j * BLOCK // page], j % (page // BLOCK)
        rest = torch.arange(closed * BLOCK, t, device="cuda") % RING
        slot = int(state["slots"][b])
        for one in range(h):
            kv = [torch.cat((_exact_values(state["codes"][at, one, sub, w], state["consts"][at, one, sub, w], d, w).reshape(-1, d),
                             state["ring"][slot, one, w][rest].double())) for w in range(2)]
            rows = q[:, one * g:(one + 1) * g].reshape(-1, d)
            for s in range(0, n * g, 4096):
                score = rows[s:s + 4096] @ kv[0].T * state["scale"]
                behind = pos[s:s + 4096, None] - torch.arange(t, device="cuda")
                score[behind < 0] = float("-inf")
                if window:
                    score[behind >= window] = float("-inf")
                o = torch.softmax(score, -1) @ kv[1]
                i = torch.arange(s, min(n * g, s + 4096), device="cuda")
                result[i // g, one * g + i % g] = o
        out.append(result)
    return {"out": torch.cat(out)}


def _exact_turned(x, p, state):
    rot = state["case"]["rot"]
    x = x.double()
    if rot:
        c, s = (state[w][p:p + len(x)].double()[:, None] for w in ("cos", "sin"))
        i = torch.arange(rot // 2, device="cuda")
        first, second = (2 * i, 2 * i + 1) if state["case"]["pairs"] else (i, i + rot // 2)
        a, b = x[..., first], x[..., second]
        x[..., first], x[..., second] = a * c - b * s, a * s + b * c
    return x


def _exact_append(state):
    d, row = state["case"]["d"], 0
    q, kv = [], ([], [])
    for b, (p, n) in enumerate(zip(state["past"], state["new"])):
        q.append(_exact_turned(state["q"][row:row + n], p, state))
        f, t, slot = p // BLOCK * BLOCK, p + n, int(state["slots"][b])
        old = torch.arange(f, p, device="cuda") % RING
        for w, x in enumerate((_exact_turned(state["k"][row:row + n], p, state).half(), state["v"][row:row + n])):
            x = torch.cat((state["ring"][slot, :, w][:, old].transpose(0, 1), x)).double()  # what a block is made of is fp16
            m = (t // BLOCK * BLOCK) - f
            y = x[:m].reshape(-1, BLOCK, *x.shape[1:])
            c = y.abs().amax((1, 3), keepdim=True)
            x[:m] = (torch.round(127.0 * y / c) * c / 127.0).reshape(m, *x.shape[1:])
            kv[w].append(x)
        row += n
    return {"q": torch.cat(q), "k": torch.cat(kv[0]), "v": torch.cat(kv[1])}


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_append(state) if case["call"] == "append" else _exact_attend(state)
