"""The bookkeeping of pages and sequences as include/llmint8.h says it, one sequence and page at a time, on lists."""
BLOCK = 32
BAD_BATCH, BAD_PAGE, NO_PAGE = 1, 2, 8


class Book:
    def __init__(self, pages, refs, kv_len, slots, page_tokens):
        self.pages, self.refs, self.kv_len, self.slots, self.page = [list(r) for r in pages], list(refs), list(kv_len), list(slots), page_tokens
        self.status, self.page_moves, self.slot_moves = 0, [], []

    def named(self, e):
        if e >= len(self.refs):
            self.status |= BAD_PAGE
        return 0 <= e < len(self.refs)

    def fork(self, parent, grow=0):
        n = len(parent)
        if any(p < -1 or p >= n for p in parent):
            self.status |= BAD_BATCH
        parent = [p if 0 <= p < n else -1 for p in parent]
        old = [[e if self.named(e) else -1 for e in row] for row in self.pages]
        for b, row in enumerate(old):
            for e in row:
                if e >= 0:
                    self.refs[e] += parent.count(b) - 1
        spare = [self.slots[b] for b in range(n) if b not in parent]
        lengths, slots = self.kv_len, self.slots
        self.pages = [(list(old[p]) if p != i else self.pages[i]) if p >= 0 else [-1] * len(old[i]) for i, p in enumerate(parent)]
        self.kv_len, self.slots, self.page_moves, self.slot_moves = [0] * n, [None] * n, [], []
        for i, p in enumerate(parent):
            if p < 0:
                continue
            length = lengths[p]
            possible = 0 <= length <= 1 << 28
            if not possible:
                self.status |= BAD_BATCH
            self.kv_len[i] = length + grow if possible and length else length
            if parent.index(p) == i:
                self.slots[i] = slots[p]
            else:
                self.slots[i] = spare.pop(0)
                first = max(0, length // BLOCK - 1) * BLOCK
                self.slot_moves.append([slots[p], self.slots[i], first, length - first] if possible else [slots[p], self.slots[i], 0, 0])
        for i, p in enumerate(parent):
            if p < 0:
                self.slots[i] = spare.pop(0)

    def reserve(self, row_start, more=False):
        n, per = len(self.pages), self.page // BLOCK
        free = [p for p, c in enumerate(self.refs) if c == 0]
        ready, wanted, refs = [], [], list(self.refs)
        for b in range(n):
            rows, length = row_start[b + 1] - row_start[b], self.kv_len[b]
            end = -(-length // self.page)
            ok = rows >= 0 and 0 <= length <= 1 << 28 and (rows == 0 or length == 0 or (rows <= length and end <= len(self.pages[b])))
            if not ok:
                self.status |= BAD_BATCH
            ready.append(length if ok else 0)
            needs = []
            if ok and rows and length:
                old = length - rows
                for j in range(old // self.page, end):
                    e = self.pages[b][j]
                    first = j == old // self.page
                    closing = max(old // BLOCK, j * per) < min(length // BLOCK, (j + 1) * per)
                    if not self.named(e):
                        needs.append([j, None, 0])
                    elif closing and refs[e] > 1:
                        needs.append([j, e, old // BLOCK - j * per if first else -1])
            wanted.append(needs)
        # the last of those that all want a page for their first tokens keeps it
        first = {}
        for b, needs in enumerate(wanted):
            for j, e, kept in needs:
                if e is not None and kept >= 0:
                    first.setdefault(e, []).append(b)
        for e, who in first.items():
            if len(who) >= refs[e]:
                wanted[who[-1]] = [x for x in wanted[who[-1]] if x[1] != e or x[2] < 0]
        self.page_moves = []
        if not more:
            self.slot_moves = []
        so_far = 0
        for b, needs in enumerate(wanted):
            so_far += len(needs)
            if needs and so_far > len(free):
                self.status |= NO_PAGE
                ready[b] = 0
                continue
            for k, (j, e, kept) in enumerate(needs):
                p = free[so_far - len(needs) + k]
                self.pages[b][j] = p
                self.refs[p] = 1
                if e is not None:
                    self.refs[e] -= 1
                    if kept > 0:
                        self.page_moves.append([e, p, kept, 0])
        return ready

    def compact(self):
        used = sum(c != 0 for c in self.refs)
        gaps = [p for p in range(used) if self.refs[p] == 0]
        to = {}
        for p in range(used, len(self.refs)):
            if self.refs[p]:
                to[p] = gaps.pop(0)
                self.refs[to[p]], self.refs[p] = self.refs[p], 0
        self.page_moves, self.slot_moves = [[p, q, self.page // BLOCK, 0] for p, q in to.items()], []
        self.pages = [[to.get(e, e) for e in row] for row in self.pages]
        return used

    def counted(self):
        """refs as the tables say."""
        refs = [0] * len(self.refs)
        for row in self.pages:
            for e in row:
                if e >= 0:
                    refs[e] += 1
        return refs
