"""The bookkeeping of kv_pages_util.py, with what include/llmint8.h says where pages are too few: no sequence that is served writes to a block
that another one holds."""
from kv_pages_util import BLOCK, NO_PAGE, Book


def written_over(pages, ready, held, rows, page_tokens):
    """Sequences that are served and would write to a block that is another's: (writer, page, block, the other).  pages: tables after the call;
    held: full blocks of each sequence before its tokens."""
    per = page_tokens // BLOCK
    names = {}
    for q, row in enumerate(pages):
        for j, e in enumerate(row):
            if e >= 0 and j * per < held[q]:
                names.setdefault(e, []).append((q, held[q] - j * per))
    found = []
    for b, length in enumerate(ready):
        if length and rows[b]:
            for k in range((length - rows[b]) // BLOCK, length // BLOCK):
                e = pages[b][k // per]
                found += [(b, e, k % per, q) for q, blocks in names.get(e, ()) if q != b and k % per < blocks]
    return found


def full_blocks(kv_len, rows):
    return [max(0, n - r) // BLOCK for n, r in zip(kv_len, rows)]


class ServedBook(Book):
    def reserve(self, row_start, more=False):
        before = [list(row) for row in self.pages]
        rows = [b - a for a, b in zip(row_start, row_start[1:])]
        ready = super().reserve(row_start, more)
        for b, _, _, q in written_over(self.pages, ready, full_blocks(self.kv_len, rows), rows, self.page):
            assert ready[q] == 0 and q < b and self.pages[b] == before[b]
            ready[b] = 0
            self.status |= NO_PAGE
        return ready
