"""A pipeline.PagedDecode on the CPU: its calls of the library are stood in for by what the header says of them, over a record of who wrote which
slot of which page."""
import torch

OK, INVALID = 0, 1


class Pages:
    def __init__(self, k, v, k_scales, v_scales, table, lengths):
        self.k = self.v = self.k_scales = self.v_scales = k         # [pages, page_size]: who wrote a slot, -1 nobody yet
        self.table, self.lengths, self.batch = table, lengths, table.shape[0]
        self.pages, self.page_size = k.shape
        self.slots = table.shape[1] * self.page_size

    @staticmethod
    def empty(pages, n_kv_heads, page_size, head_dim, table, lengths):
        store = torch.full((pages, page_size), -1, dtype=torch.int64)
        return Pages(store, store, store, store, table, lengths)

    def place(self, b, slot):
        page = int(self.table[b, slot // self.page_size])
        return (page, slot % self.page_size) if 0 <= page < self.pages else None


class Cache:
    def __init__(self, k, v, positions, weights, lengths):
        self.lengths = lengths


class Context:
    """`told`: the device status word.  `marks`: of the sequences of a call, what their rows are marked with (None: their numbers)."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim, window, max_seq, dtype, device):
        self.told, self.seen, self.marks, self.dtype = OK, [], None, dtype

    def poll_device_status(self):
        told, self.told = self.told, OK
        return told

    def attend_pages_workspace(self, pages, n_new):
        return torch.empty(256 * n_new, dtype=torch.uint8)

    def commit(self, cache, n_new, counts=None, path=None):
        assert counts.dtype == torch.int32 and counts.is_contiguous() and path is None
        for b, c in enumerate(counts.tolist()):
            if 0 <= c <= n_new:
                cache.lengths[b] += c
            else:
                self.told = INVALID

    def _rows(self, pages, b, n_new, counts):
        assert counts is None or (counts.shape == (pages.batch,) and counts.dtype == torch.int32 and counts.is_contiguous())
        n, c = int(pages.lengths[b]), n_new if counts is None else int(counts[b])
        if n < 0 or c < 0 or c > n_new or n > pages.slots - c:
            self.told = INVALID
            return n, -1
        return n, c

    def append_pages(self, pages, k_new, v_new, positions=None, rope=None, counts=None, index=None, q=None, q_out=None):
        for b in range(pages.batch):
            n, c = self._rows(pages, b, k_new.shape[1] if index is None else index.shape[-1], counts)
            for slot in range(n, n + c):
                at = pages.place(b, slot)
                if at is None:
                    self.told = INVALID
                else:
                    pages.k[at] = b if self.marks is None else self.marks[b]

    def attend_pages(self, pages, q, scale, out, workspace, counts=None, softcap=0.0, lse=None):
        """`seen`: of every sequence, who wrote the slots that its last token sees."""
        out.zero_()
        self.seen = []
        for b in range(pages.batch):
            n, c = self._rows(pages, b, q.shape[1], counts)
            places = [pages.place(b, slot) for slot in range(n + c)] if c > 0 else []
            if None in places:
                self.told = INVALID
            self.seen.append([int(pages.k[at]) for at in places if at is not None])


def decode(monkeypatch, pages, columns, batch, page_size=16, max_new=4):
    from paper_2604_06746_b200 import pipeline
    for name, fake in (("Pages", Pages), ("Cache", Cache), ("Context", Context)):
        monkeypatch.setattr(pipeline.binding, name, fake)
    return pipeline.PagedDecode(1, 4, 2, 64, pages, columns, torch.bfloat16, batch=batch, page_size=page_size, max_new=max_new, device="cpu")


def rows(batch, n, heads=2):
    return torch.zeros((batch, n, heads, 64), dtype=torch.bfloat16)


def keep(dec, sequence, n):
    """A prompt of n tokens, marked with the sequence's number."""
    dec.ctx.marks = [sequence]
    dec.keep(0, sequence, *(torch.zeros((2, n, 64), dtype=torch.bfloat16) for _ in range(2)))
    dec.ctx.marks = None
    dec.advance(torch.tensor([n if b == sequence else 0 for b in range(dec.B)], dtype=torch.int32))


def step(dec, n=1, **more):
    out = rows(dec.B, n, 4)
    dec.step(0, torch.ones_like(out), rows(dec.B, n), rows(dec.B, n), None, 1.0, out, **more)
    return dec.ctx.seen
