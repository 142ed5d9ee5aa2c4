"""Sequences in pages for the tests: random rows, page tables in no order, salient lists."""
import torch

from paper_2501_15021_amd import binding as akvq


class Sequences:
    """lens cached and rows new rows of every sequence.  The history's and the chunk's rows are kept per sequence, [Hkv, t, 128]."""

    def __init__(self, lens, rows, Hkv, G, page_rows=64, Hq=None, salient=(), seed=0, spare=2, gain=8.0, S_cap=None, extra_rows=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.rows, self.Hkv, self.G, self.Hq = list(lens), list(rows), Hkv, G, Hq or Hkv
        B = len(self.lens)
        need = [(t + n + page_rows - 1) // page_rows for t, n in zip(lens, rows)]
        max_pages, n_pages = max(max(need), 1), sum(need) + spare
        totals = [t + n for t, n in zip(lens, rows)]
        most = max(sum(1 for p in salient if p < t) for t in totals)
        S_cap = S_cap or max(64, (most + 63) // 64 * 64)
        self.cache = akvq.PagedCache(B, Hkv, G, n_pages, max_pages, page_rows, S_cap, fill=0)
        order = torch.randperm(n_pages, generator=g, device="cuda").int()
        at = 0
        for b in range(B):
            self.cache.table[b, : need[b]] = order[at:at + need[b]]
            at += need[b]
        self.unused = order[at:]
        for b, t in enumerate(totals):
            mine = [p for p in salient if p < t][:S_cap]
            if mine:
                self.cache.sal_idx[b, :, : len(mine)] = torch.tensor(mine, dtype=torch.int32, device="cuda")
                self.cache.counts()[b] = len(mine)

        def draw(n, channels=0.0):
            x = torch.randn(Hkv, n, 128, generator=g, device="cuda")
            x[:, :, 5] *= gain if channels else 1.0
            return x.half()

        self.past = [(draw(t, 1.0), draw(t)) for t in lens]
        starts = [0]
        for n in rows:
            starts.append(starts[-1] + n)
        self.n = starts[-1]
        self.starts = starts
        x = torch.randn(self.n + extra_rows, self.Hq + 2 * Hkv, 128, generator=g, device="cuda")
        x[:, self.Hq:self.Hq + Hkv, 5] *= gain
        self.x = x.half()
        self.q, self.k, self.v = self.x[:, :self.Hq], self.x[:, self.Hq:self.Hq + Hkv], self.x[:, self.Hq + Hkv:]
        self.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.max_rows = max(max(rows), 1)

    def fill_pages(self, clip=0.8, flags=0):
        """The history into the pages, in one call; leaves seq_len at lens."""
        k = torch.cat([p[0].transpose(0, 1) for p in self.past])
        v = torch.cat([p[1].transpose(0, 1) for p in self.past])
        starts = [0]
        for t in self.lens:
            starts.append(starts[-1] + t)
        self.cache.seq_len.zero_()
        if starts[-1]:
            akvq.paged_append(self.cache, k.contiguous(), v.contiguous(), torch.tensor(starts, dtype=torch.int32, device="cuda"),
                              max(self.lens), clip, flags)
        self.cache.seq_len.copy_(torch.tensor(self.lens, dtype=torch.int32))
        return self

    def contiguous(self, b, T_cap=None):
        """Sequence b's pages copied into a contiguous cache of its own (rows without a page: zeros)."""
        p = self.cache
        total = p.max_pages * p.page_rows
        T_cap = T_cap or (total + 63) // 64 * 64
        c = akvq.Cache(1, self.Hkv, self.G, T_cap, p.S_cap, fill=0)
        for i, page in enumerate(p.table[b].tolist()):
            if 0 <= page < p.n_pages:
                blocks, r = p.page_rows // 32, p.page_rows
                c.k_codes[0, :, i * blocks:(i + 1) * blocks] = p.k_codes[page]
                c.v_codes[0, :, i * blocks:(i + 1) * blocks] = p.v_codes[page]
                c.k_meta[0, :, i * r:(i + 1) * r] = p.k_meta[page]
                c.v_meta[0, :, i * r:(i + 1) * r] = p.v_meta[page]
        for name in ("k_sal", "v_sal", "sal_idx"):
            getattr(c, name)[0] = getattr(p, name)[b]
        c.counts()[0] = p.counts()[b]
        c.T_len = self.lens[b]
        return c
