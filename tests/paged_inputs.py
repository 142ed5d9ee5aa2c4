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


def _index_maps():
    """Word and lowest bit of the code of (row of a block, channel), for keys and for values."""
    r, e = torch.arange(32)[:, None], torch.arange(128)[None, :]
    half, n, m, j, i = r // 16, r % 16, e // 32, (e % 32) // 8, e % 8
    kw, kb = (16 * j + n) * 4 + 2 * half + m // 2, 2 * (8 * (m % 2) + i)
    nb, ch = e // 16, e % 16
    vw, vb = (16 * (n // 4) + ch) * 4 + 2 * (nb % 2) + nb // 4, 16 * half + 2 * (4 * ((nb // 2) % 2) + n % 4)
    return [x.expand(32, 128).contiguous() for x in (kw, kb, vw, vb)]


def hadamard(x):
    """x (64 bits) times the orthonormal 128-point matrix."""
    h = torch.ones(1, 1, dtype=torch.float64)
    for _ in range(7):
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return x @ (h / 128 ** 0.5).to(x.device)


def cached_rows(s, b, t):
    """The first t rows that sequence b's pages and overlay hold, un-rotated, in 64 bits: (k, v, there) with [Hkv, t, 128] and, for
    rows that take part (a page, or a place in the overlay), [Hkv, t] true."""
    p, Hkv, G = s.cache, s.Hkv, s.G
    maps = [m.cuda() for m in _index_maps()]
    row = torch.arange(t, device="cuda")
    page = p.table[b].long()[row // p.page_rows]
    there = (page >= 0) & (page < p.n_pages)
    page = torch.where(there, page, torch.zeros_like(page))
    at = row % p.page_rows
    there = there.expand(Hkv, t).clone()
    out = []
    slots = torch.arange(p.S_cap, device="cuda")
    for which, (codes, metas) in enumerate(((p.k_codes, p.k_meta), (p.v_codes, p.v_meta))):
        words, bits = maps[2 * which:2 * which + 2]
        block = codes[page, :, at // 32].transpose(0, 1)                                      # [Hkv, t, 256]
        code = (torch.gather(block, 2, words[at % 32].expand(Hkv, t, 128)) >> bits[at % 32]) & 3
        meta = metas[page, :, at].transpose(0, 1).repeat_interleave(G, dim=2)
        x = (meta & 0x7FFF).short().view(torch.float16).double() * (code - (meta >> 16)).double()
        for h in range(Hkv):
            k = min(int(p.counts()[b, h]), p.S_cap)
            idx = p.sal_idx[b, h, :k].long()
            keep = idx < t
            mine = slots[:k][keep]
            if which == 0:
                rows = p.k_sal[b, h, mine].view(torch.bfloat16).double()
            else:
                tiles = p.v_sal[b, h].view(torch.bfloat16).double().reshape(-1, 8, 4, 16, 4, 2)  # nb, q, n, ii, half
                rows = tiles.permute(0, 5, 2, 4, 1, 3).reshape(p.S_cap, 128)[mine]
            x[h, idx[keep]] = rows
            there[h, idx[keep]] = True
        out.append(hadamard(x))
    return out[0], out[1], there


def attention64(s, b, sm_scale):
    """The formula in 64 bits for the chunk's rows of sequence b: out [n, Hq, 128], lse [n, Hq], and what bounds rounding errors: the
    weighted norms of the value rows and the largest |q| |k| that a row meets, both [n, Hq]."""
    lo, hi, t = s.starts[b], s.starts[b + 1], s.lens[b]
    n, R = hi - lo, s.Hq // s.Hkv
    kc, vc, there = cached_rows(s, b, t)
    seen = torch.cat((torch.ones(n, t, device="cuda"), torch.ones(n, n, device="cuda").tril()), 1).bool()
    out = torch.empty(n, s.Hq, 128, dtype=torch.float64, device="cuda")
    lse, vnorm, qk = (torch.empty(n, s.Hq, dtype=torch.float64, device="cuda") for _ in range(3))
    for h in range(s.Hq):
        g = h // R
        k = torch.cat((kc[g], s.k[lo:hi, g].double()))
        v = torch.cat((vc[g], s.v[lo:hi, g].double()))
        mask = seen & torch.cat((there[g], torch.ones(n, dtype=torch.bool, device="cuda")))
        logits = (s.q[lo:hi, h].double() @ k.t().contiguous() * sm_scale).masked_fill(~mask, float("-inf"))
        p = torch.softmax(logits, 1)
        out[:, h], lse[:, h] = p @ v, torch.logsumexp(logits, 1)
        vnorm[:, h] = p @ v.norm(dim=1)
        qk[:, h] = s.q[lo:hi, h].double().norm(dim=1) * (mask * k.norm(dim=1)).amax(1)
    return out, lse, vnorm, qk * abs(sm_scale)


def check_attention(s, got, lse, sm_scale, what=""):
    """Bounds, per row in the 2-norm (which the rotation keeps): a score is off by 2^-15 |q| |k| sm_scale (queries of 20 and 16 bits, and
    32-bit sums), a weight by twice that and by half a step of binary16, 2^-11 (16-bit rows: less), and the result by its own rounding,
    2^-11 of it (2^-25 an element where it is below the smallest normal number)."""
    for b in range(s.cache.B):
        lo, hi = s.starts[b], s.starts[b + 1]
        if hi == lo:
            continue
        want, wlse, vnorm, qk = attention64(s, b, sm_scale)
        err = (got[lo:hi].double() - want).norm(dim=2)
        score = 2.0 ** -15 * qk
        bound = 2.0 ** -11 * want.norm(dim=2) + 2.0 ** -25 * 128 ** 0.5 + (2.0 ** -11 + 2 * score + 2.0 ** -18) * vnorm
        assert bool((err <= bound).all()), (what, b, float((err / bound).max()), float((err / want.norm(dim=2)).max()))
        if lse is not None:
            d = (lse[lo:hi].double() - wlse).abs()
            assert bool((d <= score + 2.0 ** -18 * (1 + wlse.abs())).all()), (what, b, float(d.max()))
