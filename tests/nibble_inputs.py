"""Sequences in pages of 4-bit codes for the tests, and the write path and attention from their definition."""
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, hadamard

THIRD, FIFTEENTH, KAPPA = 0.3333333432674408, 0.06666667014360428, 0.08838834613561630  # 1/3, 1/15 and 2^-3.5 in binary32


def with_bits(s, bits=4, fill=0):
    """Sequences of paged_inputs whose pages hold codes of so many bits."""
    old = s.cache
    s.cache = akvq.PagedCache(old.B, old.Hkv, old.G, old.n_pages, old.max_pages, old.page_rows, old.S_cap, fill=fill, bits=bits)
    for name in ("table", "sal_idx", "seq_len"):
        getattr(s.cache, name).copy_(getattr(old, name))
    s.cache.counts().copy_(old.counts())
    return s


def sequences(*args, bits=4, **kw):
    return with_bits(Sequences(*args, **kw), bits)


def code_places():
    """Word and lowest bit of the 4-bit code of (row of a block, channel), for keys and for values."""
    r, e = torch.arange(32)[:, None], torch.arange(128)[None, :]
    kw = r // 16 * 256 + (16 * ((e % 32) // 8) + r % 16) * 4 + e // 32
    kb = 4 * (e % 8)
    vw = (e // 16) % 2 * 256 + (16 * ((r % 16) // 4) + e % 16) * 4 + e // 32
    vb = 16 * (r // 16) + 4 * (r % 4)
    return [x.expand(32, 128).contiguous() for x in (kw, kb, vw, vb)]


def transformed(x, rotate=True):
    """Rows [..., 128] as 32-bit numbers, un-normalised Walsh-Hadamard transform: strides 1 to 64, (a, b) -> (a + b, a - b), each rounded."""
    x = x.float()
    h = 1
    while rotate and h < 128:
        y = x.reshape(*x.shape[:-1], 128 // (2 * h), 2, h)
        x = torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).reshape(x.shape)
        h *= 2
    return x


def quantized(x, G, bits, clip, rotate=True):
    """Codes [..., 128], meta words [..., 128/G] and 16-bit rows of rows x (binary16), by the definition: every rounding but the code's is one of a
    32-bit operation; the code is the exact u / scale + zero (exact in 64 bits but for ties that no input here has) rounded to even."""
    u = transformed(x, rotate)
    kappa = KAPPA if rotate else 1.0
    g = u.reshape(*u.shape[:-1], 128 // G, G)
    clip = torch.tensor(clip, dtype=torch.float32, device=x.device)
    lo, hi = clip * (g.amin(-1) * kappa), clip * (g.amax(-1) * kappa)
    s32 = (hi - lo) * (THIRD if bits == 2 else FIFTEENTH)
    s16 = s32.half()
    s16 = torch.where(s16.double() < s32.double(), torch.nextafter(s16.float().half(), torch.full_like(s16, float("inf"))), s16)
    s16 = torch.where(torch.isinf(s16), torch.full_like(s16, 65504.0), s16)
    s16 = torch.where(s32 > 0, s16, torch.ones_like(s16))
    rcp = (1.0 / s16.double()).float()
    zero = (-torch.round(lo * rcp)).clamp(-32768, 32767)
    exact = g.double() * (rcp * torch.tensor(kappa, dtype=torch.float32)).double()[..., None] + zero.double()[..., None]
    code = exact.round().clamp(0, 2 ** bits - 1).long().reshape(x.shape)
    meta = s16.view(torch.int16).int() | (zero.int() << 16)
    return code, meta, (u * kappa + 0.0).bfloat16()


def page_codes(s, b, t):
    """Codes, meta words (without the mark of 16-bit rows) and marks of the first t rows of sequence b: two of (keys, values) each, per head."""
    p = s.cache
    maps = [m.cuda() for m in code_places()]
    row = torch.arange(t, device="cuda")
    page, at = p.table[b].long()[row // p.page_rows], row % p.page_rows
    there = (page >= 0) & (page < p.n_pages)
    page = torch.where(there, page, torch.zeros_like(page))
    out = []
    for which, (codes, metas) in enumerate(((p.k_codes, p.k_meta), (p.v_codes, p.v_meta))):
        words, bits = maps[2 * which:2 * which + 2]
        block = codes[page, :, at // 32].transpose(0, 1)
        code = (torch.gather(block, 2, words[at % 32].expand(p.Hkv, t, 128)) >> bits[at % 32]) & 15
        meta = metas[page, :, at].transpose(0, 1)
        out.append((code, meta & ~0x8000, (meta & 0x8000) != 0))
    return out, there


def overlay(p, b, h, which):
    """16-bit rows of a head in slot order [S_cap, 128]."""
    if which == 0:
        return p.k_sal[b, h].view(torch.bfloat16).double()
    tiles = p.v_sal[b, h].view(torch.bfloat16).double().reshape(-1, 8, 4, 16, 4, 2)  # nb, q, n, ii, half
    return tiles.permute(0, 5, 2, 4, 1, 3).reshape(p.S_cap, 128)


def cached_rows(s, b, t):
    """The first t rows that sequence b's pages and overlay hold, un-rotated, in 64 bits: (k, v, there) [Hkv, t, 128], [Hkv, t]."""
    p = s.cache
    parts, there = page_codes(s, b, t)
    there = there.expand(p.Hkv, t).clone()
    out = []
    for which, (code, meta, _) in enumerate(parts):
        meta = meta.repeat_interleave(p.G, dim=2)
        x = (meta & 0x7FFF).short().view(torch.float16).double() * (code - (meta >> 16)).double()
        for h in range(p.Hkv):
            idx = p.sal_idx[b, h, :min(int(p.counts()[b, h]), p.S_cap)].long()
            slots = torch.nonzero(idx < t).flatten()
            x[h, idx[slots]] = overlay(p, b, h, which)[slots]
            there[h, idx[slots]] = True
        out.append(hadamard(x))
    return out[0], out[1], there


def check_attention(s, got, lse, sm_scale, what=""):
    """Attention from its formula in 64 bits on what the pages hold.  Bounds, per row in the 2-norm (which the rotation keeps): a score is off by
    2^-15 |q| |k| sm_scale (queries of 20 and 16 bits, and 32-bit sums), a weight by twice that and by half a step of binary16, 2^-11 (with two
    groups a row it is the product with a group's scale that is rounded); and the result by its own rounding, 2^-11 of it (2^-25 an element
    where it is below the smallest normal number)."""
    for b in range(s.cache.B):
        lo, hi, t = s.starts[b], s.starts[b + 1], s.lens[b]
        n, R = hi - lo, s.Hq // s.Hkv
        if n == 0:
            continue
        kc, vc, there = cached_rows(s, b, t)
        seen = torch.cat((torch.ones(n, t, device="cuda"), torch.ones(n, n, device="cuda").tril()), 1).bool()
        for h in range(s.Hq):
            g = h // R
            k, v = torch.cat((kc[g], s.k[lo:hi, g].double())), torch.cat((vc[g], s.v[lo:hi, g].double()))
            mask = seen & torch.cat((there[g], torch.ones(n, dtype=torch.bool, device="cuda")))
            logits = (s.q[lo:hi, h].double() @ k.t().contiguous() * sm_scale).masked_fill(~mask, float("-inf"))
            p = torch.softmax(logits, 1)
            want, wlse = p @ v, torch.logsumexp(logits, 1)
            score = 2.0 ** -15 * abs(sm_scale) * s.q[lo:hi, h].double().norm(dim=1) * (mask * k.norm(dim=1)).amax(1)
            err = (got[lo:hi, h].double() - want).norm(dim=1)
            bound = 2.0 ** -11 * want.norm(dim=1) + 2.0 ** -25 * 128 ** 0.5 + (2.0 ** -11 + 2 * score + 2.0 ** -18) * (p @ v.norm(dim=1))
            assert bool((err <= bound).all()), (what, b, h, float((err / bound).max()), float((err / want.norm(dim=1)).max()))
            if lse is not None:
                d = (lse[lo:hi, h].double() - wlse).abs()
                assert bool((d <= score + 2.0 ** -18 * (1 + wlse.abs())).all()), (what, b, h, float(d.max()))
