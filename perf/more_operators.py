"""Operators of a server that keeps a cache of 4-bit (or 2-bit) codes in pages and turns queries and keys by their positions on the way into it.

A case is one call through the public entry points (`paper_2501_15021_amd.binding`) on one layer:

  rotary       rotary positions of a chunk's query and key rows, in either layout, of a part of the head or the whole (rotary_rows)
  append_turn  a chunk's queries and keys turned, its keys and values quantized into the pages of their sequences, in one call (paged_append_rotary)
  append       keys and values that come turned, quantized into pages of 4-bit codes (paged_append)
  attend       attention of a chunk's queries over their sequences' pages of 4-bit codes and over the chunk itself (paged_attention)

Rows of a chunk are packed token by token, sequence after sequence, and come as parts of one fused projection: a row holds the query
heads, the key heads and the value heads one after the other.  Fields of a case: kind, Hq, Hkv, B (sequences), T (cached rows of the
longest one), n (new rows of the longest chunk), ragged (unequal lengths, one chunk without rows); of a cache: bits, G (quantization
group), mode ("psa": top_k pivots of every head are 16-bit, "tsa": the text tokens are, "none": no row is), P (rows of a page); of positions:
axes, pairs ("half": channels i and i + dim / 2, "next": 2 i and 2 i + 1), dim (channels that turn), stretch (how many times longer than
trained), inverse.
"""
import math

import torch

own = False

D = 128
CLIP = {2: 0.8, 4: 1.0}
SCALE = 1.0 / math.sqrt(D)
IMAGE, TEXT = 576, 96  # a 24 x 24 grid of vision tokens, and the text between two of them


def _case(name, kind, B, T, n, Hq, Hkv, ragged, **more):
    c = dict(kind=kind, B=B, T=T, n=n, Hq=Hq, Hkv=Hkv, ragged=ragged, **more)
    return dict(c, name=name) if name else c


def _turns(axes=1, pairs="half", dim=D, stretch=1.0, inverse=False):
    return dict(axes=axes, pairs=pairs, dim=dim, stretch=stretch, inverse=inverse)


def _pages(bits=4, G=128, mode="psa", top_k=16, P=64):
    return dict(bits=bits, G=G, mode=mode, top_k=top_k, P=P)


def listed():
    return [
        # a batch of conversations, one generated token each, of a model whose pairs lie next to each other: latency only
        _case("rotary_tokens_next", "rotary", 16, 0, 1, 32, 32, False, **_turns(pairs="next")),
        # gradients of a grouped-query model's rows that turn half of the head, stretched to four times their context: videos of odd lengths
        _case("rotary_part_inverse", "rotary", 8, 0, 8191, 28, 4, True, **_turns(axes=3, dim=64, stretch=4.0, inverse=True)),
        # every generated token of a batch, in every layer
        _case("turn_append_tokens", "append_turn", 16, 4096, 1, 32, 32, False, **_turns(axes=3), **_pages()),
        # chunks of unequal length of a grouped-query model in a text-salient layer, pairs next to each other, two bits
        _case("turn_append_chunks_gqa", "append_turn", 13, 3001, 1024, 28, 4, True, **_turns(pairs="next", stretch=8.0),
              **_pages(bits=2, G=64, mode="tsa")),
        # whole prompts of a batch, written at once
        _case("turn_append_prompts", "append_turn", 8, 0, 4096, 32, 32, False, **_turns(axes=3), **_pages(P=256)),
        # a few drafted tokens of every sequence, keys that come turned
        _case("append_drafts", "append", 24, 2100, 5, 32, 8, True, **_pages(G=64, mode="none", P=32)),
        # prompts of unequal length, keys that come turned
        _case("append_prompts", "append", 12, 0, 4095, 32, 32, True, **_pages(P=128)),
        # one user, one image, one generated token: the smallest call
        _case("attend_token_one", "attend", 1, 640, 1, 32, 32, False, **_pages(top_k=8)),
        # the ordinary batch of generated tokens, contexts of unequal length
        _case("attend_tokens", "attend", 16, 4096, 1, 32, 32, True, **_pages()),
        # generated tokens over long videos, grouped-query model
        _case("attend_tokens_video", "attend", 32, 32768, 1, 28, 4, False, **_pages(G=64, top_k=64, P=128)),
        # a few drafted tokens a sequence looked at in one call, in a text-salient layer: a seventh of the cached rows are 16-bit
        _case("attend_drafts_text", "attend", 4, 8191, 8, 32, 8, False, **_pages(mode="tsa", P=32)),
        # a chunk of long prompts over what is cached of them: the throughput case
        _case("attend_chunk", "attend", 4, 8192, 2048, 32, 32, False, **_pages(P=128)),
    ]


KINDS = ("rotary", "append_turn", "append", "attend")


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {k: {u: max(work(c)[u] for c in listed() if c["kind"] == k) for u in ("bytes", "flops")} for k in KINDS}
    while True:
        kind = rng.choice(["rotary", "append_turn", "append", "attend", "attend", "attend"])
        Hq, Hkv, G = rng.choice([(32, 32, 128), (32, 32, 128), (32, 32, 64), (40, 40, 128), (28, 4, 64), (32, 8, 128), (12, 2, 64)])
        ragged, B = rng.random() < 0.6, log_int(1, 32)
        turns = _turns(axes=rng.choice([1, 3]), pairs=rng.choice(["half", "next"]), dim=rng.choice([32, 64, 96, 128, 128, 128]),
                       stretch=rng.choice([1.0, 1.0, 4.0, 16.0]), inverse=kind == "rotary" and rng.random() < 0.4)
        T = 0 if rng.random() < 0.15 or kind == "rotary" else log_int(16, 32768)
        n = 1 if rng.random() < 0.3 else log_int(2, 8191 if kind == "rotary" else 4096)
        pages = _pages(bits=2 if kind == "append_turn" and rng.random() < 0.4 else 4, G=G, mode=rng.choice(["psa", "psa", "tsa", "none"]),
                       top_k=rng.choice([8, 16, 32, 64]), P=rng.choice([32, 64, 128, 256]))
        c = _case(None, kind, B, T, n, Hq, Hkv, ragged, **(turns if kind in ("rotary", "append_turn") else {}), **(pages if kind != "rotary" else {}))
        if sum(_rows(c)) == 0 or any(work(c)[u] > most[kind][u] for u in ("bytes", "flops")):
            continue
        if B * Hkv * (T + n) > 16 * 32 * 8192:  # caches within the listed ones
            continue
        if kind == "attend" and (T + n) * n * Hq > 32 * 4096 * 12288:  # scores of one sequence, held at once by the plain form
            continue
        return c


# ---------------------------------------------------------------------------------------------- sizes
def _spread(b):
    return 1.0 - 0.5 * ((b * 0.6180339887498949) % 1.0)


def _lens(c):
    """Cached rows of every sequence."""
    return [int(c["T"] * _spread(b)) if c["ragged"] else c["T"] for b in range(c["B"])]


def _rows(c):
    """New rows of every sequence; in a ragged call of several sequences the second has none."""
    if not c["ragged"]:
        return [c["n"]] * c["B"]
    return [0 if b == 1 else max(1, int(c["n"] * _spread(2 * b))) for b in range(c["B"])]


def _is_text(t):
    return t % (IMAGE + TEXT) < TEXT


def _salient_count(c, upto):
    if c["mode"] == "none":
        return 0
    if c["mode"] == "psa":
        return min(c["top_k"], upto)
    whole, rest = divmod(upto, IMAGE + TEXT)
    return whole * TEXT + min(rest, TEXT)


def work(case):
    c, rows = case, sum(_rows(case))
    turned = rows * (c["Hq"] + c["Hkv"]) * D
    if c["kind"] == "rotary":
        part = turned * c["dim"] // D
        return {"bytes": 4 * turned + 4 * c["axes"] * rows, "flops": 3 * part}
    row = 2 * (16 * c["bits"] + 4 * (D // c["G"]))  # codes and meta words of a key and a value
    if c["kind"] in ("append", "append_turn"):
        salient = sum(_salient_count(c, t + n) - _salient_count(c, t) for t, n in zip(_lens(c), _rows(c)) if c["mode"] == "tsa")
        w = {"bytes": rows * c["Hkv"] * (512 + row) + salient * c["Hkv"] * 512, "flops": 11 * 2 * rows * c["Hkv"] * D}
        if c["kind"] == "append_turn":  # queries in and out, turned keys out
            w = {"bytes": w["bytes"] + rows * (2 * c["Hq"] + c["Hkv"]) * 2 * D + 4 * c["axes"] * rows, "flops": w["flops"] + 3 * turned * c["dim"] // D}
        return w
    cached, pairs = 0, 0
    for t, n in zip(_lens(c), _rows(c)):
        if n:
            s = _salient_count(c, t)
            cached += (t - s) * row + s * 512
            pairs += n * t + n * (n + 1) // 2
    return {"bytes": c["Hkv"] * cached + rows * (2 * c["Hq"] + 2 * c["Hkv"]) * 2 * D, "flops": 4 * D * c["Hq"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _positions(c, g):
    """[axes, rows] int32: text counts up on every axis together; an image holds time and spreads height and width."""
    parts = []
    for b, n in enumerate(_rows(c)):
        first = int(torch.randint(0, 1 << (20 if b % 4 == 3 else 14), (1,), generator=g, device="cuda"))
        t = torch.arange(n, device="cuda")
        period, r = t // (IMAGE + TEXT), t % (IMAGE + TEXT)
        base = first + period * (TEXT + 24)
        text, at = r < TEXT, (r - TEXT).clamp(min=0)
        axes = [base + torch.where(text, r, TEXT + x) for x in (torch.zeros_like(at), at // 24, at % 24)]
        parts.append(torch.stack(axes[: c["axes"]]))
    return torch.cat(parts, dim=1).int()


def _frequencies(c):
    """(frequencies in 32 bits, axes of the pairs, magnitude): of a context stretched s times, frequencies that turn less than once in
    the trained context of 4096 are divided by s, those that turn more than 32 times stay, and what lies between is blended."""
    base, half, s = (1e6 if c["Hq"] != c["Hkv"] else 1e4), c["dim"] // 2, c["stretch"]
    f = base ** (-torch.arange(half, dtype=torch.float64) / half)
    keep = ((4096 * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
    f = (f * keep + f / s * (1 - keep)).float()
    first = torch.arange(half) * 64 // half  # of three axes time has a quarter of the pairs, height and width share the rest
    axis = torch.zeros(half, dtype=torch.int64) if c["axes"] == 1 else (first >= 16).long() + (first >= 40).long()
    return f, axis, 0.1 * math.log(s) + 1.0


def _projection(c, g):
    """Rows of a fused projection [rows, Hq + 2 Hkv, 128] binary16; a few key channels of every head are large."""
    rows, Hq, Hkv = sum(_rows(c)), c["Hq"], c["Hkv"]
    x = torch.randn(rows, Hq + 2 * Hkv, D, generator=g, device="cuda", dtype=torch.float16)
    x[:, Hq:Hq + Hkv] *= _gain(c)
    return x


def _gain(c):
    """[Hkv, 128]: four outlier channels a head, the same for cached and new rows."""
    h = torch.Generator().manual_seed(250115 + c["Hkv"])
    gain = torch.ones(c["Hkv"], D)
    for k in range(c["Hkv"]):
        gain[k, torch.randperm(D, generator=h)[:4]] = 20.0
    return gain.half().cuda()


def _inputs(c, seed):
    """Everything a call gets, as plain tensors."""
    g = _generator(seed)
    d = {"x": _projection(c, g)}
    if c["kind"] in ("rotary", "append_turn"):
        d["pos"] = _positions(c, g)
    if c["kind"] == "rotary":
        return d
    lens, rows, B, Hkv, P, G, bits = _lens(c), _rows(c), c["B"], c["Hkv"], c["P"], c["G"], c["bits"]
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    d["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    d["seq_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # pages: those that cached and new rows need, in no order, a few more in the pool
    need = [(t + n + P - 1) // P for t, n in zip(lens, rows)]
    max_pages, n_pages = max(max(need), 1), sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, : need[b]] = order[at:at + need[b]]
        at += need[b]
    d["table"] = table
    # salient lists: final for the cached and the new rows
    totals = [t + n for t, n in zip(lens, rows)]
    S_cap = max(64, (max(_salient_count(c, t) for t in totals) + 63) // 64 * 64)
    d["sal_idx"] = torch.full((B, Hkv, S_cap), -1, dtype=torch.int32, device="cuda")
    d["sal_cnt"] = torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")
    for b, total in enumerate(totals):
        k = _salient_count(c, total)
        if k == 0:
            continue
        if c["mode"] == "tsa":
            t = torch.arange(total, device="cuda")
            at = t[_is_text(t)].expand(Hkv, k)
        else:
            at = torch.rand(Hkv, total, generator=g, device="cuda").topk(k, dim=1).indices.sort(dim=1).values
        d["sal_idx"][b, :, :k] = at.int()
        d["sal_cnt"][b] = k
    # the pools, filled with the sequences' cached rows
    d["k_codes"] = torch.zeros(n_pages, Hkv, P // 32, 128 * bits, dtype=torch.int32, device="cuda")
    d["v_codes"] = torch.zeros_like(d["k_codes"])
    d["k_meta"] = torch.zeros(n_pages, Hkv, P, D // G, dtype=torch.int32, device="cuda")
    d["v_meta"] = torch.zeros_like(d["k_meta"])
    d["k_sal"] = torch.zeros(B, Hkv, S_cap, D, dtype=torch.bfloat16, device="cuda")
    d["v_sal"] = torch.zeros(B, Hkv, S_cap // 32, 4096, dtype=torch.bfloat16, device="cuda")
    for b, t in enumerate(lens):
        if t:
            k = torch.randn(Hkv, t, D, generator=g, device="cuda").half() * _gain(c)[:, None]
            k[:, :: max(t // 4, 1)] *= 10.0  # a few rows of large norm
            _plain_append(c, d, b, 0, k, torch.randn(Hkv, t, D, generator=g, device="cuda").half())
    return d


POOLS = ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")


def prepare(case, seed):
    c = case
    s = {"c": c, **_inputs(c, seed)}
    Hq, Hkv, x = c["Hq"], c["Hkv"], s["x"]
    s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if c["kind"] != "rotary":
        s["starts"], s["lens"] = s["row_start"].tolist(), s["seq_len"].tolist()
    if "pos" in s:
        f, axis, magnitude = _frequencies(c)
        s["f"], s["axis"], s["magnitude"] = f.cuda(), axis.cuda(), magnitude
    if own:
        from paper_2501_15021_amd import binding as akvq
        s["akvq"] = akvq
        if "pos" in s:
            s["rotary"] = akvq.Rotary(f.tolist(), axis.tolist(), dim=c["dim"], interleaved=c["pairs"] == "next", magnitude=magnitude)
        if c["kind"] != "rotary":
            cache = akvq.PagedCache(c["B"], Hkv, c["G"], s["k_codes"].shape[0], s["table"].shape[1], page_rows=c["P"], S_cap=s["sal_idx"].shape[2],
                                    bits=c["bits"])
            for name in ("k_codes", "v_codes", "k_meta", "v_meta", "table", "seq_len", "sal_idx"):
                getattr(cache, name).copy_(s[name])
            cache.counts().copy_(s["sal_cnt"])
            cache.k_sal.copy_(s["k_sal"].view(torch.int16))
            cache.v_sal.copy_(s["v_sal"].view(torch.int16))
            cache.max_len = c["T"]  # what the server knows of the longest sequence
            s["cache"] = cache
            for name in POOLS:
                del s[name]
    return s


# ---------------------------------------------------------------------------------------------- the pass
def run(state):
    s, c = state, state["c"]
    if not own:
        return {"rotary": _plain_rotary, "append_turn": _plain_append_turn, "append": _plain_append_all, "attend": _plain_attend}[c["kind"]](s)
    akvq = s["akvq"]
    if c["kind"] == "rotary":
        q, k = akvq.rotary_rows(s["rotary"], s["pos"], s["q"], s["k"], inverse=c["inverse"])
        return {"q": q, "k": k}
    cache, out = s["cache"], {}
    if c["kind"] == "attend":
        return {"out": akvq.paged_attention(cache, s["q"], s["k"], s["v"], s["row_start"], c["n"], SCALE)}
    if c["kind"] == "append_turn":
        out["q"], out["k"] = akvq.paged_append_rotary(cache, s["rotary"], s["pos"], s["q"], s["k"], s["v"], s["row_start"], c["n"], CLIP[c["bits"]])
    else:
        akvq.paged_append(cache, s["k"], s["v"], s["row_start"], c["n"], CLIP[c["bits"]])
    return {**out, "k_codes": cache.k_codes, "v_codes": cache.v_codes, "k_meta": cache.k_meta, "v_meta": cache.v_meta,
            "k_sal": cache.k_sal.view(torch.bfloat16), "v_sal": cache.v_sal.view(torch.bfloat16)}


# ---------------------------------------------------------------------------------------------- plain forms
def _turn_table(s, inverse):
    """Cosine and sine of every row and pair times the magnitude [rows, 1, pairs], 32 bits each: far positions need an angle of 64 bits."""
    angle = s["pos"].double()[s["axis"]].t() * s["f"].double()
    cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * s["magnitude"]).float()[:, None]
    return cos, -sin if inverse else sin


def _fma(x, c, t):
    """x c + t rounded once to 32 bits (the product of 11 and 24 bits is exact in 64), as what follows rounds next to a border."""
    return (x.double() * c.double() + t.double()).float()


def _turn(c, x, cos, sin):
    """Rows [rows, heads, 128] turned: one product rounded to 32 bits, its sum with the other one once, and that to binary16."""
    dim, half = c["dim"], c["dim"] // 2
    a, b = (x[..., :half], x[..., half:dim]) if c["pairs"] == "half" else (x[..., 0:dim:2], x[..., 1:dim:2])
    a2, b2 = _fma(a, cos, -(b.float() * sin)).half(), _fma(b, cos, a.float() * sin).half()
    turned = torch.cat((a2, b2), -1) if c["pairs"] == "half" else torch.stack((a2, b2), -1).flatten(-2)
    return torch.cat((turned, x[..., dim:]), -1)


def _plain_rotary(s):
    cos, sin = _turn_table(s, s["c"]["inverse"])
    return {"q": _turn(s["c"], s["q"], cos, sin), "k": _turn(s["c"], s["k"], cos, sin)}


def _butterflies(x):
    """128-point Walsh-Hadamard transform without its factor, strides 1 to 64, every sum rounded to x's type."""
    h = 1
    while h < D:
        y = x.reshape(*x.shape[:-1], D // (2 * h), 2, h)
        a, b = y[..., 0, :], y[..., 1, :]
        x = torch.stack((a + b, a - b), dim=-2).reshape(x.shape)
        h *= 2
    return x


KAPPA = 0.08838834613561630                       # 2^-3.5 in binary32
LEVELS = {2: 0.3333333432674408, 4: 0.06666667014360428}  # 1/3 and 1/15 in binary32


def _quantize(x, G, bits):
    """Rows [..., 128] binary16 -> (codes [..., 128], meta words [..., 128/G], rotated rows bfloat16): scale and zero-point a group from
    its clipped extrema, the scale rounded up to binary16, codes of the sum x / scale + zero rounded once."""
    u = _butterflies(x.float())
    ug = u.reshape(*u.shape[:-1], D // G, G)
    clip = torch.tensor(CLIP[bits], dtype=torch.float32, device=x.device)
    lo, hi = (ug.amin(-1) * KAPPA) * clip, (ug.amax(-1) * KAPPA) * clip
    want = (hi - lo) * LEVELS[bits]
    up = want.half().view(torch.int16).int()
    up = torch.where(want.half().float() < want, up + 1, up).clamp(max=0x7BFF)
    up = torch.where(want > 0, up, torch.full_like(up, 0x3C00))
    scale = up.short().view(torch.float16).float()
    r = (1.0 / scale.double()).float()
    zero = (-torch.round(lo * r)).clamp(-32768, 32767)
    t = ug.double() * (r * KAPPA).double()[..., None] + zero.double()[..., None]
    code = torch.round(t).clamp(0, 2 ** bits - 1).int().reshape(x.shape)
    meta = up | ((zero.int() & 0xFFFF) << 16)
    return code, meta, (u * KAPPA + 0.0).bfloat16()


def _pack(code, bits, value):
    """Codes [..., 32, 128] of a block -> its 128 * bits words, of keys or of values."""
    at = [torch.arange(k, device=code.device) for k in range(9)]
    y = code.long()
    if not value and bits == 2:
        y = y.reshape(-1, 2, 16, 2, 2, 4, 8).permute(0, 5, 2, 1, 3, 4, 6)      # j, n, half, m/2 | m%2, i
        shift = 2 * (8 * at[2][:, None] + at[8])
    elif not value:
        y = y.reshape(-1, 2, 16, 4, 4, 8).permute(0, 1, 4, 2, 3, 5)            # half, j, n, m | i
        shift = 4 * at[8]
    elif bits == 2:
        y = y.reshape(-1, 2, 4, 4, 2, 2, 2, 16).permute(0, 2, 7, 6, 4, 1, 5, 3)  # q, n, nb%2, nb/4 | half, (nb/2)%2, ii
        shift = 16 * at[2][:, None, None] + 2 * (4 * at[2][:, None] + at[4])
    else:
        y = y.reshape(-1, 2, 4, 4, 4, 2, 16).permute(0, 5, 2, 6, 4, 1, 3)      # nb%2, q, n, nb/2 | half, ii
        shift = 16 * at[2][:, None] + 4 * at[4]
    return (y << shift).flatten(-shift.dim()).sum(-1).int().reshape(*code.shape[:-2], 128 * bits)


def _unpack4(words, value):
    """4-bit codes [..., 32, 128] of a block's 512 words."""
    at = [torch.arange(k, device=words.device) for k in range(9)]
    if value:
        y = words.reshape(-1, 2, 4, 16, 4, 1, 1) >> (16 * at[2][:, None] + 4 * at[4])
        y = y.permute(0, 5, 2, 6, 4, 1, 3)
    else:
        y = (words.reshape(-1, 2, 4, 16, 4, 1) >> (4 * at[8])).permute(0, 1, 3, 4, 2, 5)
    return (y & 15).reshape(*words.shape[:-1], 32, D)


def _overlay_rows(tiles):
    """Value tiles [Hkv, S_cap/32, 4096] as a view whose last axes are (slot of the tile as three, channel as two)."""
    Hkv, n, _ = tiles.shape
    return tiles.reshape(Hkv, n, 8, 4, 16, 4, 2).permute(0, 1, 6, 3, 5, 2, 4)


def _plain_append(c, d, b, first, k, v):
    """Rows k, v [Hkv, n, 128] become cache rows first, first + 1, ... of sequence b."""
    Hkv, n, _ = k.shape
    P, S_cap, bits = c["P"], d["sal_idx"].shape[2], c["bits"]
    blk0, blk1 = first // 32, (first + n + 31) // 32
    pad = first - 32 * blk0, 32 * blk1 - first - n
    blocks = torch.arange(blk0, blk1, device="cuda")
    page, inside = d["table"][b].long()[blocks * 32 // P], blocks % (P // 32)
    t = torch.arange(first, first + n, device="cuda")
    row_page, row = d["table"][b].long()[t // P], t % P
    listed = d["sal_idx"][b].long()
    slot = torch.arange(S_cap, device="cuda").expand(Hkv, S_cap)
    mine = (slot < d["sal_cnt"][b][:, None]) & (listed >= first) & (listed < first + n)
    salient = torch.zeros(Hkv, n, dtype=torch.int32, device="cuda")
    head = torch.arange(Hkv, device="cuda")[:, None].expand(Hkv, S_cap)
    salient[head[mine], listed[mine] - first] = 0x8000
    new = torch.nn.functional.pad(torch.full((Hkv, n, D), 2 ** bits - 1, dtype=torch.int32, device="cuda"), (0, 0, *pad)).reshape(Hkv, -1, 32, D)
    for x, codes, metas, value, name in ((k, "k_codes", "k_meta", False, "k_sal"), (v, "v_codes", "v_meta", True, "v_sal")):
        code, meta, wide = _quantize(x, c["G"], bits)
        code = torch.nn.functional.pad(code, (0, 0, *pad)).reshape(Hkv, -1, 32, D)
        words, mask = _pack(code, bits, value).transpose(0, 1), _pack(new, bits, value).transpose(0, 1)
        d[codes][page, :, inside] = (d[codes][page, :, inside] & ~mask) | words
        d[metas][row_page, :, row] = (meta | salient[..., None]).transpose(0, 1)
        rows = wide[head[mine], listed[mine] - first]
        if not value:
            d[name][b][mine] = rows
        else:
            tiles = _overlay_rows(d[name][b])
            flat = tiles.reshape(Hkv, S_cap, D).clone()
            flat[mine] = rows
            tiles.copy_(flat.reshape(tiles.shape))


def _plain_append_all(s):
    c = s["c"]
    for b, first in enumerate(s["lens"]):
        lo, hi = s["starts"][b], s["starts"][b + 1]
        if hi > lo:
            _plain_append(c, s, b, first, s["k"][lo:hi].transpose(0, 1), s["v"][lo:hi].transpose(0, 1))
    return {name: s[name] for name in POOLS}


def _plain_append_turn(s):
    cos, sin = _turn_table(s, False)
    q, k = _turn(s["c"], s["q"], cos, sin), _turn(s["c"], s["k"], cos, sin)
    return {"q": q, "k": k, **_plain_append_all({**s, "k": k})}


def _read_cache(c, d, b, t):
    """Cached rows of sequence b as 32-bit numbers, rotated: (k, v) [Hkv, t, 128]."""
    Hkv, P, G = c["Hkv"], c["P"], c["G"]
    blocks = torch.arange((t + 31) // 32, device="cuda")
    page, inside = d["table"][b].long()[blocks * 32 // P], blocks % (P // 32)
    row = torch.arange(t, device="cuda")
    row_page, row = d["table"][b].long()[row // P], row % P
    S_cap = d["sal_idx"].shape[2]
    listed = d["sal_idx"][b].long()
    slot = torch.arange(S_cap, device="cuda").expand(Hkv, S_cap)
    mine = (slot < d["sal_cnt"][b][:, None]) & (listed < t)
    head = torch.arange(Hkv, device="cuda")[:, None].expand(Hkv, S_cap)
    v_rows = _overlay_rows(d["v_sal"][b]).reshape(Hkv, S_cap, D)
    out = []
    for codes, metas, value, wide in (("k_codes", "k_meta", False, d["k_sal"][b]), ("v_codes", "v_meta", True, v_rows)):
        code = _unpack4(d[codes][page, :, inside].transpose(0, 1), value).reshape(Hkv, -1, D)[:, :t]
        meta = d[metas][row_page, :, row].transpose(0, 1)
        scale = (meta & 0x7FFF).short().view(torch.float16).float()[..., None]
        x = (scale * (code.reshape(Hkv, t, D // G, G) - (meta >> 16)[..., None]).float()).reshape(Hkv, t, D)
        x[head[mine], listed[mine]] = wide[mine].float()
        out.append(x)
    return out


def _plain_attend(s):
    c = s["c"]
    Hkv, R = c["Hkv"], c["Hq"] // c["Hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float16, device="cuda")
    for b, t in enumerate(s["lens"]):
        lo, hi = s["starts"][b], s["starts"][b + 1]
        n = hi - lo
        if n == 0:
            continue
        q = s["q"][lo:hi].float().reshape(n, Hkv, R, D).permute(1, 0, 2, 3).reshape(Hkv, n * R, D)  # rows: token, head of the group
        k, v = (s[x][lo:hi].float().transpose(0, 1).contiguous() for x in "kv")
        ahead = torch.arange(n, device="cuda")[None, :] > torch.arange(n, device="cuda").repeat_interleave(R)[:, None]
        scores = torch.matmul(q, k.transpose(1, 2).contiguous()).masked_fill(ahead, -math.inf)
        if t:
            kc, vc = _read_cache(c, s, b, t)
            scores = torch.cat((torch.matmul(_butterflies(q) * KAPPA, kc.transpose(1, 2).contiguous()), scores), dim=-1)
        scores *= SCALE
        p = torch.exp(scores - scores.amax(-1, keepdim=True))
        p /= p.sum(-1, keepdim=True)
        o = torch.matmul(p[..., t:], v)
        if t:
            o += _butterflies(torch.matmul(p[..., :t], vc)) * KAPPA
        out[lo:hi] = o.reshape(Hkv, n, R, D).permute(1, 0, 2, 3).reshape(n, c["Hq"], D).half()
    return {"out": out}


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _hadamard64():
    h = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    for _ in range(7):
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h / math.sqrt(D)


def _slots_of_block():
    """Where the 4-bit code of (row, channel) lies in a block's 512 words: word and lowest bit, for keys and for values [32, 128]."""
    kw, kb, vw, vb = ([[0] * D for _ in range(32)] for _ in range(4))
    for r in range(32):
        for e in range(D):
            kw[r][e], kb[r][e] = r // 16 * 256 + (16 * (e % 32 // 8) + r % 16) * 4 + e // 32, 4 * (e % 8)
            vw[r][e], vb[r][e] = e // 16 % 2 * 256 + (16 * (r % 16 // 4) + e % 16) * 4 + e // 32, 16 * (r // 16) + 4 * (r % 4)
    return [torch.tensor(x, device="cuda") for x in (kw, kb, vw, vb)]


def _overlay_at(slots):
    """Where (slot, channel) lies in a head's value tiles [slots, 128]."""
    s, e = slots[:, None], torch.arange(D, device="cuda")
    r = s % 32 % 16
    return s // 32 * 4096 + e // 16 * 512 + (16 * (r // 4) + e % 16) * 8 + 2 * (r % 4) + s % 32 // 16


def _turned64(c, d):
    """Queries and keys of a chunk, turned, as complex products a pair."""
    f, axis, magnitude = _frequencies(c)
    f, out = f.double().cuda(), []
    for lo, hi in ((0, c["Hq"]), (c["Hq"], c["Hq"] + c["Hkv"])):
        y = d["x"][:, lo:hi].double()
        for i in range(c["dim"] // 2):
            a = d["pos"][int(axis[i])].double() * f[i] * (-1.0 if c["inverse"] else 1.0)
            one, two = (i, i + c["dim"] // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
            z = torch.complex(y[..., one], y[..., two]) * torch.polar(torch.full_like(a, magnitude), a)[:, None]
            y[..., one], y[..., two] = z.real, z.imag
        out.append(y)
    return out


def _exact_append(c, d, k):
    """The 16-bit rows (codes and their meta words are whole numbers); k: turned keys."""
    H, Hkv = _hadamard64(), c["Hkv"]
    k_sal, v_sal = d["k_sal"].double(), d["v_sal"].double()
    starts, lens, v = d["row_start"].tolist(), d["seq_len"].tolist(), d["x"][:, c["Hq"] + Hkv:]
    flat, at = v_sal.reshape(c["B"], Hkv, -1), _overlay_at(torch.arange(k_sal.shape[2], device="cuda"))
    for b in range(c["B"]):
        lo, n = starts[b], starts[b + 1] - starts[b]
        for h in range(Hkv if n else 0):
            idx = d["sal_idx"][b, h, : int(d["sal_cnt"][b, h])].long() - lens[b]
            slots = torch.nonzero((idx >= 0) & (idx < n)).flatten()
            if slots.numel():
                k_sal[b, h, slots] = k[lo + idx[slots], h].double() @ H
                flat[b, h, at[slots]] = v[lo + idx[slots], h].double() @ H
    return {"k_codes": None, "v_codes": None, "k_meta": None, "v_meta": None, "k_sal": k_sal, "v_sal": v_sal}


def _exact_attend(c, d):
    H, Hq, Hkv, P, NG = _hadamard64(), c["Hq"], c["Hkv"], c["P"], D // c["G"]
    R = Hq // Hkv
    kw, kb, vw, vb = _slots_of_block()
    starts, lens = d["row_start"].tolist(), d["seq_len"].tolist()
    out = torch.empty(starts[-1], Hq, D, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        lo, hi, t = starts[b], starts[b + 1], lens[b]
        n = hi - lo
        if n == 0:
            continue
        at = torch.arange(t, device="cuda")
        page, in_page = d["table"][b].long()[at // P], at % P
        causal = torch.arange(n, device="cuda")[:, None] >= torch.arange(n, device="cuda")[None, :]
        for h in range(Hkv):
            keys, values = [], []
            if t:
                for words, bits, codes, metas, into in ((kw, kb, d["k_codes"], d["k_meta"], keys), (vw, vb, d["v_codes"], d["v_meta"], values)):
                    block = codes[page, h, in_page // 32]  # [t, 512]: the block that holds the row
                    code = (torch.gather(block, 1, words[in_page % 32]) >> bits[in_page % 32]) & 15
                    meta = metas[page, h, in_page].repeat_interleave(D // NG, dim=1)
                    x = (meta & 0x7FFF).short().view(torch.float16).double() * (code - (meta >> 16)).double()
                    idx = d["sal_idx"][b, h, : int(d["sal_cnt"][b, h])].long()
                    slots = torch.nonzero(idx < t).flatten()
                    if into is keys:
                        x[idx[slots]] = d["k_sal"][b, h, slots].double()
                    else:
                        x[idx[slots]] = d["v_sal"][b, h].flatten()[_overlay_at(slots)].double()
                    into.append(x @ H)
            keys.append(d["x"][lo:hi, Hq + h].double())
            values.append(d["x"][lo:hi, Hq + Hkv + h].double())
            keys, values = torch.cat(keys), torch.cat(values)
            seen = torch.cat((torch.ones(n, t, dtype=torch.bool, device="cuda"), causal), dim=1)
            for r in range(h * R, (h + 1) * R):
                s = d["x"][lo:hi, r].double() @ keys.t().contiguous() * SCALE
                out[lo:hi, r] = torch.softmax(s.masked_fill(~seen, -math.inf), dim=1) @ values
    return {"out": out}


def exact(case, seed):
    c, d = case, _inputs(case, seed)
    if c["kind"] == "attend":
        return _exact_attend(c, d)
    if c["kind"] == "append":
        return _exact_append(c, d, d["x"][:, c["Hq"]:c["Hq"] + c["Hkv"]])
    q, k = _turned64(c, d)
    return {"q": q, "k": k, **(_exact_append(c, d, k) if c["kind"] == "append_turn" else {})}
