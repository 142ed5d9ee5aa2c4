"""Attention of a chunk over pages and over itself (akvq_paged_attention) against the formula in 64 bits on what the pages hold."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, attention64, check_attention

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700, 1001, 1500]


def _run(s, n_split=0, flags=0, sm=SM, **kw):
    out = torch.full((s.x.shape[0], s.Hq, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((s.x.shape[0], s.Hq), 7.0, device="cuda")
    akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, sm, n_split=n_split, flags=flags, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("lens,rows,Hq,Hkv,page_rows", [
    ([0], [1], 1, 1, 64), ([1], [1], 2, 2, 32), ([31, 32, 33], [1, 1, 1], 7, 1, 64), ([640], [1], 4, 4, 64), ([1000, 3], [1, 1], 8, 1, 128),
    ([0, 64, 65], [5, 16, 1], 3, 3, 32), ([100, 0], [8, 2], 28, 4, 64), ([700], [17], 2, 2, 64), ([5, 1601], [33, 64], 2, 1, 256),
    ([0], [65], 1, 1, 64), ([130], [129], 4, 2, 32), ([0, 300], [200, 0], 6, 1, 64), ([513, 64, 0, 2], [70, 1, 33, 100], 8, 2, 64),
    ([96], [257], 2, 2, 64), ([1234], [3], 16, 2, 64)])
def test_against_the_formula(lens, rows, Hq, Hkv, page_rows, G):
    s = Sequences(lens, rows, Hkv, G, page_rows, Hq=Hq, salient=SALIENT, seed=sum(lens) + sum(rows)).fill_pages()
    for n_split in (1, 0, 3, 7):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM, f"n_split {n_split}")


@pytest.mark.parametrize("lens,rows,Hq,Hkv", [
    ([70, 3, 0, 200, 33, 64, 1, 150, 90], [1, 1, 1, 1, 0, 1, 1, 1, 1], 32, 32),                 # more units than CUs: paired on them
    ([(37 * b) % 101 for b in range(65)], [b % 2 for b in range(65)], 8, 8),                    # more sequences than lanes
    ([5, 300, 0, 300, 64, 20], [70, 65, 129, 1, 0, 300], 2, 2),                                 # unequal chunks, the longest first
    ([(37 * b) % 101 for b in range(66)], [66 if b % 8 == 0 else b % 3 for b in range(66)], 1, 1)])
def test_the_order_of_unequal_sequences(lens, rows, Hq, Hkv):
    """Which sequence a workgroup takes depends on all lengths: every row is still written once, with its own result."""
    s = Sequences(lens, rows, Hkv, 128, 32, Hq=Hq, salient=SALIENT, seed=len(lens)).fill_pages()
    for n_split in (1, 2):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM, f"n_split {n_split}")


@pytest.mark.parametrize("lens,rows,Hq,Hkv", [
    ([100, 1000], [17, 32], 2, 2), ([40, 0, 333], [4, 3, 1], 28, 4),           # two tiles of 16 rows
    ([0, 500], [300, 260], 3, 3), ([0], [1100], 2, 1), ([64, 3], [70, 513], 8, 1),  # tiles of 32 of long chunks
    ([17000], [40], 4, 1), ([5000, 0, 200], [600, 2900, 1], 1, 1)])             # tiles of 256
def test_tiles_of_every_size(lens, rows, Hq, Hkv):
    s = Sequences(lens, rows, Hkv, 64, 64, Hq=Hq, salient=SALIENT, seed=sum(rows)).fill_pages()
    for n_split in (0, 1, 3):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM, f"n_split {n_split}")


@pytest.mark.parametrize("rows", [1, 20, 70])
@pytest.mark.parametrize("length,page_rows", [(2040, 32), (4070, 32), (4200, 32), (9000, 32), (20000, 64), (11000, 1024)])
def test_tables_of_every_length(length, page_rows, rows):
    """Page numbers come 64 at a time: tables of up to 64 pages, of up to 128, and longer ones, begun anywhere."""
    s = Sequences([length, 100], [rows, 1], 1, 128, page_rows, Hq=2, salient=SALIENT, seed=length).fill_pages()
    for n_split in (1, 2, 9):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM, f"n_split {n_split}")


def test_default_splits_of_the_callers_bound():
    """The library's choice is that of the max_rows it is given, also where fewer rows come: a workspace of that size serves them."""
    s = Sequences([3000, 40], [1, 0], 2, 128, Hq=4, salient=SALIENT, seed=2).fill_pages()
    L, c = akvq.lib(), s.cache.paged_struct()
    for max_rows in (1, 9, 200, 5000):
        n = L.akvq_paged_default_splits(C.byref(c), 4, max_rows)
        nws = L.akvq_paged_workspace_bytes(s.n, 4, n)
        ws = torch.empty(max(nws, 16), dtype=torch.uint8, device="cuda")
        out = torch.empty(s.n, 4, 128, dtype=torch.float16, device="cuda")
        chunk = akvq.akvq_chunk(s.row_start.data_ptr(), s.n, max_rows)
        assert L.akvq_paged_attention(C.byref(c), C.byref(chunk), s.q.data_ptr(), s.q.stride(0), 4, s.k.data_ptr(), s.k.stride(0), s.v.data_ptr(),
                                      s.v.stride(0), SM, out.data_ptr(), 512, None, 0, ws.data_ptr(), nws, 0, None) == 0
        torch.cuda.synchronize()
        check_attention(s, out, None, SM, f"max_rows {max_rows}")


@pytest.mark.parametrize("n_split", [16, 17, 33, 64, 130])
@pytest.mark.parametrize("rows", [1, 20, 70])
def test_many_splits(n_split, rows):
    """More splits than the merge takes at a time, and more than there are blocks."""
    s = Sequences([700, 20], [rows, 1], 2, 64, Hq=4, salient=SALIENT, seed=n_split).fill_pages()
    out, lse = _run(s, n_split)
    check_attention(s, out, lse, SM)


@pytest.mark.parametrize("salient", [[], range(0, 500), range(1, 500, 2), [499]])
@pytest.mark.parametrize("rows", [1, 40, 150])
def test_few_and_many_16_bit_rows(salient, rows):
    """All rows in the overlay, none, every second one; and lists that are already final for the chunk's own rows."""
    s = Sequences([300, 200, 0], [rows, rows, rows], 2, 128, Hq=4, salient=salient, seed=rows).fill_pages()
    for n_split in (1, 5):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM)


def test_rows_of_no_sequence_and_views_stay():
    """Rows behind the last sequence are left alone, split or not; out may be part of longer rows."""
    s = Sequences([50, 0, 9], [6, 3, 1], 2, 128, Hq=4, extra_rows=4).fill_pages()
    for n_split in (1, 2):
        wide = torch.full((14, 9, 128), 3.0, dtype=torch.float16, device="cuda")
        akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, SM, n_split=n_split, out=wide[:, 2:6])
        torch.cuda.synchronize()
        check_attention(s, wide[:, 2:6], None, SM)
        assert bool((wide[10:] == 3).all() and (wide[:, :2] == 3).all() and (wide[:, 6:] == 3).all())


def test_rows_without_a_page_take_no_part():
    s = Sequences([300, 64, 90], [40, 1, 2], 2, 128, Hq=4, salient=[70, 290]).fill_pages()
    s.cache.table[0, 1] = -1
    s.cache.table[0, 3] = s.cache.n_pages
    s.cache.table[1, 0] = 1 << 30   # all that is cached of it
    s.cache.table[2, 1] = -7
    for n_split in (1, 3):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM)


@pytest.mark.parametrize("rows", [1, 3, 140])
def test_what_takes_no_part_may_hold_anything(rows):
    """NaN in other sequences' rows, unused pages, rows behind the length, unused overlay slots, and rows behind the chunk."""
    make = lambda: Sequences([77, 45, 100], [rows, 2, rows], 2, 64, Hq=4, salient=[5, 70, 80], extra_rows=70, seed=4).fill_pages()
    s, clean = make(), make()
    p = s.cache
    pools = (p.k_codes, p.v_codes, p.k_meta, p.v_meta)
    used = {}
    for b in range(3):
        for i, page in enumerate(p.table[b].tolist()):
            if page >= 0:
                used[page] = min(max(s.lens[b] - i * p.page_rows, 0), p.page_rows)
    for page in range(p.n_pages):
        for t in (p.k_meta, p.v_meta):
            t[page, :, used.get(page, 0):] = 0x7E007E00   # scale NaN
        if page not in used:
            for t in pools:
                t[page] = -1
    for b in range(3):
        k = sum(1 for x in (5, 70, 80) if x < s.lens[b])
        p.k_sal[b, :, k:] = 0x7FC0
        tiles = p.v_sal[b].reshape(2, -1, 8, 4, 16, 4, 2).permute(0, 1, 6, 3, 5, 2, 4)
        flat = tiles.reshape(2, p.S_cap, 128).clone()
        flat[:, k:] = 0x7FC0
        tiles.copy_(flat.reshape(tiles.shape))
    s.x[s.n:] = float("nan")
    s.x[s.starts[1]:s.starts[2]] = float("nan")     # all of sequence 1's rows
    for n_split in (1, 4):
        got, want = _run(s, n_split), _run(clean, n_split)
        for b in (0, 2):
            lo, hi = s.starts[b], s.starts[b + 1]
            assert torch.equal(got[0][lo:hi], want[0][lo:hi]) and torch.equal(got[1][lo:hi], want[1][lo:hi]), (n_split, b)
    clean.x[clean.starts[2]:clean.n, 0] = float("nan")  # one head's queries: the other heads', and the other sequences', stay
    got = _run(clean, 4)
    for x, y in zip(got, want):
        assert torch.equal(x[clean.starts[2]:clean.n, 1:], y[clean.starts[2]:clean.n, 1:])
        assert torch.equal(x[:clean.starts[2]], y[:clean.starts[2]])


@pytest.mark.parametrize("rows", [1, 50])
def test_large_scores_and_offsets(rows):
    """Scores of hundreds (the reference is raised again and again, and one row decides), rising and falling along the keys; value
    rows of very different sizes; and unrotated groups far from zero, whose zero-points pass 11 bits."""
    for order in (1, -1):
        s = Sequences([400], [rows], 2, 128, Hq=4, gain=1.0, seed=rows)
        k, v = s.past[0]
        ramp = torch.linspace(0.1, 30, 400, device="cuda")[:: order] if order == 1 else torch.linspace(30, 0.1, 400, device="cuda")
        k *= ramp[None, :, None].half()
        v *= (10.0 ** torch.linspace(-3, 3, 400, device="cuda"))[None, :, None].half()
        s.fill_pages()
        for n_split in (1, 3):
            out, lse = _run(s, n_split)
            check_attention(s, out, lse, SM)
    # Channels near 20: zero-points past 1024, where a zero-point is summed in two parts.  |zero * scale| and |code * scale| cancel: 32-bit
    # sums of terms of 20 a channel, which the bound's |q| |k| counts (|k| is 20 * 128 ** 0.5).
    for width, least in ((0.01, 1024), (0.002, 2048)):
        far = Sequences([300], [rows], 2, 128, Hq=4, gain=1.0, seed=9)
        for x in far.past[0]:
            x.mul_(width).add_(20.0)
        far.fill_pages(clip=1.0, flags=akvq.K_PREROTATED | akvq.V_PREROTATED)
        assert int((far.cache.v_meta >> 16).abs().max()) > least
        for n_split in (1, 3):
            out, lse = _run(far, n_split)
            check_attention(far, out, lse, SM)


def test_rotated_inputs_and_outputs():
    """q, k and v of the chunk rotated by the caller, out left rotated: the same result, rotated."""
    s = Sequences([200, 30], [20, 70], 2, 64, Hq=4, salient=[3, 100]).fill_pages()
    want = [attention64(s, b, SM)[0] for b in range(2)]

    def turned(x):
        y, h = x.double(), 1
        for _ in range(7):
            z = y.reshape(*y.shape[:-1], 64 // h, 2, h)
            y = torch.stack((z[..., 0, :] + z[..., 1, :], z[..., 0, :] - z[..., 1, :]), -2).reshape(y.shape)
            h *= 2
        return y / 128 ** 0.5

    qkv = turned(s.x).half()
    for n_split in (1, 3):
        out = akvq.paged_attention(s.cache, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], s.row_start, s.max_rows, SM, n_split=n_split,
                                   flags=akvq.Q_PREROTATED | akvq.OUT_ROTATED)
        torch.cuda.synchronize()
        for b in range(2):
            lo, hi = s.starts[b], s.starts[b + 1]
            err = (turned(out[lo:hi]) - want[b]).norm(dim=2) / want[b].norm(dim=2)
            # inputs rounded to binary16 once more: 2^-11 of q, k and v each, so 2^-10 |q| |k| SM of a score, |q| 11, |k| 14 with its large channel
            assert float(err.max()) < 2 * 2.0 ** -10 * 11 * 18 * SM * 4, float(err.max())


def test_lengths_that_the_device_holds_out_of_range():
    """seq_len and row_start are device data: brought into range, never a read behind the arrays."""
    s = Sequences([40, 50], [20, 30], 2, 128, Hq=4).fill_pages()
    want, wl = _run(s)
    for starts, lens in (([0, 20, 9999], [40, 50]), ([-5, 20, 50], [40, 50])):
        s.cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        out = torch.full_like(want, 7.0)
        akvq.paged_attention(s.cache, s.q, s.k, s.v, torch.tensor(starts, dtype=torch.int32, device="cuda"), 30, SM, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    s.cache.seq_len.copy_(torch.tensor([-3, 1 << 30], dtype=torch.int32))  # none; all that the table can name
    out, _ = _run(s)
    t = Sequences([0, s.cache.max_len], [20, 0], 2, 128, Hq=4)
    t.x, t.q, t.k, t.v = s.x, s.q, s.k, s.v
    check_attention(t, out, None, SM)
    assert bool(torch.isfinite(out[:20]).all())


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_negative_and_zero_scale(rows):
    s = Sequences([333], [rows], 2, 128, Hq=4, salient=[1, 200]).fill_pages()
    for sm in (-0.05, 0.0, 1e-3):
        for n_split in (1, 2):
            out, lse = _run(s, n_split, sm=sm)
            check_attention(s, out, lse, sm)


def test_long_caches_and_many_splits():
    s = Sequences([20011, 9000, 15], [1, 1, 1], 2, 128, page_rows=256, Hq=14, salient=range(0, 20000, 97), seed=2).fill_pages()
    for n_split in (0, 1, 16, 64):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM)


def test_pages_far_apart():
    """A pool of more than 2^32 bytes of codes: offsets of its last page."""
    Hkv, page_rows = 8, 1024
    n_pages = (1 << 32) // (Hkv * page_rows * 32) + 2
    small = Sequences([1500], [3], Hkv, 128, page_rows, Hq=Hkv, salient=[7, 1400]).fill_pages()
    want, _ = _run(small)
    big = akvq.PagedCache(1, Hkv, 128, n_pages, 2, page_rows, small.cache.S_cap)
    big.table[0] = torch.tensor([n_pages - 1, n_pages - 2], dtype=torch.int32)
    for i, page in enumerate(small.cache.table[0].tolist()):
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            getattr(big, name)[n_pages - 1 - i] = getattr(small.cache, name)[page]
    for name in ("k_sal", "v_sal", "sal_idx", "sal_cnt", "seq_len"):
        getattr(big, name).copy_(getattr(small.cache, name))
    got = akvq.paged_attention(big, small.q, small.k, small.v, small.row_start, small.max_rows, SM)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    before = big.k_codes[n_pages - 2].clone()   # ... and written there
    akvq.paged_append(big, small.k, small.v, small.row_start, 3, 0.8)
    akvq.paged_append(small.cache, small.k, small.v, small.row_start, 3, 0.8)
    torch.cuda.synchronize()
    page = int(small.cache.table[0, 1])
    for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
        assert torch.equal(getattr(big, name)[n_pages - 2], getattr(small.cache, name)[page])
    assert not torch.equal(before, big.k_codes[n_pages - 2])


def test_the_same_again_and_on_two_streams():
    """No call leaves anything for the next, and calls that overlap on two streams do not meet: equal bits every time."""
    a = Sequences([3000, 100], [1, 1], 4, 128, Hq=8, salient=SALIENT, seed=1).fill_pages()
    b = Sequences([2500], [40], 4, 64, Hq=8, salient=SALIENT, seed=2).fill_pages()
    want = [_run(x, 4) for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(5):
        for st, x in zip(streams, (a, b)):
            with torch.cuda.stream(st):
                out = torch.empty(x.n, x.Hq, 128, dtype=torch.float16, device="cuda")
                akvq.paged_attention(x.cache, x.q, x.k, x.v, x.row_start, x.max_rows, SM, n_split=4, out=out)
                got.append(out)
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert torch.equal(out, want[i % 2][0])


@pytest.mark.parametrize("rows", [1, 20, 33, 300])
@pytest.mark.parametrize("G", [128, 64])
def test_rows_that_were_never_written_are_zeros(G, rows):
    """Pages of a new pool hold scales of 0: keys and values of 0 for the softmax.  (Rows of the lists keep the bit that says they are
    read elsewhere: without it they would count here as well.)"""
    s = Sequences([150, 40], [rows, 1], 2, G, 32, Hq=4, salient=[3, 60]).fill_pages()
    for page in (int(s.cache.table[0, 1]), int(s.cache.table[1, 0])):
        s.cache.k_codes[page] = 0
        s.cache.v_codes[page] = 0
        s.cache.k_meta[page] &= 0x8000
        s.cache.v_meta[page] &= 0x8000
    for n_split in (1, 2):
        out, lse = _run(s, n_split)
        check_attention(s, out, lse, SM)


def test_tables_and_caches_that_the_caller_made():
    """The two tensors that the caller may replace are looked at; a cache that describes itself is asked."""
    s = Sequences([70, 3], [2, 1], 2, 128, Hq=4).fill_pages()
    want, _ = _run(s, 2)
    good = {n: getattr(s.cache, n) for n in ("table", "seq_len")}
    for name, bad, why in [("table", good["table"].long(), "table"), ("table", good["table"][:1], "table"), ("table", good["table"].cpu(), "current device"),
                           ("seq_len", good["seq_len"].long(), "seq_len"), ("seq_len", good["seq_len"][:1], "seq_len"),
                           ("seq_len", good["seq_len"].cpu(), "current device"), ("table", torch.stack((good["table"],) * 2, 2)[:, :, 0], "table")]:
        setattr(s.cache, name, bad)
        for call in (lambda: _run(s), lambda: akvq.paged_append(s.cache, s.k, s.v, s.row_start, s.max_rows, 0.8)):
            with pytest.raises(akvq.AkvqError, match=why):
                call()
        setattr(s.cache, name, good[name])
    with pytest.raises(akvq.AkvqError):
        _run(s, 1025)

    class Own(akvq.PagedCache):
        def paged_struct(self):
            asked.append(self)
            return super().paged_struct()

    asked = []
    s.cache.__class__ = Own
    assert torch.equal(_run(s, 2)[0], want) and asked == [s.cache]
    s.cache.paged_struct = lambda: None
    with pytest.raises(akvq.AkvqError, match="None"):
        _run(s)
    s.cache.paged_struct = lambda: s.cache.struct()  # of a contiguous cache
    with pytest.raises(TypeError):
        _run(s)


@pytest.mark.parametrize("rows,Hq,Hkv", [([1] * 9, 32, 32), ([20, 0, 32], 4, 2), ([300, 70, 0], 2, 1), ([2100, 1, 900], 1, 1)])
def test_captured_while_lengths_and_pages_change(rows, Hq, Hkv):
    """One capture of every tile size, replayed over other lengths, other pages and another share of the rows, each time against an eager call."""
    lens = [(61 * b + 30) % 200 + 60 for b in range(len(rows))]
    s = Sequences(lens, rows, Hkv, 128, 32, Hq=Hq, salient=SALIENT, seed=sum(rows)).fill_pages()
    table, starts = s.cache.table.clone(), s.row_start.clone()
    out, want = torch.zeros(s.n, Hq, 128, dtype=torch.float16, device="cuda"), torch.zeros(s.n, Hq, 128, dtype=torch.float16, device="cuda")

    def call(x):
        akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, SM, out=x)

    call(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for step in range(4):
        s.cache.seq_len.copy_(torch.tensor([(t * (step + 1)) % (t + 1) for t in lens], dtype=torch.int32))
        s.cache.table.copy_(table if step % 2 == 0 else table.roll(1, 1))
        s.row_start.copy_(starts if step < 2 else starts // 2)
        out.fill_(5)
        want.fill_(5)
        graph.replay()
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
