"""Attention of a chunk over pages of 4-bit codes and over itself (paged_attention over PagedCache(bits=4)) against the formula in 64 bits on what the
pages hold, in tiles of every size: which one a call gets goes by the caller's bound of a sequence's rows, and is asserted.  Bounds: those of
nibble_inputs.check_attention."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import cached_rows, check_attention, sequences
from nibble_tiles import tile_of
from paged_inputs import hadamard

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700, 1001, 1500]
# the caller's bound of a sequence's rows, two heads a KV head, and the tile that it brings (8: of 16, up to eight rows)
TILES = [(4, 8), (8, 16), (48, 32), (8192, 256)]
tile_sizes = pytest.mark.parametrize("bound,tile", TILES)
groups = pytest.mark.parametrize("G", [128, 64])


def run(s, n_split=0, flags=0, sm=SM, x=None, Hq=None):
    q, k, v = (s.q, s.k, s.v) if x is None else (x[:, :s.Hq], x[:, s.Hq:s.Hq + s.Hkv], x[:, s.Hq + s.Hkv:])
    out = torch.full((s.x.shape[0], s.Hq, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((s.x.shape[0], s.Hq), 7.0, device="cuda")
    akvq.paged_attention(s.cache, q, k, v, s.row_start, s.max_rows, sm, n_split=n_split, flags=flags, out=out, lse=lse)
    torch.cuda.synchronize()
    assert bool((out[s.n:] == 7).all() and (lse[s.n:] == 7).all())  # rows of no sequence
    return out, lse


def make(lens, rows, bound, tile, G, **kw):
    s = sequences(lens, rows, 2, G, 32, Hq=4, extra_rows=8192, **kw)
    s.max_rows = bound
    assert tile_of(s, bound) == tile
    return s


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("lens,rows,Hq,Hkv,page_rows", [
    ([0], [1], 1, 1, 64), ([1], [1], 2, 2, 32), ([31, 32, 33], [1, 1, 1], 7, 1, 64), ([640], [1], 4, 4, 64), ([1000, 3], [1, 1], 8, 1, 128),
    ([0, 64, 65], [5, 16, 1], 3, 3, 32), ([100, 0], [8, 2], 28, 4, 64), ([700], [17], 2, 2, 64), ([5, 1601], [33, 64], 2, 1, 256),
    ([0], [65], 1, 1, 64), ([130], [129], 4, 2, 32), ([0, 300], [200, 0], 6, 1, 64), ([513, 64, 0, 2], [70, 1, 33, 100], 8, 2, 64),
    ([96], [257], 2, 2, 64), ([1234], [3], 16, 2, 64)])
def test_against_the_formula(lens, rows, Hq, Hkv, page_rows, G):
    s = sequences(lens, rows, Hkv, G, page_rows, Hq=Hq, salient=SALIENT, seed=sum(lens) + sum(rows)).fill_pages(clip=1.0)
    for n_split in (1, 0, 3, 7):
        out, lse = run(s, n_split)
        check_attention(s, out, lse, SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_tiles_of_every_size(bound, tile, G):
    s = make([0, 1, 33, 300, 64, 700], [4, 1, 3, 2, 0, 4], bound, tile, G, salient=SALIENT, seed=bound).fill_pages(clip=1.0)
    for n_split in (1, 2, 5):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@pytest.mark.parametrize("lens,rows,Hq,Hkv,tile", [
    ([17000], [40], 4, 1, 32), ([5000, 0, 200], [600, 2900, 1], 1, 1, 256), ([700, 3], [300, 260], 2, 1, 32), ([100, 1000], [17, 32], 2, 2, 16),
    ([500, 40], [4, 3], 28, 4, None)])
def test_chunks_that_bring_their_tile(lens, rows, Hq, Hkv, tile, G):
    s = sequences(lens, rows, Hkv, G, 64, Hq=Hq, salient=SALIENT, seed=sum(rows)).fill_pages(clip=1.0)
    assert tile is None or tile_of(s, s.max_rows) == tile
    for n_split in (0, 1, 3):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@pytest.mark.parametrize("lens,rows,Hq,Hkv", [
    ([70, 3, 0, 200, 33, 64, 1, 150, 90], [1, 1, 1, 1, 0, 1, 1, 1, 1], 32, 32),                 # more units than CUs: paired on them
    ([200] * 9, [1] * 9, 32, 32),                                                               # ... of equal lengths
    ([(37 * b) % 101 for b in range(64)], [b % 2 for b in range(64)], 8, 8),                    # as many sequences as lanes
    ([(37 * b) % 101 for b in range(65)], [b % 2 for b in range(65)], 8, 8),                    # more
    ([(37 * b) % 101 for b in range(29)], [b % 3 for b in range(29)], 28, 14),
    ([5, 300, 0, 300, 64, 20], [70, 65, 129, 1, 0, 300], 2, 2)])
def test_the_order_of_unequal_sequences(lens, rows, Hq, Hkv):
    """Which sequence a workgroup takes depends on all lengths: every row is still written once, with its own result."""
    s = sequences(lens, rows, Hkv, 128, 32, Hq=Hq, salient=SALIENT, seed=len(lens)).fill_pages(clip=1.0)
    for n_split in (1, 2):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@pytest.mark.parametrize("rows", [1, 5, 20, 70])
@pytest.mark.parametrize("length,page_rows", [(2040, 32), (4070, 32), (4200, 32), (9000, 32), (20000, 64), (11000, 1024)])
def test_tables_of_every_length(length, page_rows, rows):
    """Page numbers come 64 at a time: tables of up to 64 pages, of up to 128, and longer ones, begun anywhere."""
    s = sequences([length, 100], [rows, 1], 1, 128, page_rows, Hq=2, salient=SALIENT, seed=length).fill_pages(clip=1.0)
    for n_split in (1, 2, 9, 64):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
@pytest.mark.parametrize("salient", [[], range(0, 500), range(1, 500, 2), [299]])
def test_few_and_many_16_bit_rows(salient, bound, tile, G):
    """All rows in the overlay, none, every second one; lists that are already final for the chunk's own rows."""
    s = make([300, 200, 0], [4, 1, 4], bound, tile, G, salient=salient, seed=3).fill_pages(clip=1.0)
    for n_split in (1, 5):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_entries_that_are_no_page(bound, tile, G):
    s = make([300, 64, 90, 33], [4, 1, 4, 3], bound, tile, G, salient=[70, 290], seed=2).fill_pages(clip=1.0)
    s.cache.table[0, 1] = -1
    s.cache.table[0, 3] = s.cache.n_pages
    s.cache.table[0, 9] = -2 ** 31
    s.cache.table[1] = 2 ** 31 - 1   # all that is cached of it
    s.cache.table[2, 1] = -7
    for n_split in (1, 2, 5):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_what_takes_no_part_may_hold_anything(bound, tile, G):
    """NaN in other sequences' rows, unused pages, rows behind the length, unused overlay slots, and rows behind the chunk."""
    new = lambda: make([77, 45, 100], [4, 2, 4], bound, tile, G, salient=[5, 70, 80], seed=4).fill_pages(clip=1.0)
    s, clean = new(), new()
    p = s.cache
    used = {}
    for b in range(3):
        for i, page in enumerate(p.table[b].tolist()):
            if page >= 0:
                used[page] = min(max(s.lens[b] - i * p.page_rows, 0), p.page_rows)
    for page in range(p.n_pages):
        for t in (p.k_meta, p.v_meta):
            t[page, :, used.get(page, 0):] = 0x7E007E00   # scale NaN
        if page not in used:
            for t in (p.k_codes, p.v_codes, p.k_meta, p.v_meta):
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
        got, want = run(s, n_split), run(clean, n_split)
        check_attention(clean, *want, SM)
        for b in (0, 2):
            lo, hi = s.starts[b], s.starts[b + 1]
            assert torch.equal(got[0][lo:hi], want[0][lo:hi]) and torch.equal(got[1][lo:hi], want[1][lo:hi]), (n_split, b)


@groups
@tile_sizes
def test_large_scores_and_values_of_all_sizes(bound, tile, G):
    """Scores of hundreds (the reference is raised again and again, and one row decides), rising and falling along the keys."""
    for rising in (True, False):
        s = make([400], [4], bound, tile, G, gain=1.0, seed=5)
        k, v = s.past[0]
        ramp = torch.linspace(0.1, 30, 400, device="cuda")
        k *= (ramp if rising else ramp.flip(0))[None, :, None].half()
        v *= (10.0 ** torch.linspace(-3, 3, 400, device="cuda"))[None, :, None].half()
        s.fill_pages(clip=1.0)
        for n_split in (1, 3):
            check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_unrotated_groups_far_from_zero(bound, tile, G):
    """Channels near 20, whose zero-points pass 11 bits: |zero * scale| and |code * scale| cancel in 32-bit sums of terms of 20 a channel, which the
    bound's |q| |k| counts (|k| is 20 * 128 ** 0.5)."""
    s = make([300, 40], [4, 1], bound, tile, G, gain=1.0, seed=9)
    for past in s.past:
        for x in past:
            x.mul_(0.02).add_(20.0)
    s.fill_pages(clip=1.0, flags=akvq.K_PREROTATED | akvq.V_PREROTATED)
    assert int((s.cache.v_meta >> 16).abs().max()) > 2048
    for n_split in (1, 3):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_rows_that_were_never_written_are_zeros(bound, tile, G):
    s = make([150, 40], [4, 1], bound, tile, G, salient=[3, 60], seed=1).fill_pages(clip=1.0)
    for page in (int(s.cache.table[0, 1]), int(s.cache.table[1, 0])):
        s.cache.k_codes[page] = 0
        s.cache.v_codes[page] = 0
        s.cache.k_meta[page] &= 0x8000
        s.cache.v_meta[page] &= 0x8000
    for n_split in (1, 2):
        check_attention(s, *run(s, n_split), SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_rows_that_arrive_rotated(bound, tile, G):
    """The formula on the rows that were given, un-rotated; out is left rotated."""
    s = make([200, 0, 31], [4, 4, 1], bound, tile, G, salient=[3, 100], seed=3).fill_pages(clip=1.0)
    given = hadamard(s.x.double()).half()
    s.x = hadamard(given.double())
    s.q, s.k, s.v = s.x[:, :4], s.x[:, 4:6], s.x[:, 6:]
    for n_split in (1, 3):
        out, lse = run(s, n_split, akvq.Q_PREROTATED | akvq.OUT_ROTATED, x=given)
        back = out.double()
        back[:s.n] = hadamard(back[:s.n])
        check_attention(s, back, lse, SM, f"n_split {n_split}")


@groups
@tile_sizes
def test_scales_and_queries_at_their_ends(bound, tile, G):
    """Negative and zero scales; queries of zeros under a large scale; the smallest queries; one channel that decides."""
    s = make([333], [4], bound, tile, G, salient=[1, 200], seed=6).fill_pages(clip=1.0)
    s.x[1, 0] = 0.0
    s.x[2, 1] = 6e-8
    s.x[3, 2] = 0.0
    s.x[3, 2, 17] = 30.0
    for sm in (-0.05, 0.0, 1e-3, SM):
        for n_split in (1, 2):
            check_attention(s, *run(s, n_split, sm=sm), sm, f"sm {sm} n_split {n_split}")
    s.x[:s.n, :4] = 0.0
    for sm in (1e3, 1e9, 1e30, -1e30):
        out, lse = run(s, 2, sm=sm)
        check_attention(s, out, lse, 0.0, f"sm {sm}")


@groups
@tile_sizes
@pytest.mark.parametrize("zeros", [[1, -5, 300, -1000, 7], [1023, 1024, 1025, 1026, 1027], [-1021, -1024, -1025, -2045, -2047], [2047, 2048, 2049, 3583, 3584],
                                   [4095, -4096, 10000, -20001, 12345], [32767, -32768, 1025, -32767, 31743]])
def test_zero_points_and_codes_are_exact(zeros, bound, tile, G):
    """Means of cached rows whose zero-points and scales (one a group) are given; the chunk's own values are 0.  With sm_scale 0 every weight is 1, so
    that the sums are exact where the values are: zero-points are whole, scales powers of two, and up to 700 rows of multiples of one fit 24 bits.
    What is left is the division, 2^-22, a weight that up to eight rows have twice, 1 and 1 + 1.5 * 2^-12 over their unrounded sum, 2^-12 off, and
    the rounding of the result."""
    lens = [1, 31, 40, 300, 700]
    s = make(lens, [3, 1, 4, 4, 2], bound, tile, G, seed=G).fill_pages(clip=1.0)
    s.v.zero_()
    p, NG = s.cache, 128 // G
    scales = (2.0 ** -6, 2.0 ** -7)
    for b in range(len(lens)):
        for page in p.table[b].tolist():
            for g in range(NG if page >= 0 else 0):
                p.k_meta[page, :, :, g] = 0x3C00  # scale 1, zero-point 0
                bits = torch.tensor(scales[g], dtype=torch.float16).view(torch.int16).item()
                z = zeros[(b + 3 * g) % len(zeros)]
                p.v_meta[page, :, :, g] = bits | (((z & 0xFFFF) ^ 0x8000) - 0x8000) * 65536
    few = tile in (8, 16)  # (tiles of 16 have up to eight rows here)
    for n_split in (1, 2):
        out, _ = run(s, n_split, flags=akvq.OUT_ROTATED, sm=0.0)
        for b, t in enumerate(lens):
            lo, hi = s.starts[b], s.starts[b + 1]
            _, v, _ = cached_rows(s, b, t)
            total = hadamard(v).sum(1).repeat_interleave(2, 0)  # [Hq, 128], rotated
            want = total[None] / (t + 1 + torch.arange(hi - lo, device="cuda", dtype=torch.float64))[:, None, None]
            step = 2.0 ** (torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -14))) - 10)
            err = (out[lo:hi].double() - want).abs()
            bound_ = 0.5 * step + (2.0 ** -11 if few else 2.0 ** -20) * want.abs() + 2.0 ** -40
            assert bool((err <= bound_).all()), (zeros, b, n_split, float((err / bound_).max()))


@groups
@tile_sizes
def test_two_roundings_in_all(bound, tile, G):
    """A weight's and the result's, each 2.07e-4 of a number, root mean square (2^-11 / 3 ** 0.5 of its power of two, numbers spread over their
    logarithm): 2.93e-4 of the result's norm, as values and weights' errors do not follow each other; a third one would make it 3.59e-4.  Over 1024
    elements a row at least the mean is less than 5 % off."""
    rows = [4, 3] if bound == 4 else [8, 5] if bound == 8 else [40, 30]
    s = make([1500, 900], rows, bound, tile, G, seed=bound + G, gain=2.0).fill_pages(clip=1.0)
    out, _ = run(s)
    err = norm = 0.0
    for b, t in enumerate(s.lens):
        lo, hi = s.starts[b], s.starts[b + 1]
        kc, vc, _ = cached_rows(s, b, t)
        seen = torch.cat((torch.ones(hi - lo, t, device="cuda"), torch.ones(hi - lo, hi - lo, device="cuda").tril()), 1).bool()
        for h in range(4):
            k, v = torch.cat((kc[h // 2], s.k[lo:hi, h // 2].double())), torch.cat((vc[h // 2], s.v[lo:hi, h // 2].double()))
            p = torch.softmax((s.q[lo:hi, h].double() @ k.t().contiguous() * SM).masked_fill(~seen, float("-inf")), 1)
            want = p @ v
            err += float((out[lo:hi, h].double() - want).square().sum())
            norm += float(want.square().sum())
    assert (err / norm) ** 0.5 < 1.09 * 2.93e-4, (err / norm) ** 0.5


@pytest.mark.parametrize("Hq,rows", [(2, 1), (4, 2), (16, 1), (6, 1)])
def test_weights_of_few_rows_are_rounded_twice(Hq, rows):
    """One cached row decides (the others, and the chunk's own, are more than 30 below it), so that the output is its value times a rounded weight
    over the sum of unrounded ones.  A weight's error is, root mean square, 2.07e-4 of one rounding (2^-11 / 3 ** 0.5 of a number's power of two,
    numbers spread over their logarithm) and 1.10e-4 of the mean of two that are 1.5 * 2^-12 apart; of 120 weights and more it is less than 10 % off:
    1.4e-4 lies between."""
    lens = [20 + b for b in range(60 if Hq < 16 else 20)]
    s = sequences(lens, [rows] * len(lens), 2, 128, 32, Hq=Hq, seed=Hq + rows, gain=1.0)
    assert tile_of(s, s.max_rows) == 8
    for k, _ in s.past:
        k.mul_(0.01)
        k[:, 7] = 6.0  # one channel after the rotation
    s.fill_pages(clip=1.0)
    s.x[:, :Hq] = (1.0 + torch.rand(s.n, Hq, 1, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")).half()
    s.x[:, Hq:Hq + 2] = 0
    for n_split in (1, 3):
        out, _ = run(s, n_split, sm=0.06)
        errors = []
        for b, t in enumerate(lens):
            k, v, _ = cached_rows(s, b, t)
            scores = 0.06 * (s.q[s.starts[b]:s.starts[b + 1]].double().transpose(0, 1) @ k.repeat_interleave(Hq // 2, 0).transpose(1, 2).contiguous())
            first, second = scores.topk(2, dim=-1).values.unbind(-1)
            assert float(first.min()) > 30 and float((first - second).min()) > 30
            want = v[:, 7].repeat_interleave(Hq // 2, 0)
            got = out[s.starts[b]:s.starts[b + 1]].double()
            # half a step of binary16, and seven levels of 32-bit sums of the rotation and two factors, 2^-24 of the value's norm each
            half = 2.0 ** (torch.floor(torch.log2(got.abs().clamp(min=2.0 ** -14))) - 11) + 9 * 2.0 ** -24 * want.norm(dim=-1, keepdim=True)
            ends = torch.stack(((got - half) / want, (got + half) / want))
            low, high = ends.amin(0).amax(-1), ends.amax(0).amin(-1)
            assert bool((low <= high + 2.0 ** -20).all())
            errors.append(((low + high) / 2 - 1).flatten())
        errors = torch.cat(errors)
        assert len(errors) >= 120 and float(errors.square().mean().sqrt()) < 1.4e-4, float(errors.square().mean().sqrt())


@groups
@tile_sizes
def test_the_logarithm_changes_nothing_else(bound, tile, G):
    s = make([300, 40, 0], [4, 3, 4], bound, tile, G, seed=4, salient=[3, 31, 40, 200]).fill_pages(clip=1.0)
    for n_split in (1, 2, 5):
        out = akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, bound, SM, n_split=n_split)
        torch.cuda.synchronize()
        assert torch.equal(run(s, n_split)[0][:s.n], out[:s.n]), n_split


@pytest.mark.parametrize("n_split", [16, 17, 33, 64, 130])
@pytest.mark.parametrize("rows", [1, 20, 70])
def test_many_splits(n_split, rows):
    """More splits than the merge takes at a time, and more than there are blocks."""
    s = sequences([700, 20], [rows, 1], 2, 64, Hq=4, salient=SALIENT, seed=n_split).fill_pages(clip=1.0)
    check_attention(s, *run(s, n_split), SM)


@tile_sizes
def test_views_stay_and_the_same_again(bound, tile):
    """out as part of longer rows; equal bits every time."""
    s = make([50, 0, 9], [4, 3, 1], bound, tile, 64, salient=SALIENT).fill_pages(clip=1.0)
    for n_split in (1, 2):
        want, _ = run(s, n_split)
        for _ in range(3):
            wide = torch.full((s.x.shape[0], 9, 128), 7.0, dtype=torch.float16, device="cuda")
            akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, bound, SM, n_split=n_split, out=wide[:, 2:6])
            torch.cuda.synchronize()
            assert torch.equal(wide[:, 2:6], want) and bool((wide[:, :2] == 7).all() and (wide[:, 6:] == 7).all())


def test_lengths_that_the_device_holds_out_of_range():
    """seq_len and row_start are device data: brought into range, never a read behind the arrays."""
    s = sequences([40, 50], [20, 30], 2, 128, Hq=4).fill_pages(clip=1.0)
    want, _ = run(s)
    for starts in ([0, 20, 9999], [-5, 20, 50]):
        out = torch.full_like(want, 7.0)
        akvq.paged_attention(s.cache, s.q, s.k, s.v, torch.tensor(starts, dtype=torch.int32, device="cuda"), 30, SM, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    s.cache.seq_len.copy_(torch.tensor([-3, 1 << 30], dtype=torch.int32))  # none; all that the table can name
    out, _ = run(s)
    alone = sequences([0, s.cache.max_len], [20, 0], 2, 128, Hq=4)
    alone.x, alone.q, alone.k, alone.v = s.x, s.q, s.k, s.v
    check_attention(alone, out, None, SM)


def test_default_splits_of_the_callers_bound():
    """The library's choice is that of the max_rows it is given, also where fewer rows come: a workspace of that size serves them."""
    s = sequences([3000, 40], [1, 0], 2, 128, Hq=4, salient=SALIENT, seed=2).fill_pages(clip=1.0)
    L, c = akvq.lib(), s.cache.paged_struct()
    for max_rows in (1, 9, 200, 5000):
        n = L.akvq_paged_nibble_default_splits(C.byref(c), 4, max_rows)
        nws = L.akvq_paged_workspace_bytes(s.n, 4, n)
        ws = torch.empty(max(nws, 16), dtype=torch.uint8, device="cuda")
        out = torch.empty(s.n, 4, 128, dtype=torch.float16, device="cuda")
        chunk = akvq.akvq_chunk(s.row_start.data_ptr(), s.n, max_rows)
        assert L.akvq_paged_nibble_attention(C.byref(c), C.byref(chunk), s.q.data_ptr(), s.q.stride(0), 4, s.k.data_ptr(), s.k.stride(0), s.v.data_ptr(),
                                             s.v.stride(0), SM, out.data_ptr(), 512, None, 0, ws.data_ptr(), nws, 0, None) == 0
        torch.cuda.synchronize()
        check_attention(s, out, None, SM, f"max_rows {max_rows}")


def test_pages_far_apart():
    """A pool of more than 2^32 bytes of codes: offsets of its last page."""
    Hkv, page_rows = 8, 1024
    n_pages = (1 << 32) // (Hkv * page_rows * 64) + 2
    small = sequences([1500], [3], Hkv, 128, page_rows, Hq=Hkv, salient=[7, 1400]).fill_pages(clip=1.0)
    want, _ = run(small)
    big = akvq.PagedCache(1, Hkv, 128, n_pages, 2, page_rows, small.cache.S_cap, bits=4)
    big.table[0] = torch.tensor([n_pages - 1, n_pages - 2], dtype=torch.int32)
    for i, page in enumerate(small.cache.table[0].tolist()):
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            getattr(big, name)[n_pages - 1 - i] = getattr(small.cache, name)[page]
    for name in ("k_sal", "v_sal", "sal_idx", "sal_cnt", "seq_len"):
        getattr(big, name).copy_(getattr(small.cache, name))
    got = akvq.paged_attention(big, small.q, small.k, small.v, small.row_start, small.max_rows, SM)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    for call in (lambda c: akvq.paged_append(c, small.k, small.v, small.row_start, 3, 1.0),
                 lambda c: akvq.paged_append(c, small.k[:1], small.v[:1], torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1, 0.9)):
        call(big)   # ... and written there
        call(small.cache)
        torch.cuda.synchronize()
        page = int(small.cache.table[0, 1])
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            assert torch.equal(getattr(big, name)[n_pages - 2], getattr(small.cache, name)[page])


def test_calls_on_two_streams():
    """No call leaves anything for the next, and calls that overlap on two streams do not meet: equal bits every time."""
    a = sequences([3000, 100], [1, 1], 4, 128, Hq=8, salient=SALIENT, seed=1).fill_pages(clip=1.0)
    b = sequences([2500], [40], 4, 64, Hq=8, salient=SALIENT, seed=2).fill_pages(clip=1.0)
    want = [run(x, 4) for x in (a, b)]
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


@groups
@tile_sizes
def test_captured_while_lengths_pages_and_rows_change(bound, tile, G):
    """One capture of every tile size, replayed over other lengths, other pages and another share of the rows, each time against an eager call and the
    formula, with other work in between."""
    lens, rows = [250, 90, 130], [4, 1, 3]
    s = make(lens, rows, bound, tile, G, salient=SALIENT, seed=6).fill_pages(clip=1.0)
    table = s.cache.table.clone()
    out, lse = torch.full((s.x.shape[0], 4, 128), 7.0, dtype=torch.float16, device="cuda"), torch.full((s.x.shape[0], 4), 7.0, device="cuda")
    call = lambda: akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, bound, SM, out=out, lse=lse)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        s.lens = [t * (step + 1) % (t + 1) for t in lens]
        s.rows = rows if step < 2 else [1, 4, 3]
        s.starts = [0, s.rows[0], s.rows[0] + s.rows[1], sum(s.rows)]
        s.cache.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
        s.cache.table.copy_(table if step % 2 == 0 else table.roll(1, 1))
        s.row_start.copy_(torch.tensor(s.starts, dtype=torch.int32))
        want, wlse = run(s)
        out.fill_(7)
        lse.fill_(7)
        torch.randn(1 << 20, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wlse), step
        if step % 2 == 0:  # the other steps read pages of another sequence, whose lists do not agree with the marks in them
            check_attention(s, out, lse, SM, f"step {step}")
