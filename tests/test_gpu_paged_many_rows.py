"""Attention of a chunk in tiles of 256 rows (paged_attention_kernel with eight wavefronts), against the formula in 64 bits.  Which tile a call
gets goes by the caller's bound of the rows, so sequences of any length are brought there by arrays with many rows that belong to no
sequence; every call's tile is asserted.

Bounds: those of paged_inputs.check_attention (a score is off by 2^-15 |q| |k| sm_scale, a weight by twice that and half a step of binary16), and
with two groups a row half a step of binary16, 2^-11, of every value: there a value is a binary16 product of its group's scale."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, attention64, hadamard
from tile_rule import tile_of

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700, 1001, 1500]
BOUND = 8192  # of a sequence's rows, as the caller gives it


def _many(lens, rows, Hkv, G, page_rows=64, **kw):
    s = Sequences(lens, rows, Hkv, G, page_rows, extra_rows=BOUND, **kw)
    s.max_rows = BOUND
    assert tile_of(s, BOUND) == 256
    return s


def _run(s, n_split=1, flags=0, sm=SM, out=None):
    out = torch.full((s.x.shape[0], s.Hq, 128), 7.0, dtype=torch.float16, device="cuda") if out is None else out
    lse = torch.full((s.x.shape[0], s.Hq), 7.0, device="cuda")
    akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, sm, n_split=n_split, flags=flags, out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def _check(s, got, lse, sm=SM, what=""):
    value = 2.0 ** -11 if s.G == 64 else 0.0
    for b in range(s.cache.B):
        lo, hi = s.starts[b], s.starts[b + 1]
        if hi == lo:
            continue
        want, wlse, vnorm, qk = attention64(s, b, sm)
        err, score = (got[lo:hi].double() - want).norm(dim=2), 2.0 ** -15 * qk
        bound = 2.0 ** -11 * want.norm(dim=2) + 2.0 ** -25 * 128 ** 0.5 + (2.0 ** -11 + value + 2 * score + 2.0 ** -18) * vnorm
        assert bool((err <= bound).all()), (what, b, float((err / bound).max()), float((err / want.norm(dim=2)).max()))
        d = (lse[lo:hi].double() - wlse).abs()
        assert bool((d <= score + 2.0 ** -18 * (1 + wlse.abs())).all()), (what, b, float(d.max()))
    assert bool((got[s.n:] == 7).all() and (lse[s.n:] == 7).all())  # rows of no sequence


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("lens,rows,Hq,Hkv,page_rows", [
    ([0], [1], 1, 1, 64), ([1], [2], 2, 1, 32), ([31, 32, 33], [1, 0, 40], 7, 1, 64), ([640], [64], 4, 4, 64), ([127, 128, 129], [65, 1, 129], 8, 2, 32),
    ([1000, 0, 3], [31, 300, 1], 8, 1, 128), ([700], [600], 28, 4, 64), ([5, 1601], [33, 256], 2, 2, 256), ([2000], [37], 14, 2, 64)])
def test_against_the_formula(lens, rows, Hq, Hkv, page_rows, G):
    s = _many(lens, rows, Hkv, G, page_rows, Hq=Hq, salient=SALIENT, seed=sum(lens) + sum(rows)).fill_pages()
    for n_split in (1, 2, 7):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


def test_chunks_that_bring_the_tile_by_themselves():
    """... and a call whose bound is its longest chunk."""
    for G in (128, 64):
        s = Sequences([300, 0, 77], [1111, 700, 3], 4, G, Hq=28, salient=SALIENT, seed=8, extra_rows=2).fill_pages()
        assert tile_of(s, s.max_rows) == 256
        for n_split in (0, 3):
            _check(s, *_run(s, n_split), what=f"G {G} n_split {n_split}")


@pytest.mark.parametrize("lens,rows", [
    ([(37 * b) % 101 for b in range(65)], [(29 * b) % 71 for b in range(65)]),                                    # more sequences than lanes
    ([(37 * b) % 331 for b in range(64)], [300 if b % 9 == 0 else (29 * b) % 40 for b in range(64)]),             # as many
    ([5, 300, 0, 300, 64, 20], [70, 400, 129, 1, 0, 300])])
def test_the_order_of_unequal_sequences(lens, rows):
    for G in (128, 64):
        s = _many(lens, rows, 1, G, 32, Hq=2, salient=SALIENT, seed=len(lens)).fill_pages()
        for n_split in (1, 2):
            _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("length,page_rows", [(2040, 32), (4200, 32), (9000, 32), (20000, 64), (11000, 1024)])
def test_tables_of_every_length(length, page_rows):
    s = _many([length, 100], [40, 1], 1, 128, page_rows, Hq=2, salient=SALIENT, seed=length).fill_pages()
    for n_split in (1, 9):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("salient", [[], range(0, 500), range(1, 500, 2), [299], range(0, 65)])
def test_few_and_many_16_bit_rows(salient, G):
    """All rows in the overlay, none, every second one, one more than a stage."""
    s = _many([300, 200, 0], [150, 1, 90], 2, G, Hq=6, salient=salient, seed=3).fill_pages()
    for n_split in (1, 5):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_rows_without_a_page_take_no_part(G):
    s = _many([300, 64, 90], [40, 1, 270], 2, G, Hq=4, salient=[70, 290]).fill_pages()
    s.cache.table[0, 1] = -1
    s.cache.table[0, 3] = s.cache.n_pages
    s.cache.table[1, 0] = 1 << 30   # all that is cached of it
    s.cache.table[2, 1] = -7
    for n_split in (1, 3):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_what_takes_no_part_may_hold_anything(G):
    """NaN in other sequences' rows, unused pages, rows behind the length, unused overlay slots, and rows behind the chunk."""
    make = lambda: _many([77, 45, 100], [140, 2, 30], 2, G, Hq=6, salient=[5, 70, 80], seed=4).fill_pages()
    s, clean = make(), make()
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
        got, want = _run(s, n_split), _run(clean, n_split)
        for b in (0, 2):
            lo, hi = s.starts[b], s.starts[b + 1]
            assert torch.equal(got[0][lo:hi], want[0][lo:hi]) and torch.equal(got[1][lo:hi], want[1][lo:hi]), (n_split, b)
        _check(clean, *want)


@pytest.mark.parametrize("G", [128, 64])
def test_large_scores_and_values_of_all_sizes(G):
    """Scores of hundreds (the reference is raised again and again, and one row decides), rising and falling along the keys."""
    for rising in (True, False):
        s = _many([400], [50], 2, G, Hq=4, gain=1.0, seed=5)
        k, v = s.past[0]
        ramp = torch.linspace(0.1, 30, 400, device="cuda")
        k *= (ramp if rising else ramp.flip(0))[None, :, None].half()
        v *= (10.0 ** torch.linspace(-3, 3, 400, device="cuda"))[None, :, None].half()
        s.fill_pages()
        for n_split in (1, 3):
            _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_rows_that_were_never_written_are_zeros(G):
    s = _many([150, 40], [270, 1], 2, G, 32, Hq=4, salient=[3, 60]).fill_pages()
    for page in (int(s.cache.table[0, 1]), int(s.cache.table[1, 0])):
        s.cache.k_codes[page] = 0
        s.cache.v_codes[page] = 0
        s.cache.k_meta[page] &= 0x8000
        s.cache.v_meta[page] &= 0x8000
    for n_split in (1, 2):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_rotated_inputs_and_outputs(G):
    """q, k and v of the chunk rotated by the caller, out left rotated: the formula on the rows that were given."""
    s = _many([200, 30], [20, 270], 2, G, Hq=4, salient=[3, 100]).fill_pages()
    given = hadamard(s.x.double()).half()  # what the call gets; un-rotated again it is what the formula gets
    s.x = hadamard(given.double())
    s.q, s.k, s.v = s.x[:, :4], s.x[:, 4:6], s.x[:, 6:]
    for n_split in (1, 3):
        out = torch.full((s.x.shape[0], 4, 128), 7.0, dtype=torch.float16, device="cuda")
        lse = torch.full((s.x.shape[0], 4), 7.0, device="cuda")
        akvq.paged_attention(s.cache, given[:, :4], given[:, 4:6], given[:, 6:], s.row_start, BOUND, SM, n_split=n_split, out=out, lse=lse,
                             flags=akvq.Q_PREROTATED | akvq.OUT_ROTATED)
        torch.cuda.synchronize()
        back = torch.full(out.shape, 7.0, dtype=torch.float64, device="cuda")
        back[:s.n] = hadamard(out[:s.n].double())
        _check(s, back, lse, what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_negative_and_zero_scale(G):
    s = _many([333], [200], 2, G, Hq=4, salient=[1, 200]).fill_pages()
    for sm in (-0.05, 0.0, 1e-3):
        for n_split in (1, 2):
            _check(s, *_run(s, n_split, sm=sm), sm=sm, what=f"n_split {n_split}")


def test_views_stay_and_the_same_again():
    """out as part of longer rows; equal bits every time."""
    s = _many([50, 0, 9], [260, 3, 1], 2, 64, Hq=6, salient=SALIENT).fill_pages()
    for n_split in (1, 2):
        want, _ = _run(s, n_split)
        for _ in range(3):
            wide = torch.full((s.x.shape[0], 11, 128), 7.0, dtype=torch.float16, device="cuda")
            _run(s, n_split, out=wide[:, 2:8])
            assert torch.equal(wide[:, 2:8], want) and bool((wide[:, :2] == 7).all() and (wide[:, 8:] == 7).all())


@pytest.mark.parametrize("G", [128, 64])
def test_captured_while_lengths_and_rows_change(G):
    """Replayed over other lengths and another share of the rows, each time against the formula."""
    lens, rows = [250, 90, 130], [270, 5, 70]
    s = _many(lens, rows, 2, G, 32, Hq=4, salient=SALIENT, seed=6).fill_pages()
    out = torch.full((s.x.shape[0], 4, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((s.x.shape[0], 4), 7.0, device="cuda")
    call = lambda: akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, BOUND, SM, out=out, lse=lse)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        s.lens = [t * (step + 1) % (t + 1) for t in lens]
        s.rows = rows if step < 2 else [5, 270, 70]
        s.starts = [0, s.rows[0], s.rows[0] + s.rows[1], sum(s.rows)]
        s.cache.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
        s.row_start.copy_(torch.tensor(s.starts, dtype=torch.int32))
        out.fill_(7)
        lse.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        _check(s, out, lse, what=f"step {step}")
