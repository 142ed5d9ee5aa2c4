"""akvq_paged_attention in tiles of 16, 32 and 256 rows, each asserted: entries of the table that are no page, and rows that arrive rotated, against
the formula in 64 bits, within the bounds of test_gpu_paged_many_rows."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, hadamard
from test_gpu_paged_many_rows import _check
from tile_rule import tile_of

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
TILES = [(8, 16), (48, 32), (8192, 256)]


def _make(lens, rows, bound, tile, G, **kw):
    s = Sequences(lens, rows, 2, G, 32, Hq=4, extra_rows=8192, **kw)
    s.max_rows = bound
    assert tile_of(s, bound) == tile
    return s


def _run(s, n_split, flags=0, x=None):
    x = s.x if x is None else x
    out, lse = torch.full((x.shape[0], 4, 128), 7.0, dtype=torch.float16, device="cuda"), torch.full((x.shape[0], 4), 7.0, device="cuda")
    akvq.paged_attention(s.cache, x[:, :4], x[:, 4:6], x[:, 6:], s.row_start, s.max_rows, SM, n_split=n_split, flags=flags, out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("bound,tile", TILES)
def test_entries_that_are_no_page(bound, tile, G):
    s = _make([300, 64, 90, 33], [8, 1, 5, 3], bound, tile, G, salient=[70, 290], seed=2).fill_pages()
    s.cache.table[0, 1] = -1
    s.cache.table[0, 3] = s.cache.n_pages
    s.cache.table[0, 9] = -2 ** 31
    s.cache.table[1] = 2 ** 31 - 1   # all that is cached of it
    s.cache.table[2, 1] = -7
    for n_split in (1, 2, 5):
        _check(s, *_run(s, n_split), what=f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("bound,tile", TILES)
def test_rows_that_arrive_rotated(bound, tile, G):
    """The formula on the rows that were given, un-rotated; out is left rotated."""
    s = _make([200, 0, 31], [8, 4, 1], bound, tile, G, salient=[3, 100], seed=3).fill_pages()
    given = hadamard(s.x.double()).half()
    s.x = hadamard(given.double())
    s.q, s.k, s.v = s.x[:, :4], s.x[:, 4:6], s.x[:, 6:]
    for n_split in (1, 3):
        out, lse = _run(s, n_split, akvq.Q_PREROTATED | akvq.OUT_ROTATED, given)
        back = out.double()
        back[:s.n] = hadamard(back[:s.n])
        _check(s, back, lse, what=f"n_split {n_split}")
