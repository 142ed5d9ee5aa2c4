"""Attention of a chunk over pages of 4-bit codes and over itself (paged_attention over PagedCache(bits=4)) against the formula in 64 bits on what the
pages hold."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import check_attention, sequences

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700, 1001, 1500]


def run(s, n_split=0, flags=0, sm=SM):
    out = torch.full((s.x.shape[0], s.Hq, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((s.x.shape[0], s.Hq), 7.0, device="cuda")
    akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, sm, n_split=n_split, flags=flags, out=out, lse=lse)
    torch.cuda.synchronize()
    return out, lse


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
