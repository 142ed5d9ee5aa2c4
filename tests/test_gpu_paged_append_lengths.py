"""Where akvq_paged_append puts rows goes by the length that the device holds: the host's bound of it (max_len) sizes what reads, and a length
that names no row of the table drops the rows."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences

pytestmark = pytest.mark.gpu
ALL = ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")


def _append(s, max_rows=None):
    s.cache.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, max_rows or s.max_rows, 0.8)
    torch.cuda.synchronize()


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("rows", [1, 2, 70])
def test_a_bound_that_lengths_have_passed(rows, G):
    """Every bound stores the same, one row a sequence and more; nothing between the bound and the length changes."""
    make = lambda: Sequences([40, 97, 64, 33], [rows, rows, 0, rows], 2, G, 32, salient=[0, 33, 40, 41, 90, 97, 98], seed=rows).fill_pages()
    want = make()
    before = {name: getattr(want.cache, name).clone() for name in ALL}
    _append(want)
    assert not all(torch.equal(getattr(want.cache, name), before[name]) for name in ALL)
    for bound in (0, 1, 33, 64, 96):
        s = make()
        s.cache.max_len = bound
        _append(s)
        for name in ALL:
            assert torch.equal(getattr(s.cache, name), getattr(want.cache, name)), (bound, name)


@pytest.mark.parametrize("rows", [1, 70])
def test_lengths_that_name_no_row_drop_the_rows(rows):
    s = Sequences([40, 97, 10], [rows] * 3, 2, 128, 32, salient=[0, 33, 40, 41], seed=rows).fill_pages()
    end = s.cache.max_pages * s.cache.page_rows
    before = {name: getattr(s.cache, name).clone() for name in ALL}
    for lens in ([-1, end, 2 ** 31 - 1], [-2 ** 31, end + 1, -40]):
        s.lens = lens
        _append(s)
        for name in ALL:
            assert torch.equal(getattr(s.cache, name), before[name]), (lens, name)


def test_a_captured_step_that_runs_past_its_bound():
    """max_len set once, at the capture: the rows of later replays lie where the lengths are."""
    s, want = (Sequences([30, 5], [6, 6], 2, 128, 32, salient=[31, 32], seed=3).fill_pages() for _ in range(2))
    want.cache.seq_len.copy_(torch.tensor(want.lens, dtype=torch.int32))
    akvq.paged_append(want.cache, want.k, want.v, want.row_start, 6, 0.8)
    p = s.cache
    p.max_len = 31
    p.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
    k, v = torch.zeros(2, 2, 128, dtype=torch.float16, device="cuda"), torch.zeros(2, 2, 128, dtype=torch.float16, device="cuda")
    starts = torch.arange(3, dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        akvq.paged_append(p, k, v, starts, 1, 0.8)
        p.seq_len.add_(1)
    for i in range(6):
        rows = [s.starts[b] + i for b in range(2)]
        k.copy_(s.k[rows])
        v.copy_(s.v[rows])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    assert p.seq_len.tolist() == [36, 11]
    for name in ALL:
        assert torch.equal(getattr(p, name), getattr(want.cache, name)), name
