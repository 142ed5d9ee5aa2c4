"""Rows written into pages (akvq_paged_append): bit for bit what the contiguous write path stores for the same rows, and what the
CPU oracle does; everything else in the pools stays."""
import numpy as np
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences

pytestmark = pytest.mark.gpu
POOLS = ("k_codes", "v_codes", "k_meta", "v_meta")


def _scramble(s):
    """Pools and overlays hold something, and not zeros, before the call."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for name in POOLS + ("k_sal", "v_sal"):
        t = getattr(s.cache, name)
        lim = 1 << (15 if t.dtype == torch.int16 else 31)
        t.copy_(torch.randint(-lim, lim, t.shape, generator=g, device="cuda"))


def _check(s, clip=0.8, flags=0, call=None):
    p = s.cache
    p.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
    before = {name: getattr(p, name).clone() for name in POOLS + ("k_sal", "v_sal")}
    want = [s.contiguous(b) for b in range(p.B)]
    for b, c in enumerate(want):
        lo, hi = s.starts[b], s.starts[b + 1]
        if hi > lo:
            akvq.quantize_append(c, s.k[lo:hi].transpose(0, 1)[None].contiguous(), s.v[lo:hi].transpose(0, 1)[None].contiguous(), clip, flags)
    (call or (lambda: akvq.paged_append(p, s.k, s.v, s.row_start, s.max_rows, clip, flags)))()
    torch.cuda.synchronize()
    touched = set()
    for b, c in enumerate(want):
        got = s.contiguous(b)
        for name in POOLS + ("k_sal", "v_sal"):
            assert torch.equal(getattr(got, name), getattr(c, name)), (b, name)
        touched |= {x for x in p.table[b].tolist() if 0 <= x < p.n_pages}
    for page in set(range(p.n_pages)) - touched:
        for name in POOLS:
            assert torch.equal(getattr(p, name)[page], before[name][page]), (page, name)
    assert p.seq_len.tolist() == s.lens


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("lens,rows,Hkv,page_rows", [
    ([0], [1], 1, 64), ([63], [1], 3, 32), ([64], [2], 2, 64), ([0, 31, 32, 100], [1, 1, 1, 1], 4, 32),
    ([5, 0, 77], [40, 0, 64], 2, 64), ([0], [33], 5, 128), ([17, 1000, 3], [300, 1, 31], 2, 256), ([1, 2, 3, 4, 5], [31, 32, 33, 34, 65], 1, 64),
    ([4000], [129], 8, 64)])
def test_like_the_contiguous_write_path(lens, rows, Hkv, page_rows, G):
    s = Sequences(lens, rows, Hkv, G, page_rows, salient=[0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 1001, 4003], seed=sum(lens))
    _scramble(s)
    _check(s)


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("flags", [0, akvq.K_PREROTATED | akvq.V_PREROTATED])
def test_single_rows(G, flags):
    """One row a sequence at every kind of place in a block and a page, none for some; rows that are salient and rows that are not."""
    lens = [0, 1, 3, 15, 16, 17, 31, 32, 47, 63, 64, 95, 127, 200]
    s = Sequences(lens, [0 if i in (4, 9) else 1 for i in range(len(lens))], 3, G, 32, salient=[0, 1, 15, 31, 33, 64, 95, 200], seed=G + flags)
    _scramble(s)
    _check(s, flags=flags)


@pytest.mark.parametrize("count,step", [(1, 1), (64, 2), (65, 1), (66, 3), (1000, 1), (4097, 2), (6000, 1)])
def test_single_rows_and_long_salient_lists(count, step):
    """The row's entry first, last, in the middle of the list, just missing from it, and behind all of it."""
    lens = [0, (count - 1) * step, count // 2 * step, count // 2 * step + 1, count * step + 5]
    s = Sequences(lens, [1] * 5, 2, 128, salient=range(0, count * step, step), seed=count, S_cap=(count + 63) // 64 * 64)
    for b in range(5):  # final for rows that are still to come, as they are while a prompt is written
        s.cache.sal_idx[b, :, :count] = torch.arange(0, count * step, step, dtype=torch.int32, device="cuda")
        s.cache.counts()[b] = count
    _scramble(s)
    _check(s)


def test_single_rows_without_a_page_and_behind_the_table_are_dropped():
    s = Sequences([63, 64, 40], [1, 1, 1], 2, 128)
    p = s.cache
    p.table[1, 1] = -1
    p.table[2, 0] = p.n_pages
    p.max_len = p.max_pages * p.page_rows
    _scramble(s)
    p.seq_len.copy_(torch.tensor([p.max_len, 64, 40], dtype=torch.int32))  # the first is full
    before = {name: getattr(p, name).clone() for name in POOLS + ("k_sal", "v_sal")}
    akvq.paged_append(p, s.k, s.v, s.row_start, 1, 0.8)
    torch.cuda.synchronize()
    for name, old in before.items():
        assert torch.equal(getattr(p, name), old), name


@pytest.mark.parametrize("flags", [akvq.K_PREROTATED, akvq.V_PREROTATED, akvq.K_PREROTATED | akvq.V_PREROTATED])
def test_rows_that_arrive_rotated(flags):
    s = Sequences([9, 40], [50, 7], 3, 64, salient=range(0, 60, 7))
    _scramble(s)
    _check(s, clip=1.0, flags=flags)


@pytest.mark.parametrize("count", [64, 65, 200, 2500, 6000])
def test_long_salient_lists(count):
    """Runs of a block found by sampling: dense and sparse lists, entries before, inside and behind the chunk."""
    for step in (1, 3):
        s = Sequences([count * step // 2, 0], [200, 70], 2, 128, salient=range(0, count * step, step), seed=count, S_cap=(count + 63) // 64 * 64)
        s.cache.sal_idx[:, 1] += 1  # the heads' lists differ
        _scramble(s)
        _check(s)


def test_against_the_oracle(orc):
    s = Sequences([0, 0], [70, 33], 2, 64, salient=[1, 2, 40, 69], extra_rows=3)
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, s.max_rows, 0.8)
    torch.cuda.synchronize()
    for b, (lo, hi) in enumerate(zip(s.starts, s.starts[1:])):
        got = s.contiguous(b)
        oc = orc.OracleCache(1, 2, 64, got.T_cap, 64)
        text = np.zeros((1, hi - lo), np.uint8)
        text[0, [p for p in (1, 2, 40, 69) if p < hi - lo]] = 1
        oc.select_tsa(text)
        oc.quantize_append(s.k[lo:hi].transpose(0, 1)[None].contiguous().cpu().numpy(), s.v[lo:hi].transpose(0, 1)[None].contiguous().cpu().numpy(), 0.8)
        for name in POOLS:
            g, w = getattr(got, name).cpu().numpy().view(np.uint32), getattr(oc, name)
            if name.endswith("meta"):
                g, w = g[:, :, :hi - lo], w.reshape(g.shape)[:, :, :hi - lo]
            assert np.array_equal(g, w.reshape(g.shape)), (b, name)
        n = int(text.sum())
        assert np.array_equal(got.k_sal.cpu().numpy().view(np.uint16)[:, :, :n], oc.k_sal.view(np.uint16).reshape(1, 2, 64, 128)[:, :, :n])


def test_rows_without_a_page_and_behind_the_table_are_dropped():
    s = Sequences([30, 10], [100, 60], 2, 128, salient=[31, 50, 90])
    p = s.cache
    p.table[0, 1] = -1            # rows 64 to 127 of sequence 0
    p.table[1, 1] = p.n_pages     # rows 64 and up of sequence 1
    _scramble(s)
    before = {name: getattr(p, name).clone() for name in POOLS}
    p.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
    akvq.paged_append(p, s.k, s.v, s.row_start, s.max_rows, 0.8)
    torch.cuda.synchronize()
    for b, holes in ((0, [1]), (1, [1])):
        c = s.contiguous(b)
        full = Sequences(s.lens, s.rows, 2, 128, salient=[31, 50, 90])  # the same rows, all pages there
        _scramble(full)
        full.cache.seq_len.copy_(p.seq_len)
        akvq.paged_append(full.cache, full.k, full.v, full.row_start, full.max_rows, 0.8)
        w = full.contiguous(b)
        keep = 64
        assert torch.equal(c.k_codes[:, :, :2], w.k_codes[:, :, :2]) and torch.equal(c.v_meta[:, :, :keep], w.v_meta[:, :, :keep])
    used = {x for x in p.table.flatten().tolist() if 0 <= x < p.n_pages}
    for page in set(range(p.n_pages)) - used:
        for name in POOLS:
            assert torch.equal(getattr(p, name)[page], before[name][page])
    # a table that is too short for the rows: the last page ends the sequence
    t = Sequences([100], [200], 2, 128)
    t.cache.max_pages = 2         # of the five that the table has
    t.cache.max_len = 128
    t.cache.seq_len.fill_(100)
    table = t.cache.table.clone()
    t.cache.table = table[:, :2].contiguous()
    _scramble(t)
    old = t.cache.k_codes.clone()
    akvq.paged_append(t.cache, t.k, t.v, t.row_start, t.max_rows, 0.8)
    torch.cuda.synchronize()
    for page in table[0, 2:].tolist():
        assert torch.equal(t.cache.k_codes[page], old[page])
    assert not torch.equal(t.cache.k_codes[int(table[0, 1])], old[int(table[0, 1])])


def test_row_starts_out_of_range_write_nothing_wrong():
    """row_start and seq_len are device data: whatever they hold, only rows of the chunk and pages of the table are touched."""
    s = Sequences([40, 50], [20, 30], 2, 128)
    p = s.cache
    _scramble(s)
    before = {name: getattr(p, name).clone() for name in POOLS}
    for starts, lens in (([0, 20, 9999], [40, 50]), ([-5, 20, 10], [40, 50]), ([50, 20, 50], [-7, 1 << 30]), ([0, 0, 0], [40, 50])):
        for name in POOLS:
            getattr(p, name).copy_(before[name])
        p.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        akvq.paged_append(p, s.k, s.v, torch.tensor(starts, dtype=torch.int32, device="cuda"), 30, 0.8)
        torch.cuda.synchronize()
        for page in s.unused.tolist():
            for name in POOLS:
                assert torch.equal(getattr(p, name)[page], before[name][page])
    for name in POOLS:  # no rows at all: nothing changed
        assert torch.equal(getattr(p, name), before[name])


def test_max_rows_bounds_a_sequences_share():
    s, t = (Sequences([3, 8], [40, 12], 2, 128, seed=5) for _ in range(2))
    for x in (s, t):
        _scramble(x)
        x.cache.seq_len.copy_(torch.tensor(x.lens, dtype=torch.int32))
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, 12, 0.8)
    cut = torch.cat((t.x[:12], t.x[40:]))
    akvq.paged_append(t.cache, cut[:, 2:4], cut[:, 4:], torch.tensor([0, 12, 24], dtype=torch.int32, device="cuda"), 12, 0.8)
    torch.cuda.synchronize()
    for name in POOLS:
        assert torch.equal(getattr(s.cache, name), getattr(t.cache, name)), name


def test_another_stream_and_a_graph_over_many_steps():
    """Captured once, replayed while the caller advances seq_len: the pages of single rows written one after the other."""
    s = Sequences([30, 0, 62], [6, 6, 6], 2, 128, salient=[31, 32, 64])
    p, B = s.cache, 3
    _scramble(s)
    p.seq_len.copy_(torch.tensor(s.lens, dtype=torch.int32))
    k, v = torch.zeros(B, 2, 128, dtype=torch.float16, device="cuda"), torch.zeros(B, 2, 128, dtype=torch.float16, device="cuda")
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    want = [s.contiguous(b) for b in range(B)]
    for b, c in enumerate(want):
        lo = s.starts[b]
        for i in range(6):
            akvq.quantize_append(c, s.k[lo + i][None, :, None].contiguous(), s.v[lo + i][None, :, None].contiguous(), 0.8)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        akvq.paged_append(p, k, v, starts, 1, 0.8)
        p.seq_len.add_(1)
    for i in range(6):
        rows = [s.starts[b] + i for b in range(B)]
        k.copy_(s.k[rows])
        v.copy_(s.v[rows])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    assert p.seq_len.tolist() == [36, 6, 68]
    for b, c in enumerate(want):
        got = s.contiguous(b)
        for name in POOLS + ("k_sal", "v_sal"):
            assert torch.equal(getattr(got, name), getattr(c, name)), (b, name)
