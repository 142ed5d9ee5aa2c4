"""The write path into pages of 4-bit codes (paged_append over PagedCache(bits=4)) against its definition, bit for bit."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import overlay, page_codes, quantized, sequences

pytestmark = pytest.mark.gpu
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700]


def check_rows(s, b, first, k, v, clip=1.0, rotate_k=True, rotate_v=True, dropped=()):
    """Rows first, first + 1, ... of sequence b hold k, v [n, Hkv, 128]; `dropped`: rows of the sequence that have no page."""
    n = k.shape[0]
    parts, there = page_codes(s, b, first + n)
    keep = torch.tensor([t not in dropped for t in range(first, first + n)], dtype=torch.bool, device="cuda")
    assert torch.equal(there[first:], keep)
    for which, (x, rotate) in enumerate(((k, rotate_k), (v, rotate_v))):
        code, meta, wide = quantized(x.transpose(0, 1), s.G, 4, clip, rotate)
        got_code, got_meta, mark = parts[which]
        assert torch.equal(got_code[:, first:][:, keep].long(), code[:, keep]), (b, which)
        assert torch.equal(got_meta[:, first:][:, keep], meta[:, keep] & ~0x8000), (b, which)
        for h in range(s.Hkv):
            idx = s.cache.sal_idx[b, h, :int(s.cache.counts()[b, h])].tolist()
            rows = overlay(s.cache, b, h, which)
            for t in range(first, first + n):
                if t in dropped:
                    continue
                assert bool(mark[h, t].all()) == (t in idx) and bool(mark[h, t].any()) == (t in idx)
            new = [i for i, t in enumerate(idx) if first <= t < first + n and t not in dropped]
            if new:
                at = torch.tensor([idx[i] - first for i in new], device="cuda")
                assert torch.equal(rows[torch.tensor(new, device="cuda")], wide[h, at].double())


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("lens,rows,Hkv,page_rows", [
    ([0], [1], 1, 32), ([31, 32, 33, 0], [1, 1, 1, 1], 3, 64), ([0], [32], 2, 32), ([5], [27], 1, 64), ([5, 40, 0], [28, 0, 70], 2, 32),
    ([700], [129], 4, 256), ([1, 2, 3, 4, 300], [2, 3, 31, 33, 5], 2, 64), ([16, 15, 17], [16, 1, 15], 1, 32)])
def test_against_the_definition(lens, rows, Hkv, page_rows, G):
    s = sequences(lens, rows, Hkv, G, page_rows, salient=SALIENT, seed=sum(lens) + sum(rows)).fill_pages(clip=1.0)
    before = [page_codes(s, b, t)[0] for b, t in enumerate(lens)]
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, s.max_rows, 0.9)
    for b, t in enumerate(lens):
        check_rows(s, b, t, s.k[s.starts[b]:s.starts[b + 1]], s.v[s.starts[b]:s.starts[b + 1]], 0.9)
        if t:  # what was there has stayed
            check_rows(s, b, 0, s.past[b][0].transpose(0, 1), s.past[b][1].transpose(0, 1))
            for old, new in zip(before[b], page_codes(s, b, t)[0]):
                assert all(torch.equal(x, y) for x, y in zip(old, new))


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("flags", [akvq.K_PREROTATED, akvq.V_PREROTATED, akvq.K_PREROTATED | akvq.V_PREROTATED])
def test_rows_that_come_rotated(rows, flags):
    s = sequences([33, 0], [rows, rows], 2, 64, salient=SALIENT, seed=rows + flags)
    s.cache.seq_len.copy_(torch.tensor([33, 0], dtype=torch.int32))
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, s.max_rows, 1.0, flags)
    for b, t in enumerate([33, 0]):
        lo, hi = s.starts[b], s.starts[b + 1]
        check_rows(s, b, t, s.k[lo:hi], s.v[lo:hi], 1.0, not flags & akvq.K_PREROTATED, not flags & akvq.V_PREROTATED)


@pytest.mark.parametrize("rows", [1, 5, 64])
def test_extreme_rows(rows):
    """Constant rows, zeros, one large channel, the largest and the smallest binary16, rows far from zero."""
    s = sequences([0, 30], [rows, rows], 1, 128, seed=rows)
    n = 2 * rows
    x = torch.zeros(n, 1, 128, dtype=torch.float16, device="cuda")
    kinds = [lambda: torch.zeros(128), lambda: torch.full((128,), 3.0), lambda: torch.eye(128)[7] * 60000, lambda: torch.full((128,), 65504.0),
             lambda: torch.full((128,), -65504.0), lambda: torch.full((128,), 6e-8), lambda: torch.randn(128) + 500, lambda: torch.randn(128) * 1e-6]
    torch.manual_seed(rows)
    for i in range(n):
        x[i, 0] = kinds[i % len(kinds)]().half().cuda()
    s.cache.seq_len.copy_(torch.tensor([0, 30], dtype=torch.int32))
    for flags in (0, akvq.K_PREROTATED | akvq.V_PREROTATED):
        akvq.paged_append(s.cache, x, x.flip(0).contiguous(), s.row_start, rows, 1.0, flags)
        for b, t in enumerate([0, 30]):
            lo, hi = s.starts[b], s.starts[b + 1]
            check_rows(s, b, t, x[lo:hi], x.flip(0)[lo:hi], 1.0, not flags, not flags)


def _pools(c):
    return [getattr(c, n).clone() for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")]


@pytest.mark.parametrize("rows", [1, 70])
def test_rows_without_a_place(rows):
    """Pages that are not named, lengths outside of the table: rows are dropped, everything else stays."""
    s = sequences([40, 90, 64, 0], [rows] * 4, 2, 128, 32, salient=[40, 41, 95], seed=rows)
    s.cache.table[0, 1:3] = torch.tensor([-1, s.cache.n_pages], dtype=torch.int32)  # rows 32 to 95
    if rows > 1:
        s.cache.table[1, 3] = -5  # rows 96 on
    s.cache.seq_len.copy_(torch.tensor([40, 90, -3, s.cache.max_pages * 32], dtype=torch.int32))
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, rows, 1.0)
    lo = s.starts
    check_rows(s, 0, 40, s.k[lo[0]:lo[1]], s.v[lo[0]:lo[1]], dropped=range(32, 96))
    check_rows(s, 1, 90, s.k[lo[1]:lo[2]], s.v[lo[1]:lo[2]], dropped=range(96, 128))
    used = set(s.cache.table[0].tolist()) | set(s.cache.table[1].tolist())
    for page in range(s.cache.n_pages):
        if page not in used:
            assert not bool(s.cache.k_codes[page].any() or s.cache.v_codes[page].any() or s.cache.k_meta[page].any() or s.cache.v_meta[page].any())


def test_bounds_of_the_call():
    """Rows behind max_rows, and rows of no sequence, take no part; no rows is no launch."""
    s = sequences([10, 0, 7], [6, 3, 40], 2, 64, extra_rows=5, seed=1)
    s.cache.seq_len.copy_(torch.tensor([10, 0, 7], dtype=torch.int32))
    fresh = _pools(s.cache)
    akvq.paged_append(s.cache, s.k[:0], s.v[:0], torch.zeros(4, dtype=torch.int32, device="cuda"), 3, 1.0)
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, 0, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(fresh, _pools(s.cache)))
    akvq.paged_append(s.cache, s.k, s.v, s.row_start, 4, 1.0)
    for b, t in enumerate([10, 0, 7]):
        n = min(4, s.rows[b])
        check_rows(s, b, t, s.k[s.starts[b]:s.starts[b] + n], s.v[s.starts[b]:s.starts[b] + n])
        page = s.cache.table[b, 0]
        assert not bool(s.cache.k_meta[page, :, t + n:].any())


def test_the_same_rows_in_pieces_and_at_once():
    """Chunk by chunk and row by row the pages get the bits of one call."""
    whole = sequences([0, 0], [150, 81], 2, 64, 32, salient=SALIENT, seed=3)
    akvq.paged_append(whole.cache, whole.k, whole.v, whole.row_start, 150, 0.95)
    parts = sequences([0, 0], [150, 81], 2, 64, 32, salient=SALIENT, seed=3)
    done = [0, 0]
    for take in ([1, 1], [30, 0], [0, 31], [1, 1], [70, 40], [1, 1], [1, 1], [46, 6]):
        rows = [r for b in range(2) for r in range(parts.starts[b] + done[b], parts.starts[b] + done[b] + take[b])]
        start = torch.tensor([0, take[0], sum(take)], dtype=torch.int32, device="cuda")
        akvq.paged_append(parts.cache, parts.k[rows], parts.v[rows], start, max(take), 0.95)
        done = [a + b for a, b in zip(done, take)]
        parts.cache.seq_len.copy_(torch.tensor(done, dtype=torch.int32))
    assert done == [150, 81]
    assert all(torch.equal(a, b) for a, b in zip(_pools(whole.cache), _pools(parts.cache)))
