"""Offsets that pass 32 bits in the calls that turn rows and write pages of 4-bit codes: rows, positions and pages that lie gigabytes apart, against the same
call on compact arrays."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq

pytestmark = pytest.mark.gpu
HQ, HKV, N = 6, 2, 20
HEADS = HQ + 2 * HKV


def apart(x, stride):
    """Rows x `stride` elements from one to the next (what lies between is not initialised)."""
    far = torch.empty((x.shape[0] - 1) * stride + x[0].numel(), dtype=x.dtype, device="cuda")
    far = far.as_strided(x.shape, (stride,) + x[0].stride())
    far.copy_(x)
    return far


def parts(x):
    return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]


def inputs(n):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, HEADS, 128, generator=g, device="cuda").half()
    return x, torch.randint(0, 9000, (3, n), generator=g, device="cuda", dtype=torch.int32)


PLAN = akvq.Rotary([1e4 ** (-i / 48) for i in range(48)], [i % 3 for i in range(48)], 96, True)
STRIDE = 1 << 27  # 20 rows of it: 2.7e9 elements


def test_rows_and_positions_far_apart():
    x, pos = inputs(N)
    q, k, _ = parts(x)
    want = akvq.rotary_rows(PLAN, pos, q, k)
    fx, fpos = apart(x, STRIDE), apart(pos, (1 << 30) + 8)
    fq, fk, _ = parts(fx)
    got = akvq.rotary_rows(PLAN, fpos, fq, fk)
    akvq.rotary_rows(PLAN, fpos, fq, fk, q_out=fq, k_out=fk)
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, (fq, fk)):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("rows", [[1] * N, [15, 5]])
def test_chunks_far_apart(rows):
    x, pos = inputs(N)
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    fx, fpos = apart(x, STRIDE), apart(pos, (1 << 30) + 8)
    caches, outs = [], []
    for data, at in ((x, pos), (fx, fpos)):
        cache = akvq.PagedCache(len(rows), HKV, 128, len(rows), 1, 64, fill=0, bits=4)
        cache.table.copy_(torch.arange(len(rows), dtype=torch.int32)[:, None])
        cache.seq_len.fill_(21)
        q, k, v = parts(data)
        outs.append(akvq.paged_append_rotary(cache, PLAN, at, q, k, v, starts, max(rows), 1.0))
        other = akvq.PagedCache(len(rows), HKV, 128, len(rows), 1, 64, fill=0, bits=4)
        other.table.copy_(cache.table)
        akvq.paged_append(other, k, v, starts, max(rows), 1.0)
        caches.append((cache, other))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for a, b in zip(*caches):
        assert all(torch.equal(getattr(a, name), getattr(b, name)) for name in ("k_codes", "v_codes", "k_meta", "v_meta"))


@pytest.mark.parametrize("rows", [1, 100])
def test_pages_far_apart(rows):
    """Pages behind 2^31 words of codes."""
    pages, page_rows = 2060, 65536
    x, pos = inputs(rows)
    q, k, v = parts(x)
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    near, far = (akvq.PagedCache(1, HKV // 2, 64, n, 2, page_rows, bits=4) for n in (2, pages))
    for cache, table in ((near, [1, 0]), (far, [pages - 1, 2055])):
        cache.table.copy_(torch.tensor([table], dtype=torch.int32))
        cache.seq_len.fill_(page_rows - (50 if rows > 1 else 1))
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            getattr(cache, name)[table] = 0
    assert far.k_codes.numel() > 1 << 31
    for turned in (True, False):
        for cache in (near, far):
            if turned:
                akvq.paged_append_rotary(cache, PLAN, pos, None, k[:, :1], v[:, :1], starts, rows, 1.0)
            else:
                akvq.paged_append(cache, k[:, :1], v[:, :1], starts, rows, 1.0)
        torch.cuda.synchronize()
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            a, b = getattr(near, name), getattr(far, name)
            assert torch.equal(a[1], b[pages - 1]) and torch.equal(a[0], b[2055]), (turned, name)
        assert bool(near.k_codes[1].any()) and (rows == 1 or bool(near.v_codes[0].any()))
