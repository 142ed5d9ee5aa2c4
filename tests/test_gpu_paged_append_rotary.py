"""A chunk turned and written into the pages in one call (paged_append_rotary): bit for bit what rotary_rows and paged_append do one after the
other, in pages of 2-bit and of 4-bit codes."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import sequences
from rotary_reference import check_turned

pytestmark = pytest.mark.gpu
SALIENT = [0, 3, 31, 32, 40, 63, 64, 65, 100, 101, 300, 301, 302, 303, 700]
POOLS = ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")


def plan_of(dim=128, interleaved=False, axes=1, magnitude=1.0):
    freq = [1e4 ** (-2 * i / dim) for i in range(dim // 2)]
    axis = [i % axes for i in range(dim // 2)]
    return akvq.Rotary(freq, axis, dim, interleaved, magnitude), (freq, axis, dim, interleaved, magnitude)


def positions(n, axes, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 1 << 17, (axes, n), generator=g, device="cuda", dtype=torch.int32)


def both(make, rot, pos, clip=0.9, max_rows=None, flags=0, lens=None, q=True):
    """The caches and rows of the one call and of the two."""
    a, b = make(), make()
    for s in (a, b):
        s.cache.seq_len.copy_(torch.tensor(lens if lens is not None else s.lens, dtype=torch.int32))
    most = a.max_rows if max_rows is None else max_rows
    one = akvq.paged_append_rotary(a.cache, rot, pos, a.q if q else None, a.k, a.v, a.row_start, most, clip, flags=flags)
    two = akvq.rotary_rows(rot, pos, b.q if q else None, b.k)
    akvq.paged_append(b.cache, two[1], b.v, b.row_start, most, clip, flags)
    torch.cuda.synchronize()
    return a, b, one, two


def same_pools(a, b):
    for name in POOLS:
        assert torch.equal(getattr(a.cache, name), getattr(b.cache, name)), name


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (128, True), (16, False), (16, True), (64, False), (80, False), (96, True), (112, False)])
@pytest.mark.parametrize("lens,rows,Hq,Hkv,G,page_rows", [
    ([0], [1], 1, 1, 128, 32), ([31, 32, 33, 700], [1, 1, 0, 1], 7, 1, 64, 64), ([5, 40, 0, 63], [28, 0, 70, 33], 4, 2, 128, 32),
    ([1, 200], [140, 3], 28, 4, 64, 64), ([16], [47], 3, 3, 128, 64)])
def test_as_the_two_calls(lens, rows, Hq, Hkv, G, page_rows, dim, interleaved, bits):
    rot, plan = plan_of(dim, interleaved, 3, 1.2)
    make = lambda: sequences(lens, rows, Hkv, G, page_rows, Hq=Hq, salient=SALIENT, seed=sum(lens) + dim, bits=bits).fill_pages()
    s = make()
    pos = positions(s.n, 3)
    a, b, one, two = both(make, rot, pos)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    same_pools(a, b)
    check_turned(one[0], s.q, pos, *plan)
    check_turned(one[1], s.k, pos, *plan)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("rows", [1, 50])
def test_values_that_come_rotated_and_no_queries(rows, bits):
    rot, _ = plan_of(64, True)
    make = lambda: sequences([3, 90], [rows, rows], 2, 64, Hq=4, salient=SALIENT, seed=rows, bits=bits)
    pos = positions(2 * rows, 1)
    a, b, one, two = both(make, rot, pos, flags=akvq.V_PREROTATED, q=False)
    assert one[0] is None and torch.equal(one[1], two[1])
    same_pools(a, b)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (128, True), (48, False), (48, True)])
def test_in_place(dim, interleaved, rows, bits):
    """The parts of one fused projection turned where they lie; values stay."""
    rot, _ = plan_of(dim, interleaved)
    make = lambda: sequences([3, 90], [rows, rows], 2, 128, Hq=4, salient=SALIENT, seed=rows, bits=bits)
    pos = positions(2 * rows, 1)
    a, b, one, two = both(make, rot, pos)
    s = make()
    s.cache.seq_len.copy_(torch.tensor([3, 90], dtype=torch.int32))
    v = s.v.clone()
    got = akvq.paged_append_rotary(s.cache, rot, pos, s.q, s.k, s.v, s.row_start, s.max_rows, 0.9, q_out=s.q, k_out=s.k)
    assert got[0] is s.q and got[1] is s.k
    assert torch.equal(s.q, two[0]) and torch.equal(s.k, two[1]) and torch.equal(s.v, v)
    same_pools(s, b)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("rows", [1, 70])
def test_rows_without_a_place_are_turned_all_the_same(rows, bits):
    rot, plan = plan_of(128, False)

    def make():
        s = sequences([40, 90, 64, 0], [rows] * 4, 2, 128, 32, Hq=4, salient=[40, 41, 95], seed=rows, bits=bits)
        s.cache.table[0, 1:3] = torch.tensor([-1, s.cache.n_pages], dtype=torch.int32)
        if rows > 1:
            s.cache.table[1, 3] = -5
        return s
    pos = positions(4 * rows, 1)
    a, b, one, two = both(make, rot, pos, lens=[40, 90, -3, make().cache.max_pages * 32])
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    same_pools(a, b)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("lens", [[10, 0, 7], [10, 33, -1]])
def test_rows_that_are_nobodys_stay(lens, bits):
    """Rows behind max_rows and behind the last sequence: not turned, not stored, whatever q_out and k_out hold; a sequence without rows in a block
    that others begin in."""
    rot, plan = plan_of(32, True)
    s = sequences([10, 33, 7], [6, 0, 40], 2, 64, Hq=3, extra_rows=5, seed=1, bits=bits)
    s.cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
    pos = positions(s.x.shape[0], 1)
    q_out, k_out = (torch.full_like(x.contiguous(), 7.0) for x in (s.q, s.k))
    akvq.paged_append_rotary(s.cache, rot, pos, s.q, s.k, s.v, s.row_start, 4, 1.0, q_out=q_out, k_out=k_out)
    mine = [r for b in range(3) for r in range(s.starts[b], s.starts[b] + min(4, s.rows[b]))]
    rest = [r for r in range(s.x.shape[0]) if r not in mine]
    assert bool((q_out[rest] == 7).all() and (k_out[rest] == 7).all())
    check_turned(q_out[mine], s.q[mine], pos[:, mine], *plan)
    check_turned(k_out[mine], s.k[mine], pos[:, mine], *plan)
    pages = [getattr(s.cache, n).clone() for n in POOLS]
    akvq.paged_append_rotary(s.cache, rot, pos, s.q, s.k, s.v, s.row_start, 0, 1.0)
    akvq.paged_append_rotary(s.cache, rot, pos[:, :0], s.q[:0], s.k[:0], s.v[:0], s.row_start * 0, 4, 1.0)
    assert all(torch.equal(x, getattr(s.cache, n)) for x, n in zip(pages, POOLS))


def test_more_heads_than_a_workgroup_takes():
    rot, plan = plan_of(128, False, 2)
    make = lambda: sequences([0, 20], [40, 33], 40, 128, Hq=80, salient=SALIENT, seed=9)
    pos = positions(73, 2)
    a, b, one, two = both(make, rot, pos)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    same_pools(a, b)
