"""Attention over 4-bit codes where the scales of a row's two groups lie far apart, in tiles of every size: each group's channels against the formula
in 64 bits, apart, in the rotated frame.

All weights are equal here (sm_scale 0): 2^6.5 to 2^15, and 2^-4 of that in tiles of 16 and 32 for every other row, whose codes lie 4 bits above the others.  A
group's is that times the group's scale over the larger one (tiles of 256: over twice the larger one's power of two), and is off by half a step of
binary16: 2^-11 of it, or 2^-25 where it is below the smallest normal number, which is up to 2^-25 * 16 * larger / (2^6.5 * scale) of it (tiles of 256: 2 for
16).  The result's own rounding is 2^-11 of it or 2^-25, and 32-bit sums leave 2^-18."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import cached_rows, sequences
from nibble_tiles import tile_of
from paged_inputs import hadamard

pytestmark = pytest.mark.gpu
TILES = [(4, 8), (8, 16), (48, 32), (8192, 256)]  # the caller's bound of a sequence's rows, and the tile that it brings


def make(lens, rows, bound, tile):
    s = sequences(lens, rows, 2, 64, 32, Hq=4, extra_rows=8192, seed=tile)
    s.max_rows = bound
    assert tile_of(s, bound) == tile
    return s


def check(s, bound, tile, larger, smallest):
    """larger: of a row's scales; smallest: of each group's."""
    s.x[:, s.Hq + s.Hkv:] = 0  # the chunk's own values
    for n_split in (1, 3):
        out = akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, bound, 0.0, n_split=n_split, flags=akvq.OUT_ROTATED)
        torch.cuda.synchronize()
        for b, t in enumerate(s.lens):
            lo, hi = s.starts[b], s.starts[b + 1]
            v = hadamard(cached_rows(s, b, t)[1]).repeat_interleave(s.Hq // s.Hkv, 0)  # [Hq, t, 128], rotated
            seen = (t + 1 + torch.arange(hi - lo, device="cuda", dtype=torch.float64))[:, None, None]
            want, size = v.sum(1)[None] / seen, v.abs().sum(1)[None] / seen
            err = (out[lo:hi].double() - want).abs()
            for g in range(2):
                at = slice(64 * g, 64 * g + 64)
                weight = max(2.0 ** -11, 2.0 ** -25 * (2 if tile == 256 else 16) * larger / (2 ** 6.5 * smallest[g]))
                limit = 2.0 ** -11 * want[..., at].abs() + 2.0 ** -25 + (weight + 2.0 ** -18) * size[..., at]
                assert bool((err[..., at] <= limit).all()), (n_split, b, g, float((err[..., at] / limit).max()))


@pytest.mark.parametrize("bound,tile", TILES)
@pytest.mark.parametrize("scales", [(1.0, 21 * 2.0 ** -24), (1.0, 3 * 2.0 ** -24), (2047 * 2.0 ** -24, 1.0), (16.0, 1027 * 2.0 ** -24), (1025 * 2.0 ** -20, 256.0),
                                    (1.5, 1.75), (2048.0, 1.0 + 2.0 ** -10)])
def test_scales_far_apart(scales, bound, tile):
    """Scales that are given, codes as they come, zero-points in their middle and outside."""
    s = make([300, 33, 1], [4, 1, 2], bound, tile).fill_pages(clip=1.0)
    bits = torch.tensor(scales, dtype=torch.float64).half()
    assert bits.double().tolist() == list(scales)
    zero = torch.tensor([7, -1], dtype=torch.int32)
    s.cache.k_meta[...] = 0x3C00
    s.cache.v_meta.copy_((bits.view(torch.int16).int() | (zero << 16)).expand_as(s.cache.v_meta))
    check(s, bound, tile, max(scales), scales)


@pytest.mark.parametrize("bound,tile", TILES)
@pytest.mark.parametrize("small", [0, 1])
@pytest.mark.parametrize("steps", [40, 310, 5000])
def test_a_constant_group_beside_a_small_one(steps, small, bound, tile):
    """Rows that arrive rotated, one group of them zeros, which are stored with a scale of 1, the other of a few or many steps of 2^-24."""
    s = make([200, 70], [4, 3], bound, tile)
    for _, v in s.past:
        v.zero_()
        x = torch.randint(0, steps + 1, (*v.shape[:2], 64), generator=torch.Generator(device="cuda").manual_seed(steps), device="cuda")
        v[..., 64 * small:64 * small + 64] = (x.double() * 2.0 ** -24).half()
    s.fill_pages(clip=1.0, flags=akvq.V_PREROTATED)
    meta = s.cache.v_meta[s.cache.v_meta[..., small] != 0]
    scale = (meta[:, small] & 0x7FFF).short().view(torch.float16).double()
    assert bool((meta[:, 1 - small] == 0x3C00).all()) and float(scale.max()) <= (steps / 15 + 1) * 2.0 ** -24
    smallest = [1.0, 1.0]
    smallest[small] = float(scale.min())
    check(s, bound, tile, 1.0, smallest)
