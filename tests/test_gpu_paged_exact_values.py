"""Values of tiles of 256 rows (akvq_paged_attention): zero-points of any size and groups of different scales, seen where every weight is the same, so that the
kernel's own sums are exact; and rows far from zero against the formula."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import cached_rows, hadamard
from test_gpu_paged_many_rows import _check, _many, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [128, 64])
def test_unrotated_groups_far_from_zero(G):
    """Channels near 20, whose zero-points pass 10 and 11 bits."""
    for width, least in ((0.01, 1024), (0.002, 2048)):
        s = _many([300, 40], [50, 1], 2, G, Hq=4, gain=1.0, seed=9)
        for past in s.past:
            for x in past:
                x.mul_(width).add_(20.0)
        s.fill_pages(clip=1.0, flags=akvq.K_PREROTATED | akvq.V_PREROTATED)
        assert int((s.cache.v_meta >> 16).abs().max()) > least
        for n_split in (1, 3):
            _check(s, *_run(s, n_split), what=f"n_split {n_split}")


def _equal_weights(G, zeros, scales):
    """Means of cached rows whose zero-points and scales (one a group) are given, sequence by sequence; the chunk's own values are 0.  With
    sm_scale 0 every weight is 1, so that the sums are exact where the values are: zero-points are whole, scales have few bits, and up to
    700 rows of multiples of a power of two fit 24 bits.  What is left is the division, 2^-22, and the rounding of the result."""
    lens = [1, 31, 40, 300, 700]
    s = _many(lens, [3, 1, 40, 270, 2], 2, G, 32, Hq=4, seed=G).fill_pages()
    s.v.zero_()
    p, NG = s.cache, 128 // G
    for b in range(len(lens)):
        for page in p.table[b].tolist():
            if page < 0:
                continue
            for g in range(NG):
                p.k_meta[page, :, :, g] = 0x3C00  # scale 1, zero-point 0
                bits = torch.tensor(scales[g], dtype=torch.float16).view(torch.int16).item()
                z = zeros[(b + 3 * g) % len(zeros)]
                p.v_meta[page, :, :, g] = bits | (((z & 0xFFFF) ^ 0x8000) - 0x8000) * 65536
    for n_split in (1, 2):
        out, _ = _run(s, n_split, flags=akvq.OUT_ROTATED, sm=0.0)
        for b, t in enumerate(lens):
            lo, hi = s.starts[b], s.starts[b + 1]
            _, v, _ = cached_rows(s, b, t)
            total = hadamard(v).sum(1).repeat_interleave(2, 0)  # [Hq, 128], rotated
            want = total[None] / (t + 1 + torch.arange(hi - lo, device="cuda", dtype=torch.float64))[:, None, None]
            step = 2.0 ** (torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -14))) - 10)
            err = (out[lo:hi].double() - want).abs()
            bound = 0.5 * step + 2.0 ** -20 * want.abs() + 2.0 ** -40
            assert bool((err <= bound).all()), (zeros, b, n_split, float((err / bound).max()))


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("zeros", [[1, -5, 300, -1000, 7], [1023, 1024, 1025, 1026, 1027], [-1021, -1024, -1025, -2045, -2047], [2047, 2048, 2049, 3583, 3584],
                                   [4095, -4096, 10000, -20001, 12345], [32767, -32768, 1025, -32767, 31743]])
def test_zero_points_are_exact(zeros, G):
    _equal_weights(G, zeros, (2.0 ** -6, 2.0 ** -7))


@pytest.mark.parametrize("scales", [(1.5, 1.0), (1.0, 1.75), (1.25, 0.75), (1.75, 0.0009765625), (0.625, 1.5)])
def test_groups_of_different_scales_are_exact(scales):
    """Values whose product with a scale of a few bits fits binary16."""
    _equal_weights(64, [1, -5, 200, -190, 7], tuple(x * 2.0 ** -6 for x in scales))
