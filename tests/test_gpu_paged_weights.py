"""The weights of akvq_paged_attention: those of up to eight rows in a tile are rounded twice, apart from each other; and the logarithm of their
sum, in tiles of every size, changes nothing else."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, cached_rows
from tile_rule import tile_of

pytestmark = pytest.mark.gpu
TILES = [(8, 16), (48, 32), (8192, 256)]  # the caller's bound of a sequence's rows, two heads a KV head, and the tile that it brings


def _make(lens, rows, bound, tile, G, **kw):
    s = Sequences(lens, rows, 2, G, 32, Hq=4, extra_rows=8192, **kw)
    s.max_rows = bound
    assert tile_of(s, bound) == tile
    return s


def _run(s, n_split, lse=None, sm=1.0, flags=0):
    out = torch.full((s.x.shape[0], s.Hq, 128), 7.0, dtype=torch.float16, device="cuda")
    akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, sm, n_split=n_split, out=out, lse=lse, flags=flags)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("Hq,rows", [(2, 1), (4, 2), (16, 1), (6, 1)])
def test_weights_of_few_rows_are_rounded_twice(Hq, rows):
    """One cached row decides (the others, and the chunk's own, are more than 30 below it), so that the output is its value times a rounded weight
    over the sum of unrounded ones.  That factor is the same in all channels, and is where the intervals meet that their roundings leave of it.  A weight's error is, root mean square, 2.07e-4 of one rounding
    (2^-11 / 3 ** 0.5 of a number's power of two, numbers spread over their logarithm) and 1.10e-4 of the mean of two that are 1.5 * 2^-12 apart;
    of 120 weights and more it is less than 10 % off: 1.4e-4 lies between."""
    lens = [20 + b for b in range(60 if Hq < 16 else 20)]
    s = Sequences(lens, [rows] * len(lens), 2, 128, 32, Hq=Hq, seed=Hq + rows, gain=1.0)
    assert tile_of(s, s.max_rows) == 16 and Hq // 2 * rows <= 8
    for k, _ in s.past:
        k.mul_(0.01)
        k[:, 7] = 6.0  # one channel after the rotation
    s.fill_pages()
    s.x[:, :Hq] = (1.0 + torch.rand(s.n, Hq, 1, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")).half()
    s.x[:, Hq:Hq + 2] = 0
    for n_split in (1, 3):
        out = akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, s.max_rows, 0.06, n_split=n_split)
        torch.cuda.synchronize()
        errors = []
        for b, t in enumerate(lens):
            k, v, _ = cached_rows(s, b, t)
            scores = 0.06 * (s.q[s.starts[b]:s.starts[b + 1]].double().transpose(0, 1) @ k.repeat_interleave(Hq // 2, 0).transpose(1, 2).contiguous())
            first, second = scores.topk(2, dim=-1).values.unbind(-1)
            assert float(first.min()) > 30 and float((first - second).min()) > 30
            want = v[:, 7].repeat_interleave(Hq // 2, 0)
            got = out[s.starts[b]:s.starts[b + 1]].double()
            # half a step of binary16, and seven levels of 32-bit sums of the rotation and two factors, 2^-24 of the value's norm each
            half = 2.0 ** (torch.floor(torch.log2(got.abs().clamp(min=2.0 ** -14))) - 11) + 9 * 2.0 ** -24 * want.norm(dim=-1, keepdim=True)
            ends = torch.stack(((got - half) / want, (got + half) / want))
            low, high = ends.amin(0).amax(-1), ends.amax(0).amin(-1)
            assert bool((low <= high + 2.0 ** -20).all())
            errors.append(((low + high) / 2 - 1).flatten())
        errors = torch.cat(errors)
        assert len(errors) >= 120 and float(errors.square().mean().sqrt()) < 1.4e-4, float(errors.square().mean().sqrt())


@pytest.mark.parametrize("G", [128, 64])
@pytest.mark.parametrize("bound,tile", TILES)
def test_the_logarithm_changes_nothing_else(bound, tile, G):
    s = _make([300, 40, 0], [8, 3, 5], bound, tile, G, seed=4, salient=[3, 31, 40, 200]).fill_pages()
    for n_split in (1, 2, 5):
        lse = torch.zeros(s.x.shape[0], s.Hq, device="cuda")
        assert torch.equal(_run(s, n_split, lse=lse, sm=0.088), _run(s, n_split, sm=0.088)), n_split
        assert bool((lse[:s.n] != 0).all())
