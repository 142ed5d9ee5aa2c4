"""Rotary positions with several axes (akvq_rope_axes, akvq_rope_axes_table) against the formula in 64 bits.

Bound on an element: cosine and sine are within 2e-7 (32-bit functions of an angle whose whole turns were dropped in 64 bits; up to
2^20 the angle itself adds under 1e-9, at 2^31 under 1e-6), two products and a sum in 32 bits add 2^-23 of |x| + |y|, and the result
is rounded to binary16 once: half a step, 2^-11 of it (2^-25 where it is below the smallest normal number)."""
import numpy as np
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paper_2501_15021_amd import synth

pytestmark = pytest.mark.gpu
AXES = akvq.RopeAxes.sections(1e6, (16, 24, 24))
MIXED = akvq.RopeAxes.sections(1e4, (24, 20, 20), interleaved=True)
PLAIN = akvq.RopeAxes.sections(1e4, (64,))


def _formula(axes, pos, x, inverse=False):
    f = torch.tensor(list(axes._struct.inv_freq), dtype=torch.float64)
    a = pos.cpu().double().reshape(-1, pos.shape[-1])[list(axes._struct.axis)].t() * f * (-1 if inverse else 1)
    lo, hi = x.cpu().double()[..., :64], x.cpu().double()[..., 64:]
    c, s = a.cos()[:, None], a.sin()[:, None]
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1), (lo.abs() + hi.abs()).repeat(1, 1, 2)


def _close(got, want, size, angle=1e-9):
    err = (got.cpu().double() - want).abs()
    bound = want.abs() * 2.0 ** -11 + 2.0 ** -25 + size * (2e-7 + 2.0 ** -23 + angle)
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 63, 257, 4099])
@pytest.mark.parametrize("Hq,Hkv", [(32, 32), (28, 4), (7, 1), (9, 0), (0, 5)])
@pytest.mark.parametrize("axes", [AXES, MIXED, PLAIN])
def test_rows_of_a_fused_projection(rows, Hq, Hkv, axes):
    g = torch.Generator(device="cuda").manual_seed(rows * 100 + Hq)
    x = torch.randn(rows, Hq + 2 * Hkv + 1, 128, generator=g, device="cuda").half()  # longer rows than q and k together
    pos = torch.randint(-50, 1 << 20, (3, rows), generator=g, device="cuda", dtype=torch.int32)[: axes.n_axes]
    before = x.clone()
    q, k = (x[:, :Hq] if Hq else None), (x[:, Hq:Hq + Hkv] if Hkv else None)
    for inverse in (False, True):
        outs = akvq.rope_axes(axes, pos, q, k, inverse=inverse)
        torch.cuda.synchronize()
        for got, given in zip(outs, (q, k)):
            assert (got is None) == (given is None)
            if given is not None:
                _close(got, *_formula(axes, pos, given, inverse))
    assert torch.equal(x, before)
    akvq.rope_axes(axes, pos, q, k, q_out=q, k_out=k)  # in place: the rest of the rows stays
    torch.cuda.synchronize()
    for given, old in ((q, before[:, :Hq]), (k, before[:, Hq:Hq + Hkv])):
        if given is not None:
            _close(given, *_formula(axes, pos, old))
    assert torch.equal(x[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_far_positions_and_the_ends_of_the_numbers():
    pos = torch.tensor([[0, 1, 2 ** 31 - 1, -2 ** 31, 12345678, 7], [0, 5, 2 ** 30, -1, 99999, 7], [3, 0, 2 ** 31 - 2, 1, -5, 7]],
                       dtype=torch.int32, device="cuda")
    x = torch.randn(6, 2, 128, device="cuda").half()
    x[5, 0, :] = 6e-8   # the smallest numbers
    x[5, 1, :] = 40000.0
    out, _ = akvq.rope_axes(AXES, pos, x)
    torch.cuda.synchronize()
    want, size = _formula(AXES, pos, x)
    fits = want.abs() < 65504
    _close(torch.where(fits.cuda(), out, torch.zeros_like(out)), torch.where(fits, want, torch.zeros_like(want)), size, 1e-6)
    assert bool((out.cpu()[want.abs() >= 65520].isinf()).all())


def test_positions_zero_and_frequency_zero_change_nothing():
    x = torch.randn(9, 3, 128, device="cuda").half()
    zero = torch.zeros(3, 9, dtype=torch.int32, device="cuda")
    assert torch.equal(akvq.rope_axes(AXES, zero, x)[0], x)
    half = akvq.RopeAxes([1.0] * 32 + [0.0] * 32, [0] * 64)  # pairs 32 to 63 stay: a partial embedding
    out, _ = akvq.rope_axes(half, torch.arange(9, dtype=torch.int32, device="cuda"), x)
    assert torch.equal(out[..., 32:64], x[..., 32:64]) and torch.equal(out[..., 96:], x[..., 96:])


def test_the_inverse_is_the_gradient():
    """y = R x, so the gradient of sum(y g) by x is R^T g: against differences of the formula and against the call."""
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 5000, (3, 4), generator=g, dtype=torch.int32)
    x = torch.randn(4, 2, 128, generator=g).half().double()
    up = torch.randn(4, 2, 128, generator=g).half()
    want = torch.empty_like(x)
    for e in range(128):
        step = torch.zeros(128, dtype=torch.float64)
        step[e] = 0.5
        hi, lo = (_formula(AXES, pos, x + d)[0] for d in (step, -step))
        want[..., e] = ((hi - lo) * up.double()).sum(-1)  # linear in x: differences of any width are exact
    got, _ = akvq.rope_axes(AXES, pos.cuda(), up.cuda(), inverse=True)
    torch.cuda.synchronize()
    _close(got, want, _formula(AXES, pos, up)[1], 1e-8)


@pytest.mark.parametrize("rows", [1, 37, 2000])
def test_tables_feed_the_fused_embedding(rows):
    pos = torch.randint(0, 1 << 18, (3, rows), device="cuda", dtype=torch.int32)
    cos, sin = akvq.rope_axes_table(AXES, pos)
    f = torch.tensor(list(AXES._struct.inv_freq), dtype=torch.float64)
    a = pos.cpu().double()[list(AXES._struct.axis)].t() * f
    for got, want in ((cos, a.cos()), (sin, a.sin())):
        assert got.shape == (rows, 64)
        err = (got.cpu().double() - want).abs()
        assert bool((err <= want.abs() * 2.0 ** -11 + 2.0 ** -25 + 2e-7).all())
    # text has one position on every axis: the tables of the plain embedding, to the rounding of a value next to a border
    p = torch.arange(rows, dtype=torch.int32, device="cuda").repeat(3, 1)
    mine = akvq.rope_axes_table(akvq.RopeAxes.sections(1e4, (16, 24, 24)), p)
    for got, want in zip(mine, synth.rope_tables(np.arange(rows))):
        step = np.maximum(np.abs(want.astype(np.float64)) * 2.0 ** -10, 2.0 ** -24)
        # (frequencies are 32-bit here and 64-bit there: 2^-24 of an angle of up to 2000)
        assert (np.abs(got.cpu().numpy().astype(np.float64) - want.astype(np.float64)) <= step + rows * 2.0 ** -24).all()


def test_another_stream_and_a_graph():
    x = torch.randn(33, 8, 128, device="cuda").half()
    pos = torch.arange(99, dtype=torch.int32, device="cuda").reshape(3, 33)
    want, _ = akvq.rope_axes(AXES, pos, x)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        akvq.rope_axes(AXES, pos, x, q_out=out)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        assert torch.equal(out, want)
        with torch.cuda.graph(graph, stream=side):
            akvq.rope_axes(AXES, pos, x, q_out=out)
    for i in range(3):
        pos.add_(1)  # read by the replay, not kept from the capture
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, akvq.rope_axes(AXES, pos, x)[0])
