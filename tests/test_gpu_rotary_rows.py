"""Rotary positions in either layout, of the whole head or part of it (rotary_rows) against the formula in 64 bits."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from rotary_reference import check_turned, turned64

pytestmark = pytest.mark.gpu


def _plan(dim, interleaved, axes=1, magnitude=1.0, theta=1e4):
    freq = [theta ** (-2 * i / dim) for i in range(dim // 2)]
    axis = [i % axes for i in range(dim // 2)]
    return akvq.Rotary(freq, axis, dim, interleaved, magnitude), (freq, axis, dim, interleaved, magnitude)


def _rows(n, heads, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, heads, 128, generator=g, device="cuda").half()


def _pos(n, axes=1, top=5000, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    return torch.randint(0, top, (axes, n), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim", list(range(16, 129, 16)))
@pytest.mark.parametrize("n,Hq,Hkv", [(1, 1, 0), (5, 28, 4), (33, 0, 2), (67, 9, 9)])
def test_against_the_formula(n, Hq, Hkv, dim, interleaved):
    rot, plan = _plan(dim, interleaved, 3, 1.25)
    x, pos = _rows(n, Hq + Hkv, dim), _pos(n, 3)
    q, k = (x[:, :Hq] if Hq else None), (x[:, Hq:] if Hkv else None)
    for inverse in (False, True):
        q2, k2 = akvq.rotary_rows(rot, pos, q, k, inverse=inverse)
        for got, rows in ((q2, q), (k2, k)):
            assert (got is None) == (rows is None)
            if rows is not None:
                check_turned(got, rows, pos, *plan, inverse=inverse)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads", [(3000, 8), (20, 300), (2, 3)])
def test_many_rows_and_heads(n, heads, interleaved):
    rot, plan = _plan(64, interleaved)
    x, pos = _rows(n, heads), _pos(n)
    check_turned(akvq.rotary_rows(rot, pos, x)[0], x, pos, *plan)


def test_the_half_layout_of_a_whole_head_is_that_of_rope_axes():
    """To a unit in the last place of binary16: they form sine and cosine apart."""
    freq, axis = [1e6 ** (-i / 64) for i in range(64)], [0] * 16 + [1] * 24 + [2] * 24
    x, pos = _rows(200, 6), _pos(200, 3, 1 << 20)
    a = akvq.rope_axes(akvq.RopeAxes(freq, axis), pos, x)[0].double()
    b = akvq.rotary_rows(akvq.Rotary(freq, axis), pos, x)[0].double()
    assert bool(((a - b).abs() <= 2.0 ** -10 * b.abs() + 2.0 ** -20 * x.double().abs().amax()).all()) and float((a != b).double().mean()) < 1e-2


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_odd_frequencies(interleaved):
    """Angles of 2^28, negative positions, frequencies of zero and below."""
    n = 64
    freq = [1.0, 0.5, -1.0, 0.0, 3.7, 1e-9] + [10.0 ** (-i / 8) for i in range(58)]
    rot = akvq.Rotary(freq, None, 128, interleaved)
    pos = torch.tensor([[(1 << 28) - 5, -(1 << 28), 0, 1, -1, 123456789, 99999, 7] * 8], dtype=torch.int32, device="cuda")
    x = _rows(n, 2)
    got = akvq.rotary_rows(rot, pos, x)[0]
    check_turned(got, x, pos, freq, [0] * 64, 128, interleaved)
    a, b = (6, 7) if interleaved else (3, 67)  # the pair of frequency 0 stays
    assert torch.equal(got[..., [a, b]], x[..., [a, b]])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim", [32, 96, 128])
def test_in_place_and_parts_of_longer_rows(dim, interleaved):
    rot, plan = _plan(dim, interleaved, 2)
    wide, pos = _rows(50, 11), _pos(50, 2)
    q, k = wide[:, 1:5], wide[:, 5:8]
    want = akvq.rotary_rows(rot, pos, q, k)
    before = wide.clone()
    got = akvq.rotary_rows(rot, pos, q, k, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, 8:], before[:, 8:])
    check_turned(want[0], before[:, 1:5], pos, *plan)


def test_rows_that_are_not_finite():
    """They stay with their pair; channels that do not turn keep their bits."""
    for interleaved in (False, True):
        rot, plan = _plan(64, interleaved)
        x, pos = _rows(6, 2), _pos(6)
        clean = akvq.rotary_rows(rot, pos, x)[0]
        bad = x.clone()
        bad[1, 0, 3], bad[2, 1, 70], bad[3, 0, 127] = float("nan"), float("inf"), float("nan")
        got = akvq.rotary_rows(rot, pos, bad)[0]
        pair = (2, 3) if interleaved else (3, 35)
        where = torch.zeros(6, 2, 128, dtype=torch.bool)
        where[1, 0, list(pair)] = True
        where[2, 1, 70] = where[3, 0, 127] = True
        assert torch.equal(got[~where.cuda()], clean[~where.cuda()]) and bool(torch.isnan(got[1, 0, list(pair)]).all())
        assert torch.equal(got[..., 64:].view(torch.int16), bad[..., 64:].contiguous().view(torch.int16))


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_gradient(interleaved):
    """The transposed rotation: against the formula's gradient in 64 bits, and against differences (the map is linear: any step serves)."""
    rot, (freq, axis, dim, _, m) = _plan(96, interleaved, 1, 1.5)
    x, g, pos = _rows(4, 3, 1), _rows(4, 3, 2), _pos(4)
    got = akvq.rotary_rows(rot, pos, g, inverse=True)[0].double()
    leaf = x.double().requires_grad_()
    y = leaf.clone()
    for i in range(dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
        f = torch.tensor(freq[i], dtype=torch.float32).double().item()
        c, s = (pos[0].double() * f).cos()[:, None] * m, (pos[0].double() * f).sin()[:, None] * m
        u, v = leaf[..., a], leaf[..., b]
        y = y.index_copy(2, torch.tensor([a, b], device="cuda"), torch.stack((u * c - v * s, v * c + u * s), -1))
    (y * g.double()).sum().backward()
    # 2^-11 of the result and 2^-21 of the products, as check_turned has it
    assert bool(((got - leaf.grad).abs() <= 2.0 ** -11 * leaf.grad.abs() + 2.0 ** -20 * g.double().abs().amax()).all())
    base = turned64(x, pos, freq, axis, dim, interleaved, m)[0]
    for e in (0, 1, 2, 47, 48, 95, 96, 127):
        step = x.double()
        step[..., e] += 0.5
        slope = ((turned64(step, pos, freq, axis, dim, interleaved, m)[0] - base) * g.double()).sum(-1) / 0.5
        assert bool(((got[..., e] - slope).abs() <= 2.0 ** -11 * slope.abs() + 2.0 ** -20 * g.double().abs().amax()).all())


def test_stretched_contexts():
    """The frequencies of the classmethods, and a turn with them."""
    x, pos = _rows(30, 2), _pos(30, 1, 100000)
    for rot, freq, magnitude in [
            (akvq.Rotary.plain(1e4, 64), [1e4 ** (-2 * i / 64) for i in range(32)], 1.0),
            (akvq.Rotary.linear(1e4, 8.0, 64), [1e4 ** (-2 * i / 64) / 8 for i in range(32)], 1.0),
            (akvq.Rotary.yarn(1e4, 4.0, 4096, 64, magnitude=1.0), None, 1.0)]:
        freq = list(rot._struct.inv_freq)[:32] if freq is None else freq
        check_turned(akvq.rotary_rows(rot, pos, x)[0], x, pos, freq, [0] * 32, 64, False, magnitude)
