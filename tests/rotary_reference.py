"""Rotary positions of rows from their formula in 64 bits."""
import torch


def turned64(x, pos, freq, axis, dim, interleaved, magnitude=1.0, inverse=False):
    """Rows x [n, heads, 128] turned, and what bounds an element's rounding: the sum of what its two products are of, both [n, heads, 128].  pos
    [axes, n]; freq, axis: of every pair.  (Angles are exact: a position below 2^29 times a 32-bit frequency fits 53 bits.)"""
    y, size = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    for i in range(dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
        f = torch.tensor(freq[i], dtype=torch.float32).double().item()
        angle = pos[axis[i]].double()[:, None] * f
        c, s = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if inverse else 1)
        u, v = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
        size[..., a], size[..., b] = (u * c).abs() + (v * s).abs(), (v * c).abs() + (u * s).abs()
    return y, size


def check_turned(got, x, pos, freq, axis, dim, interleaved, magnitude=1.0, inverse=False):
    """Sine and cosine are rounded to 32 bits (2^-24 of them), so is one product and the sum (2^-24 of what it is of, twice): 2^-22 of the
    two products' sizes covers them; the result is rounded to binary16: 2^-11 of it, 2^-25 where it is below the smallest normal number.
    Channels that do not turn are the same bits."""
    want, size = turned64(x, pos, freq, axis, dim, interleaved, magnitude, inverse)
    err = (got.double() - want).abs()
    bound = 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -21 * size
    assert bool((err <= bound).all()), float((err / bound).max())
    assert torch.equal(got[..., dim:].view(torch.int16), x[..., dim:].contiguous().view(torch.int16))
