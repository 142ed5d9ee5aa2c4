"""The angle of rotary positions at the ends of their range (akvq_rope_axes): an error of 1e-7, which is half a step of a 32-bit turn next to a half
(2^-26 turns, 9.4e-8).  Seen where a sine is close to 0, so that binary16 does not hide it; expected values from 64-bit mantissas and a
turn to 30 digits, which leave 2e-11 turns."""
import numpy as np
import pytest
import torch

from paper_2501_15021_amd import binding as akvq

TURN = np.longdouble("6.283185307179586476925286766559005768")


def angles(freq, pos):
    """(sine, cosine) in 64 bits of every frequency (binary32) at every position."""
    assert np.finfo(np.longdouble).nmant >= 63
    t = pos.astype(np.longdouble)[:, None] * freq.astype(np.longdouble)[None, :] / TURN
    r = ((t - np.rint(t)) * TURN).astype(np.float64)
    return np.sin(r), np.cos(r)


@pytest.mark.gpu
@pytest.mark.parametrize("first", [2 ** 31 - 20000, -2 ** 31, 2 ** 24, 2 ** 30 + 12345])
@pytest.mark.parametrize("inverse", [False, True])
def test_angles_of_far_positions(first, inverse):
    freq = np.linspace(0.51, 1.0, 64).astype(np.float32)
    axes = akvq.RopeAxes(freq.tolist(), [0] * 64)
    pos = np.arange(first, first + 20000, dtype=np.int64)
    sine, cosine = angles(freq, pos)
    x = torch.zeros(20000, 1, 128, dtype=torch.float16, device="cuda")
    x[..., :64] = 1.0
    out, _ = akvq.rope_axes(axes, torch.from_numpy(pos.astype(np.int32)).cuda(), x, inverse=inverse)
    torch.cuda.synchronize()
    got = out[:, 0].cpu().double().numpy()
    for want, y in ((cosine, got[:, :64]), (-sine if inverse else sine, got[:, 64:])):
        near = np.abs(want) < 1e-4
        assert near.sum() >= 30
        # half a step of binary16: 2^-11 of the value, 2^-25 below its smallest normal number; the sine itself 2^-22 of it
        bound = 1e-7 + np.abs(want) * (2.0 ** -11 + 2.0 ** -22) + 2.0 ** -25
        err = np.abs(y - want)
        assert (err[near] <= bound[near]).all(), float(err[near].max())
        assert (err <= bound).all()
