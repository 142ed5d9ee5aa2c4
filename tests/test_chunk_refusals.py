"""Arguments that the chunk entry points refuse, on the host (no GPU: nothing is launched)."""
import ctypes as C

import pytest
import torch

from paper_2501_15021_amd import binding as akvq

OK, INVALID, UNSUPPORTED = 0, -1, -2
P = C.c_void_p(1 << 20)      # aligned, never read
ODD = C.c_void_p((1 << 20) + 8)


def _axes(n=3, axis=0, f=1.0):
    return akvq.akvq_axes(n, (C.c_float * 64)(*[f] * 64), (C.c_uint8 * 64)(*[axis] * 64))


def _rope(axes=None, pos=P, pos_stride=5, rows=5, q=P, qs=256, Hq=2, k=P, ks=128, Hkv=1, qo=P, qos=256, ko=P, kos=128, flags=0):
    return akvq.lib().akvq_rope_axes(C.byref(axes or _axes()), pos, pos_stride, rows, q, qs, Hq, k, ks, Hkv, qo, qos, ko, kos, flags, None)


@pytest.mark.parametrize("args,want", [
    (dict(axes=_axes(0)), INVALID), (dict(axes=_axes(5)), UNSUPPORTED), (dict(axes=_axes(2, axis=2)), INVALID),
    (dict(axes=_axes(f=float("inf"))), INVALID), (dict(axes=_axes(f=float("nan"))), INVALID),
    (dict(pos=None), INVALID), (dict(pos=C.c_void_p((1 << 20) + 2)), INVALID), (dict(pos_stride=4), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=(1 << 25) + 1, pos_stride=1 << 26), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(q=ODD), INVALID), (dict(qs=248), INVALID), (dict(qs=260), INVALID), (dict(Hq=-1), INVALID),
    (dict(k=None), INVALID), (dict(k=ODD), INVALID), (dict(ks=120), INVALID), (dict(Hkv=-1), INVALID), (dict(Hkv=70000), UNSUPPORTED),
    (dict(qo=None), INVALID), (dict(qo=ODD), INVALID), (dict(qos=255), INVALID), (dict(ko=None), INVALID), (dict(kos=64), INVALID),
    (dict(q=P, qo=P, qs=512, qos=256), INVALID),  # in place with another stride
    (dict(Hq=0, Hkv=0), INVALID), (dict(flags=1), INVALID), (dict(flags=64), INVALID),
    (dict(rows=0), OK), (dict(rows=0, pos=None, q=None, k=None, qo=None, ko=None), OK),
])
def test_rope_axes(args, want):
    assert _rope(**args) == want


def test_rope_axes_table():
    call = akvq.lib().akvq_rope_axes_table
    assert call(C.byref(_axes()), P, 5, 0, None, None, None) == OK
    assert call(None, P, 5, 5, P, P, None) == INVALID
    for cos, sin in ((None, P), (P, None), (ODD, P), (P, ODD)):
        assert call(C.byref(_axes()), P, 5, 5, cos, sin, None) == INVALID
    assert call(C.byref(_axes()), P, 3, 5, P, P, None) == INVALID


def test_binding_of_rope_axes():
    """Shapes, types and devices (host tensors here) are refused before the library is called."""
    with pytest.raises(akvq.AkvqError):
        akvq.RopeAxes([1.0] * 63, [0] * 63)
    with pytest.raises(akvq.AkvqError):
        akvq.RopeAxes([1.0] * 64, [4] * 64)
    with pytest.raises(akvq.AkvqError):
        akvq.RopeAxes.sections(1e4, (16, 24, 23))
    axes = akvq.RopeAxes.sections(1e4, (16, 24, 24))
    assert list(akvq.RopeAxes.sections(1e4, (30, 20, 14), interleaved=True)._struct.axis)[:6] == [0, 1, 2, 0, 1, 2]
    assert sorted(akvq.RopeAxes.sections(1e4, (30, 20, 14), interleaved=True)._struct.axis).count(0) == 30
    pos, x = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, 2, 128, dtype=torch.float16)
    for p, q, k, kw, why in [
            (pos, None, None, {}, "neither"), (pos, x.float(), None, {}, "fp16"), (pos, x[:, 0], None, {}, "fp16"),
            (pos, x, x[:3], {}, "do not fit"), (pos, x, None, dict(k_out=x), "without"), (pos[:2], x, None, {}, "axis and row"),
            (pos[:, :3], x, None, {}, "axis and row"), (pos.long(), x, None, {}, "int32"), (pos[0], x, None, {}, "axis and row"),
            (pos, torch.zeros(4, 4, 128, dtype=torch.float16)[:, ::2], None, {}, "next to each other"),
            (pos, x, None, dict(q_out=torch.zeros(4, 3, 128, dtype=torch.float16)), "do not fit"),
            (torch.zeros(4, 3, dtype=torch.int32).t(), x, None, {}, "next to each other"),
            (pos, x, None, {}, "current device")]:
        with pytest.raises(akvq.AkvqError, match=why):
            akvq.rope_axes(axes, p, q, k, **kw)
