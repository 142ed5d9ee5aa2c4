"""Arguments that the calls for 4-bit pages and for rotary positions in either layout refuse, on the host (no GPU: nothing is launched)."""
import ctypes as C

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from test_chunk_refusals import CHUNKS, INVALID, ODD, OK, P, POINTERS, SHAPES, UNSUPPORTED, _paged

UNALIGNED = C.c_void_p((1 << 20) + 2)


def _rotary(n=3, axis=0, f=1.0, dim=128, layout=0, magnitude=1.0, **at):
    r = akvq.akvq_rotary(n, layout, dim, magnitude, (C.c_float * 64)(*[f] * 64), (C.c_uint8 * 64)(*[axis] * 64))
    for i, x in at.get("freq", {}).items():
        r.inv_freq[i] = x
    for i, x in at.get("axes", {}).items():
        r.axis[i] = x
    return r


PLANS = [
    (dict(n=0), INVALID), (dict(n=5), UNSUPPORTED), (dict(n=2, axis=2), INVALID), (dict(f=float("inf")), INVALID), (dict(f=float("nan")), INVALID),
    (dict(magnitude=float("nan")), INVALID), (dict(magnitude=float("inf")), INVALID), (dict(layout=2), INVALID), (dict(layout=-1), INVALID),
    (dict(dim=0), UNSUPPORTED), (dict(dim=8), UNSUPPORTED), (dict(dim=24), UNSUPPORTED), (dict(dim=136), UNSUPPORTED), (dict(dim=-16), UNSUPPORTED),
    (dict(dim=144), UNSUPPORTED), (dict(dim=32, freq={15: float("nan")}), INVALID), (dict(dim=32, axes={15: 3}), INVALID)]
UNSEEN = dict(dim=32, freq={16: float("nan"), 63: float("inf")}, axes={16: 200})  # pairs that do not turn


def _rows(r=None, pos=P, pos_stride=5, rows=5, q=P, qs=256, Hq=2, k=P, ks=128, Hkv=1, qo=P, qos=256, ko=P, kos=128, flags=0):
    return akvq.lib().akvq_rotary_rows(C.byref(r or _rotary()), pos, pos_stride, rows, q, qs, Hq, k, ks, Hkv, qo, qos, ko, kos, flags, None)


@pytest.mark.parametrize("args,want", [
    (dict(pos=None), INVALID), (dict(pos=UNALIGNED), INVALID), (dict(pos_stride=4), INVALID), (dict(rows=-1), INVALID),
    (dict(rows=(1 << 25) + 1, pos_stride=1 << 26), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=ODD), INVALID), (dict(qs=248), INVALID),
    (dict(qs=260), INVALID), (dict(Hq=-1), INVALID), (dict(Hq=70000), UNSUPPORTED), (dict(k=None), INVALID), (dict(k=ODD), INVALID), (dict(ks=120), INVALID),
    (dict(Hkv=-1), INVALID), (dict(Hkv=70000), UNSUPPORTED), (dict(qo=None), INVALID), (dict(qo=ODD), INVALID), (dict(qos=255), INVALID),
    (dict(ko=None), INVALID), (dict(kos=64), INVALID), (dict(qs=512, qos=256), INVALID), (dict(Hq=0, Hkv=0), INVALID), (dict(flags=1), INVALID),
    (dict(flags=64), INVALID), (dict(rows=0), OK), (dict(rows=0, pos=None, q=None, k=None, qo=None, ko=None), OK), (dict(rows=0, r=_rotary(**UNSEEN)), OK)])
def test_rotary_rows(args, want):
    assert _rows(**args) == want


@pytest.mark.parametrize("plan,want", PLANS)
def test_plans(plan, want):
    assert _rows(r=_rotary(**plan)) == want and _rows(r=_rotary(**plan), rows=0) == want
    assert _turn(r=_rotary(**plan)) == want
    assert akvq.lib().akvq_rotary_rows(None, P, 5, 5, P, 256, 2, P, 128, 1, P, 256, P, 128, 0, None) == INVALID


def _turn(c=None, bits=4, rows=(P, 5, 5), r=None, pos=P, pos_stride=5, q=P, qs=1024, Hq=8, k=P, ks=512, v=P, vs=512, qo=P, qos=1024, ko=P, kos=512, clip=1.0,
          flags=0):
    return akvq.lib().akvq_paged_append_rotary(C.byref(c or _paged()), bits, C.byref(akvq.akvq_chunk(*rows)), C.byref(r or _rotary()), pos, pos_stride, q, qs,
                                               Hq, k, ks, v, vs, qo, qos, ko, kos, clip, flags, None)


def test_paged_append_rotary():
    for kw, want in SHAPES + POINTERS:
        assert _turn(_paged(**kw)) == want, kw
    for rows, want in CHUNKS:
        assert _turn(rows=rows) == want, rows
    for kw in (dict(pos=None), dict(pos=UNALIGNED), dict(pos_stride=4), dict(q=None), dict(q=ODD), dict(qs=1016), dict(qs=1028), dict(Hq=-1), dict(k=None),
               dict(k=ODD), dict(ks=504), dict(v=None), dict(v=ODD), dict(vs=504), dict(qo=None), dict(qo=ODD), dict(qos=1016), dict(ko=None), dict(ko=ODD),
               dict(kos=504), dict(qs=2048, qos=1024), dict(ks=1024, kos=512), dict(clip=0.0), dict(clip=1.5), dict(clip=float("nan")),
               dict(flags=akvq.K_PREROTATED), dict(flags=2), dict(flags=32)):
        assert _turn(**kw) == INVALID, kw
    for bits in (0, 1, 3, 8, -4):
        assert _turn(bits=bits) == UNSUPPORTED
    assert _turn(Hq=70000, qs=70000 * 128, qos=70000 * 128) == UNSUPPORTED
    assert _turn(rows=(P, 0, 5), q=None, k=None, v=None, qo=None, ko=None, pos=None) == OK
    assert akvq.lib().akvq_paged_append_rotary(None, 4, C.byref(akvq.akvq_chunk(P, 5, 5)), C.byref(_rotary()), P, 5, P, 1024, 8, P, 512, P, 512, P, 1024, P,
                                               512, 1.0, 0, None) == INVALID
    assert akvq.lib().akvq_paged_append_rotary(C.byref(_paged()), 4, None, C.byref(_rotary()), P, 5, P, 1024, 8, P, 512, P, 512, P, 1024, P, 512, 1.0, 0,
                                               None) == INVALID


def test_nibble_bytes():
    sizes = (C.c_size_t * 8)()
    assert akvq.lib().akvq_paged_nibble_bytes(C.byref(_paged()), sizes) == OK
    assert list(sizes) == [5 * 4 * 64 * 64] * 2 + [5 * 4 * 64 * 4] * 2 + [8 * 64 * 256] * 2 + [8 * 64 * 4, 32]
    assert akvq.lib().akvq_paged_nibble_bytes(C.byref(_paged(G=64)), sizes) == OK and sizes[2] == 5 * 4 * 64 * 8
    assert akvq.lib().akvq_paged_nibble_bytes(C.byref(_paged()), None) == INVALID
    for kw, want in SHAPES:
        assert akvq.lib().akvq_paged_nibble_bytes(C.byref(_paged(**kw)), sizes) == want, kw


def test_nibble_append():
    def call(c=None, rows=(P, 5, 5), k=P, ks=512, v=P, vs=512, clip=0.8, flags=0):
        return akvq.lib().akvq_paged_nibble_append(C.byref(c or _paged()), C.byref(akvq.akvq_chunk(*rows)), k, ks, v, vs, clip, flags, None)
    for kw, want in SHAPES + POINTERS:
        assert call(_paged(**kw)) == want, kw
    for rows, want in CHUNKS:
        assert call(rows=rows) == want, rows
    for kw in (dict(k=None), dict(k=ODD), dict(ks=504), dict(ks=516), dict(v=None), dict(v=ODD), dict(vs=0), dict(clip=0.0), dict(clip=1.5),
               dict(clip=float("nan")), dict(flags=2), dict(flags=16), dict(flags=32)):
        assert call(**kw) == INVALID, kw


def test_nibble_attention():
    def call(c=None, rows=(P, 5, 5), q=P, qs=1024, Hq=8, k=P, ks=512, v=P, vs=512, out=P, os=1024, lse=None, n_split=1, ws=None, nws=0, flags=0):
        return akvq.lib().akvq_paged_nibble_attention(C.byref(c or _paged()), C.byref(akvq.akvq_chunk(*rows)), q, qs, Hq, k, ks, v, vs, 0.1, out, os, lse,
                                                      n_split, ws, nws, flags, None)
    for kw, want in SHAPES + POINTERS:
        assert call(_paged(**kw)) == want, kw
    for rows, want in CHUNKS:
        assert call(rows=rows) == want, rows
    for kw in (dict(q=None), dict(q=ODD), dict(qs=1016), dict(qs=1028), dict(Hq=0), dict(Hq=6), dict(k=None), dict(k=ODD), dict(ks=504), dict(v=None),
               dict(v=ODD), dict(vs=504), dict(out=None), dict(out=ODD), dict(os=1016), dict(lse=UNALIGNED), dict(n_split=1025), dict(flags=1), dict(flags=4),
               dict(flags=16), dict(n_split=2), dict(n_split=2, ws=ODD, nws=1 << 30)):
        assert call(**kw) == INVALID, kw
    assert call(Hq=36, qs=36 * 128, os=36 * 128) == UNSUPPORTED
    assert call(n_split=2, ws=P, nws=akvq.lib().akvq_paged_workspace_bytes(5, 8, 2) - 1) == -4
    n = akvq.lib().akvq_paged_nibble_default_splits
    assert n(C.byref(_paged()), 6, 1) == 1 and n(None, 6, 1) == 1 and 1 <= n(C.byref(_paged(max_pages=1 << 15, max_len=1 << 20)), 8, 1) <= 64


def _cache(**kw):
    return akvq.PagedCache(2, 4, 128, 5, 3, device="cpu", fill=0, **kw)


def test_binding_of_the_cache():
    c = _cache(bits=4)
    assert c.bits == 4 and c.k_codes.shape == c.v_codes.shape == (5, 4, 2, 512) and c.v_meta.shape == (5, 4, 64, 1)
    assert _cache().bits == 2 and _cache().k_codes.shape == (5, 4, 2, 256)
    for bits in (1, 3, 8):
        with pytest.raises(akvq.AkvqError, match="bits"):
            _cache(bits=bits)
    x, start = torch.zeros(5, 4, 128, dtype=torch.float16), torch.tensor([0, 2, 5], dtype=torch.int32)
    c.bits = 3
    with pytest.raises(akvq.AkvqError, match="bits"):
        akvq.paged_append(c, x, x, start, 3, 0.8)
    with pytest.raises(akvq.AkvqError, match="bits"):
        akvq.paged_attention(c, x, x, x, start, 3, 0.1)


def test_binding_of_rotary():
    """Shapes, types and devices (host tensors here) are refused before the library is called."""
    for args in (([1.0] * 63,), ([1.0] * 64, [0] * 63), ([1.0] * 64, [4] * 64), ([1.0] * 64, [-1] * 64), ([1.0] * 64, None, 120), ([1.0] * 12, None, 24), ([], None, 0)):
        with pytest.raises(akvq.AkvqError):
            akvq.Rotary(*args)
    for args in ((1e4, 0.5), (1e4, 0.0)):
        with pytest.raises(akvq.AkvqError):
            akvq.Rotary.linear(*args)
    with pytest.raises(akvq.AkvqError):
        akvq.Rotary.yarn(1e4, 4.0, 4096, fast=1.0, slow=2.0)
    rot = akvq.Rotary([1.0] * 64, [0, 1, 2, 0] * 16)
    assert rot.n_axes == 3
    pos, x = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, 2, 128, dtype=torch.float16)
    for p, q, k, kw, why in [
            (pos, None, None, {}, "neither"), (pos, x.float(), None, {}, "fp16"), (pos, x[:, 0], None, {}, "fp16"), (pos, x, x[:3], {}, "do not fit"),
            (pos, x, None, dict(k_out=x), "without"), (pos[:2], x, None, {}, "axis and row"), (pos[:, :3], x, None, {}, "axis and row"),
            (pos.long(), x, None, {}, "int32"), (pos[0], x, None, {}, "axis and row"),
            (pos, torch.zeros(4, 4, 128, dtype=torch.float16)[:, ::2], None, {}, "next to each other"),
            (pos, x, None, dict(q_out=torch.zeros(4, 3, 128, dtype=torch.float16)), "do not fit"),
            (pos, x.clone().requires_grad_(), None, {}, "gradient"), (pos, x, None, {}, "current device")]:
        with pytest.raises(akvq.AkvqError, match=why):
            akvq.rotary_rows(rot, p, q, k, **kw)
    with pytest.raises(akvq.AkvqError, match="something else"):  # another call's axes
        akvq.rotary_rows(type("R", (), {"_struct": akvq.RopeAxes([1.0] * 64, [0] * 64)._struct}), pos, x)


def test_binding_of_paged_append_rotary():
    c, rot = _cache(bits=4), akvq.Rotary([1.0] * 64, [0] * 64)
    q, x, start, pos = (torch.zeros(5, 8, 128, dtype=torch.float16), torch.zeros(5, 4, 128, dtype=torch.float16), torch.tensor([0, 2, 5], dtype=torch.int32),
                        torch.zeros(1, 5, dtype=torch.int32))
    good = dict(pos=pos, q=q, k=x, v=x, row_start=start, max_rows=3)
    for kw, why in [(dict(q=q.float()), "fp16"), (dict(q=q[:4]), "do not fit"), (dict(k=x[:, :3]), "do not fit"), (dict(v=x[:4]), "do not fit"),
                    (dict(k=x.float()), "fp16"), (dict(k=x[:, 0]), "fp16"), (dict(pos=pos[:, :4]), "axis and row"), (dict(pos=pos.long()), "int32"),
                    (dict(row_start=start[:2]), "row_start"), (dict(max_rows=-1), "max_rows"), (dict(q=None, q_out=q), "without"),
                    (dict(q_out=q[:, :4]), "do not fit"), (dict(k_out=x[:4]), "do not fit"), (dict(flags=1 << 32), "flags"),
                    (dict(q=q.clone().requires_grad_()), "gradient"), (dict(k=x.clone().requires_grad_()), "gradient"), ({}, "current device")]:
        with pytest.raises(akvq.AkvqError, match=why):
            akvq.paged_append_rotary(c, rot, clip=1.0, **{**good, **kw})


def test_frequencies_of_stretched_contexts():
    """Against their formulas, in 64 bits; what the call gets is rounded to 32."""
    import math
    theta, dim, trained, factor = 1e4, 64, 4096, 8.0
    plain = [theta ** (-2 * i / dim) for i in range(dim // 2)]
    near = lambda got, want: all(abs(g / w - 1) < 2.0 ** -23 for g, w in zip(got, want))
    assert near(akvq.Rotary.plain(theta, dim)._struct.inv_freq, plain)
    assert near(akvq.Rotary.linear(theta, factor, dim)._struct.inv_freq, [f / factor for f in plain])
    yarn = akvq.Rotary.yarn(theta, factor, trained, dim, interleaved=True)
    assert yarn._struct.layout == akvq.ROTARY_INTERLEAVED and abs(yarn._struct.magnitude - (0.1 * math.log(factor) + 1)) < 1e-6
    want = []
    for f in plain:
        ramp = min(max((trained * f / (2 * math.pi) - 1) / 31, 0), 1)
        want.append((1 - ramp) * f / factor + ramp * f)
    assert near(yarn._struct.inv_freq, want) and want[0] == plain[0] and want[-1] == plain[-1] / factor
    assert akvq.Rotary.yarn(theta, 1.0, trained, dim)._struct.magnitude == 1.0
    assert akvq.Rotary.yarn(theta, factor, trained, dim, magnitude=0.5)._struct.magnitude == 0.5
