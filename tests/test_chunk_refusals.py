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


def _paged(**kw):
    f = dict(B=2, Hkv=4, G=128, page_rows=64, n_pages=5, max_pages=3, S_cap=64, max_len=100)
    p = {n: P for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal", "sal_idx", "sal_cnt", "table", "seq_len")}
    for d in (f, p):
        d.update({n: v for n, v in kw.items() if n in d})
    return akvq.akvq_paged(*f.values(), *p.values())


SHAPES = [
    (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(G=32), UNSUPPORTED), (dict(page_rows=0), INVALID), (dict(page_rows=16), UNSUPPORTED),
    (dict(page_rows=96), UNSUPPORTED), (dict(page_rows=1 << 17), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(S_cap=0), INVALID), (dict(S_cap=96), INVALID), (dict(max_len=-1), INVALID), (dict(max_pages=1 << 24), UNSUPPORTED),
    (dict(B=20000), UNSUPPORTED)]
POINTERS = [(dict([(n, x)]), INVALID) for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal", "sal_idx", "sal_cnt") for x in (None, ODD)]
POINTERS += [(dict([(n, x)]), INVALID) for n in ("table", "seq_len") for x in (None, C.c_void_p((1 << 20) + 2))]
CHUNKS = [((None, 5, 5), INVALID), ((C.c_void_p((1 << 20) + 1), 5, 5), INVALID), ((P, -1, 5), INVALID), ((P, 5, -1), INVALID),
          ((P, (1 << 25) + 1, 5), UNSUPPORTED), ((P, 0, 5), OK), ((P, 5, 0), OK)]


def test_paged_bytes():
    sizes = (C.c_size_t * 8)()
    assert akvq.lib().akvq_paged_bytes(C.byref(_paged()), sizes) == OK
    assert list(sizes) == [5 * 4 * 64 * 32] * 2 + [5 * 4 * 64 * 4] * 2 + [8 * 64 * 256] * 2 + [8 * 64 * 4, 32]
    assert akvq.lib().akvq_paged_bytes(C.byref(_paged(G=64)), sizes) == OK and sizes[2] == 5 * 4 * 64 * 8
    assert akvq.lib().akvq_paged_bytes(C.byref(_paged()), None) == INVALID
    for kw, want in SHAPES:
        assert akvq.lib().akvq_paged_bytes(C.byref(_paged(**kw)), sizes) == want, kw


def test_paged_append():
    def call(c=None, rows=(P, 5, 5), k=P, ks=512, v=P, vs=512, clip=0.8, flags=0):
        return akvq.lib().akvq_paged_append(C.byref(c or _paged()), C.byref(akvq.akvq_chunk(*rows)), k, ks, v, vs, clip, flags, None)
    for kw, want in SHAPES + POINTERS:
        assert call(_paged(**kw)) == want, kw
    for rows, want in CHUNKS:
        assert call(rows=rows) == want, rows
    for kw in (dict(k=None), dict(k=ODD), dict(ks=504), dict(ks=516), dict(v=None), dict(v=ODD), dict(vs=0), dict(clip=0.0), dict(clip=1.5),
               dict(clip=float("nan")), dict(flags=2), dict(flags=16), dict(flags=32)):
        assert call(**kw) == INVALID, kw
    assert akvq.lib().akvq_paged_append(C.byref(_paged()), None, P, 512, P, 512, 0.8, 0, None) == INVALID
    assert akvq.lib().akvq_paged_append(None, C.byref(akvq.akvq_chunk(P, 5, 5)), P, 512, P, 512, 0.8, 0, None) == INVALID


def test_binding_of_paged_append():
    c = akvq.PagedCache(2, 4, 128, 5, 3, device="cpu", fill=0)
    assert c.k_codes.shape == (5, 4, 2, 256) and c.v_meta.shape == (5, 4, 64, 1) and c.max_len == 192 and bool((c.table == -1).all())
    x, start = torch.zeros(5, 4, 128, dtype=torch.float16), torch.tensor([0, 2, 5], dtype=torch.int32)
    for k, v, s, m, why in [(x.float(), x, start, 3, "fp16"), (x[:, :3], x[:, :3], start, 3, "do not fit"), (x, x[:4], start, 3, "do not fit"),
                            (x, x, start[:2], 3, "row_start"), (x, x, start.long(), 3, "row_start"), (x, x, start, -1, "max_rows"),
                            (x, x, start, 3, "current device")]:
        with pytest.raises(akvq.AkvqError, match=why):
            akvq.paged_append(c, k, v, s, m, 0.8)
    with pytest.raises(akvq.AkvqError):
        akvq.PagedCache(2, 4, 128, 5, 3, page_rows=48, device="cpu")
    # a call for contiguous caches takes no pages
    s = c.struct()
    assert akvq.lib().akvq_quantize_append(C.byref(s), P, P, 1, 0.8, 0, None) == INVALID


def test_paged_attention():
    def call(c=None, rows=(P, 5, 5), q=P, qs=1024, Hq=8, k=P, ks=512, v=P, vs=512, out=P, os=1024, lse=None, n_split=1, ws=None, nws=0, flags=0):
        return akvq.lib().akvq_paged_attention(C.byref(c or _paged()), C.byref(akvq.akvq_chunk(*rows)), q, qs, Hq, k, ks, v, vs, 0.1, out, os, lse,
                                               n_split, ws, nws, flags, None)
    for kw, want in SHAPES + POINTERS:
        assert call(_paged(**kw)) == want, kw
    for rows, want in CHUNKS:
        assert call(rows=rows) == want, rows
    for kw in (dict(q=None), dict(q=ODD), dict(qs=1016), dict(qs=1028), dict(Hq=0), dict(Hq=6), dict(k=None), dict(k=ODD), dict(ks=504), dict(v=None),
               dict(v=ODD), dict(vs=504), dict(out=None), dict(out=ODD), dict(os=1016), dict(lse=C.c_void_p((1 << 20) + 2)), dict(n_split=1025),
               dict(flags=1), dict(flags=4), dict(flags=16), dict(n_split=2), dict(n_split=2, ws=ODD, nws=1 << 30)):
        assert call(**kw) == INVALID, kw
    assert call(Hq=36, qs=36 * 128, os=36 * 128) == UNSUPPORTED
    need = akvq.lib().akvq_paged_workspace_bytes(5, 8, 2)
    assert need == 5 * 8 * 2 * 132 * 4 and akvq.lib().akvq_paged_workspace_bytes(5, 8, 1) == 0 == akvq.lib().akvq_paged_workspace_bytes(0, 8, 2)
    assert call(n_split=2, ws=P, nws=need - 1) == -4


def test_default_splits():
    L = akvq.lib()
    for B, Hkv, Hq, rows, length in ((1, 32, 32, 1, 640), (16, 32, 32, 1, 4096), (32, 4, 28, 1, 32768), (4, 8, 32, 8, 8191), (1, 1, 8, 4096, 1 << 20), (2, 2, 2, 1, 0)):
        c = _paged(B=B, Hkv=Hkv, max_pages=1 << 15, max_len=length)
        n = L.akvq_paged_default_splits(C.byref(c), Hq, rows)
        assert 1 <= n <= 32 and n <= max(1, length // 32)
    assert L.akvq_paged_default_splits(C.byref(_paged()), 6, 1) == 1 and L.akvq_paged_default_splits(None, 6, 1) == 1


def test_binding_of_paged_attention():
    c = akvq.PagedCache(2, 4, 128, 5, 3, device="cpu", fill=0)
    q, x, start = torch.zeros(5, 8, 128, dtype=torch.float16), torch.zeros(5, 4, 128, dtype=torch.float16), torch.tensor([0, 2, 5], dtype=torch.int32)
    for q_, k, v, kw, why in [(q.float(), x, x, {}, "fp16"), (q, x[:4], x, {}, "do not fit"), (q, x, x[:, :2], {}, "do not fit"),
                              (q, x, x, dict(out=q[:4]), "do not fit"), (q, x, x, dict(lse=torch.zeros(5, 4)), "lse"), (q[:, 0], x, x, {}, "fp16"),
                              (q, x, x, {}, "current device")]:
        with pytest.raises(akvq.AkvqError, match=why):
            akvq.paged_attention(c, q_, k, v, start, 3, 0.1, **kw)
