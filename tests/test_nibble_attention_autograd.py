"""Attention over pages of 4-bit codes and torch's recording of derivatives: it records no gradient and carries no tangent, so rows that ask for one are refused
instead of answered without."""
import pytest
import torch
import torch.autograd.forward_ad as forward

from paper_2501_15021_amd import binding as akvq

START = torch.tensor([0, 4], dtype=torch.int32)


def _call(bits, **kw):
    t = dict(q=torch.ones(4, 4, 128, dtype=torch.float16), k=torch.ones(4, 2, 128, dtype=torch.float16), v=torch.ones(4, 2, 128, dtype=torch.float16))
    t.update(kw)
    cache = akvq.PagedCache(1, 2, 128, 2, 2, device="cpu", fill=0, bits=bits)
    return akvq.paged_attention(cache, t.pop("q"), t.pop("k"), t.pop("v"), START, 4, 0.1, **t)


def _tensor(what):
    shape = dict(q=(4, 4, 128), out=(4, 4, 128), lse=(4, 4)).get(what, (4, 2, 128))
    return torch.ones(shape, dtype=torch.float32 if what == "lse" else torch.float16)


@pytest.mark.parametrize("what", ["q", "k", "v", "out", "lse"])
def test_rows_that_ask_for_derivatives_are_refused(what):
    """(On the host: what follows the refusal is that of host tensors.)"""
    with pytest.raises(akvq.AkvqError, match="current device"):
        _call(4, **{what: _tensor(what)})
    leaf = _tensor(what).requires_grad_()
    for x in (leaf, leaf * 2):
        with pytest.raises(akvq.AkvqError, match=what + ".*gradient"):
            _call(4, **{what: x})
        for off in (torch.no_grad, torch.inference_mode):
            with off(), pytest.raises(akvq.AkvqError, match="current device"):
                _call(4, **{what: x})
    with forward.dual_level():
        dual = forward.make_dual(_tensor(what), _tensor(what))
        for off in (torch.enable_grad, torch.no_grad):
            with off(), pytest.raises(akvq.AkvqError, match=what + ".*tangent"):
                _call(4, **{what: dual})
        with torch.inference_mode(), pytest.raises(akvq.AkvqError, match="current device"):
            _call(4, **{what: dual})


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_pages_of_2_bit_codes_take_them_as_they_did(what):
    with pytest.raises(akvq.AkvqError, match="current device"):
        _call(2, **{what: _tensor(what).requires_grad_()})


@pytest.mark.gpu
def test_without_recording_it_answers():
    x = torch.randn(4, 8, 128, device="cuda").half()
    cache = akvq.PagedCache(1, 2, 128, 2, 2, fill=0, bits=4)
    start = START.cuda()
    call = lambda y: akvq.paged_attention(cache, y[:, :4], y[:, 4:6], y[:, 6:], start, 4, 0.1)
    want, leaf = call(x), x.clone().requires_grad_()
    with pytest.raises(akvq.AkvqError, match="gradient"):
        call(leaf)
    with torch.no_grad():
        got = call(leaf)
    assert torch.equal(got, want) and torch.equal(call(leaf.detach()), want)
