"""The calls that turn rows and torch's forward-mode derivatives: they carry none, so rows that have a tangent are refused, as rows that ask for a gradient are."""
import pytest
import torch
import torch.autograd.forward_ad as forward

from paper_2501_15021_amd import binding as akvq

POS = torch.zeros(3, 4, dtype=torch.int32)
START = torch.tensor([0, 4], dtype=torch.int32)
AXES = akvq.RopeAxes.sections(1e4, (16, 24, 24))
ROTARY = akvq.Rotary([1.0] * 32, [0, 1, 2, 0] * 8, 64)


def append_rotary(pos, q, k, **outs):
    return akvq.paged_append_rotary(akvq.PagedCache(1, 2, 128, 2, 2, device="cpu", fill=0, bits=4), ROTARY, pos, q, k, torch.zeros_like(k), START, 4, 1.0, **outs)


CALLS = dict(rope_axes=lambda *a, **kw: akvq.rope_axes(AXES, *a, **kw), rotary_rows=lambda *a, **kw: akvq.rotary_rows(ROTARY, *a, **kw),
             paged_append_rotary=append_rotary)


def _rows(heads):
    return torch.ones(4, heads, 128, dtype=torch.float16)


@pytest.mark.parametrize("what", ["q", "k", "q_out", "k_out"])
@pytest.mark.parametrize("call", sorted(CALLS))
def test_rows_with_a_tangent_are_refused(call, what):
    """(On the host: what follows the refusal is that of host tensors.)"""
    t = dict(q=_rows(3), k=_rows(2), q_out=_rows(3), k_out=_rows(2))
    turn = lambda: CALLS[call](POS, t["q"], t["k"], q_out=t["q_out"], k_out=t["k_out"])
    with pytest.raises(akvq.AkvqError, match="current device"):
        turn()
    plain = t[what]
    with forward.dual_level():
        t[what] = forward.make_dual(plain, torch.ones_like(plain))
        for off in (torch.enable_grad, torch.no_grad):  # no_grad stops the recording of gradients alone
            with off(), pytest.raises(akvq.AkvqError, match=what + ".*tangent"):
                turn()
        t[what] = t[what].flatten().view(plain.shape)  # not the one that was made, but what comes of it
        with pytest.raises(akvq.AkvqError, match=what + ".*tangent"):
            turn()
        t[what] = forward.unpack_dual(t[what]).primal
        with pytest.raises(akvq.AkvqError, match="current device"):
            turn()
        t[what] = forward.make_dual(plain, torch.ones_like(plain))
        with torch.inference_mode(), pytest.raises(akvq.AkvqError, match="current device"):
            turn()
    with pytest.raises(akvq.AkvqError, match="current device"):  # a tangent ends with its level
        turn()


@pytest.mark.gpu
def test_the_tangent_as_a_program_writes_it():
    """The map is linear: a tangent turns as the rows do."""
    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(x, pos):
            return akvq.rotary_rows(ROTARY, pos, x)[0]

        @staticmethod
        def setup_context(ctx, inputs, output):
            ctx.save_for_forward(inputs[1])

        @staticmethod
        def jvp(ctx, tangent, _):
            return akvq.rotary_rows(ROTARY, ctx.saved_tensors[0], tangent)[0]

    pos = torch.randint(0, 9000, (3, 4), dtype=torch.int32, device="cuda")
    x, d = (torch.randn(4, 3, 128, device="cuda").half() for _ in range(2))
    with forward.dual_level():
        dual = forward.make_dual(x, d)
        with pytest.raises(akvq.AkvqError, match="tangent"):
            akvq.rotary_rows(ROTARY, pos, dual)
        got = forward.unpack_dual(Turn.apply(dual, pos))
    assert torch.equal(got.primal, akvq.rotary_rows(ROTARY, pos, x)[0]) and torch.equal(got.tangent, akvq.rotary_rows(ROTARY, pos, d)[0])
