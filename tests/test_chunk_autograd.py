"""The calls for chunks and torch's recording of gradients: rotary positions record none, so rows that ask for one are refused, and what is
written into a caller's tensor counts as a change of it."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq

AXES = akvq.RopeAxes.sections(1e4, (16, 24, 24))


def _rows(heads, **kw):
    return torch.zeros(4, heads, 128, dtype=torch.float16, **kw)


@pytest.mark.parametrize("what", ["q", "k", "q_out", "k_out"])
def test_rows_that_ask_for_a_gradient_are_refused(what):
    """(On the host: what follows the refusal is that of host tensors.)"""
    pos = torch.zeros(3, 4, dtype=torch.int32)
    t = dict(q=_rows(3), k=_rows(2), q_out=_rows(3), k_out=_rows(2))
    call = lambda: akvq.rope_axes(AXES, pos, t["q"], t["k"], q_out=t["q_out"], k_out=t["k_out"])
    with pytest.raises(akvq.AkvqError, match="current device"):
        call()
    t[what].requires_grad_()
    with pytest.raises(akvq.AkvqError, match=what + ".*gradient"):
        call()
    t[what] = _rows(t[what].shape[1], requires_grad=True) * 2  # no leaf
    with pytest.raises(akvq.AkvqError, match=what + ".*gradient"):
        call()
    for off in (torch.no_grad, torch.inference_mode):
        with off(), pytest.raises(akvq.AkvqError, match="current device"):
            call()


@pytest.mark.gpu
def test_the_gradient_as_a_program_writes_it():
    """A function of its own, whose backward pass is the inverse."""
    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos):
            ctx.save_for_backward(pos)
            return akvq.rope_axes(AXES, pos, x)[0]

        @staticmethod
        def backward(ctx, g):
            return akvq.rope_axes(AXES, ctx.saved_tensors[0], g, inverse=True)[0], None

    pos = torch.randint(0, 9000, (3, 4), dtype=torch.int32, device="cuda")
    x, g = (torch.randn(4, 3, 128, device="cuda").half() for _ in range(2))
    leaf = x.clone().requires_grad_()
    y = Turn.apply(leaf, pos)
    y.backward(g)
    assert torch.equal(y.detach(), akvq.rope_axes(AXES, pos, x)[0])
    assert torch.equal(leaf.grad, akvq.rope_axes(AXES, pos, g, inverse=True)[0])


@pytest.mark.gpu
def test_what_is_written_counts_as_changed():
    """Rows that another operation keeps for its gradient, turned in place: its backward pass is refused instead of wrong."""
    pos = torch.randint(0, 9000, (3, 4), dtype=torch.int32, device="cuda")
    x = torch.randn(4, 5, 128, device="cuda").half()
    w = torch.ones(5, 128, dtype=torch.float16, device="cuda", requires_grad=True)
    y = (x * w).float().sum()   # keeps x
    akvq.rope_axes(AXES, pos, x[:, :3], x[:, 3:], q_out=x[:, :3], k_out=x[:, 3:])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    before = x._version
    akvq.rope_axes(AXES, pos, x[:, :3])  # into a new tensor
    assert x._version == before
    cache = akvq.PagedCache(1, 2, 128, 2, 2, fill=0)
    out, lse = torch.zeros(4, 2, 128, dtype=torch.float16, device="cuda"), torch.zeros(4, 2, device="cuda")
    versions = out._version, lse._version
    akvq.paged_attention(cache, x[:, :2], x[:, :2], x[:, 2:4], torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4, 0.1, out=out, lse=lse)
    assert out._version > versions[0] and lse._version > versions[1]
    with torch.inference_mode():
        kept = torch.zeros_like(out)
    akvq.rope_axes(AXES, pos, out, q_out=kept)  # has no count
    with torch.inference_mode():
        akvq.rope_axes(AXES, pos, out, q_out=out)
    torch.cuda.synchronize()
