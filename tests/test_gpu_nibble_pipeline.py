"""The calls around pages of 4-bit codes as a server uses them: a chunk turned and stored in one call, attention over the pages and the chunk, the lengths
advanced; prompts in chunks of unequal length, then generated tokens, eager and captured; two captured programs side by side."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from nibble_inputs import check_attention, sequences
from paged_inputs import Sequences

pytestmark = pytest.mark.gpu
SM, CLIP = 1 / math.sqrt(128), 1.0
B, HQ, HKV = 3, 8, 2
POOLS = ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")
PLANS = {"half": akvq.Rotary([1e6 ** (-i / 64) for i in range(64)], [0] * 16 + [1] * 24 + [2] * 24),
         "next": akvq.Rotary([1e4 ** (-i / 32) for i in range(32)], [i % 3 for i in range(32)], 64, True, 1.1)}


class Server:
    """Sequences whose rows arrive chunk by chunk (sequences draws them all at once, as new rows, and owns the pages)."""

    def __init__(self, totals, G, bits, seed=0):
        self.s = sequences([0] * B, totals, HKV, G, 64, Hq=HQ, salient=[0, 1, 2, 30, 31, 90, 91, 140], seed=seed, bits=bits)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.pos = torch.randint(0, 4000, (3, self.s.n), generator=g, device="cuda", dtype=torch.int32)
        self.s.cache.seq_len.zero_()

    def chunk(self, take):
        """The next take[b] rows of every sequence as one packed projection, and their positions."""
        at = self.s.cache.seq_len.tolist()
        rows = [r for b in range(B) for r in range(self.s.starts[b] + at[b], self.s.starts[b] + at[b] + take[b])]
        starts = [0]
        for n in take:
            starts.append(starts[-1] + n)
        return self.s.x[rows].clone(), self.pos[:, rows].contiguous(), torch.tensor(starts, dtype=torch.int32, device="cuda")


def parts(x):
    return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]


def step(cache, plan, x, pos, row_start, max_rows, out, lse=None):
    """In place: the rows are stored first, and count as the chunk's own, since seq_len is advanced behind the attention."""
    q, k, v = parts(x)
    akvq.paged_append_rotary(cache, plan, pos, q, k, v, row_start, max_rows, CLIP, q_out=q, k_out=k)
    akvq.paged_attention(cache, q, k, v, row_start, max_rows, SM, out=out, lse=lse)
    cache.seq_len.add_(row_start[1:] - row_start[:-1])


def _view(srv, x, take, lens):
    """What the formula looks at: the pages as they were, and the chunk with its positions in."""
    v = Sequences.__new__(Sequences)
    v.__dict__.update(srv.s.__dict__)
    starts = [0]
    for n in take:
        starts.append(starts[-1] + n)
    v.lens, v.rows, v.starts, v.n, v.x = lens, take, starts, starts[-1], x
    v.q, v.k, v.v = parts(x)
    return v


@pytest.mark.parametrize("layout", ["half", "next"])
@pytest.mark.parametrize("G", [128, 64])
def test_chunks_then_tokens(G, layout):
    srv, plan = Server([150, 97, 40], G, 4), PLANS[layout]
    cache = srv.s.cache
    for take in ([40, 97, 0], [33, 0, 37], [70, 0, 1], [1, 0, 1], [1, 0, 1]):
        x, pos, starts = srv.chunk(take)
        lens = cache.seq_len.tolist()
        out, lse = torch.zeros(x.shape[0], HQ, 128, dtype=torch.float16, device="cuda"), torch.zeros(x.shape[0], HQ, device="cuda")
        step(cache, plan, x, pos, starts, max(take), out, lse)
        torch.cuda.synchronize()
        assert cache.seq_len.tolist() == [a + b for a, b in zip(lens, take)]
        check_attention(_view(srv, x, take, lens), out, lse, SM, str(take))  # (rows behind lens have changed: none of them is read)
    # the pages now hold what the calls one after the other write of every sequence's rows at once
    whole = Server([150, 97, 40], G, 4)
    x = whole.s.x.clone()
    q, k, v = parts(x)
    akvq.rotary_rows(plan, whole.pos, q, k, q_out=q, k_out=k)
    rows = [r for b, n in enumerate(cache.seq_len.tolist()) for r in range(whole.s.starts[b], whole.s.starts[b] + n)]
    starts = torch.tensor([0, 145, 242, 282], dtype=torch.int32, device="cuda")
    assert cache.seq_len.tolist() == [145, 97, 40]
    akvq.paged_append(whole.s.cache, k[rows], v[rows], starts, 150, CLIP)
    torch.cuda.synchronize()
    for name in POOLS:
        assert torch.equal(getattr(cache, name), getattr(whole.s.cache, name)), name


@pytest.mark.parametrize("bits", [2, 4])
def test_tokens_in_two_graphs(bits):
    """The step of one token of two programs, each captured once, with its split attention, and replayed in turn while pages fill up: every replay
    against the eager step, with eager work in between."""
    n, starts = 5, torch.arange(B + 1, dtype=torch.int32, device="cuda")
    programs = []
    for seed, totals, layout in ((3, [1300, 700, 40], "half"), (4, [900, 33, 1500], "next")):
        eager, srv = (Server(totals, 64, bits, seed=seed) for _ in range(2))
        outs = []
        for x in (eager, srv):
            first = [t - n for t in totals]
            data, pos, rs = x.chunk(first)
            step(x.s.cache, PLANS[layout], data, pos, rs, max(first), torch.empty(data.shape[0], HQ, 128, dtype=torch.float16, device="cuda"))
        for _ in range(n):
            data, pos, _ = eager.chunk([1] * B)
            out = torch.zeros(B, HQ, 128, dtype=torch.float16, device="cuda")
            step(eager.s.cache, PLANS[layout], data, pos, starts, 1, out)
            outs.append(out)
        torch.cuda.synchronize()
        data, pos, _ = srv.chunk([1] * B)
        x_in, pos_in, out = torch.empty_like(data), torch.empty_like(pos), torch.zeros(B, HQ, 128, dtype=torch.float16, device="cuda")
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(srv.s.cache, PLANS[layout], x_in, pos_in, starts, 1, out)
        programs.append((eager, srv, outs, x_in, pos_in, out, graph))
    split = akvq.lib().akvq_paged_default_splits if bits == 2 else akvq.lib().akvq_paged_nibble_default_splits
    assert split(akvq.C.byref(programs[0][1].s.cache.paged_struct()), HQ, 1) > 1
    for i in range(n):
        for _, srv, outs, x_in, pos_in, out, graph in programs:
            data, pos, _ = srv.chunk([1] * B)
            x_in.copy_(data)
            pos_in.copy_(pos)
            out.fill_(float("nan"))
            torch.randn(1 << 20, device="cuda").sum().item()
        for *_, graph in programs:
            graph.replay()
        torch.cuda.synchronize()
        for _, _, outs, _, _, out, _ in programs:
            assert torch.equal(out, outs[i]), i
    for eager, srv, *_ in programs:
        for name in POOLS + ("seq_len",):
            assert torch.equal(getattr(srv.s.cache, name), getattr(eager.s.cache, name)), name


def test_a_captured_chunk_while_rows_and_lengths_change():
    """One capture for chunks of up to 70 rows, replayed over other shares of the rows and other lengths."""
    a, b = (sequences([100, 5, 60], [70, 33, 40], HKV, 128, 32, Hq=HQ, salient=[3, 101, 130], seed=8) for _ in range(2))
    plan, pos = PLANS["half"], torch.randint(0, 9000, (3, a.n), dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(x.contiguous()) for x in (a.q, a.k)]
    call = lambda s, q, k: akvq.paged_append_rotary(s.cache, plan, pos, s.q, s.k, s.v, s.row_start, 70, CLIP, q_out=q, k_out=k)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(a, *outs)
    for lens, starts in (([100, 5, 60], [0, 70, 103, 143]), ([31, 0, 32], [0, 1, 1, 60]), ([0, 0, 0], [10, 50, 90, 143]), ([64, -2, 1], [0, 0, 0, 70])):
        want = [torch.full_like(x, 7.0) for x in outs]
        for s in (a, b):
            s.cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
            s.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
        for x in outs:
            x.fill_(7.0)
        graph.replay()
        call(b, *want)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), lens
        for name in POOLS:
            assert torch.equal(getattr(a.cache, name), getattr(b.cache, name)), (lens, name)


def test_the_gradient_as_a_program_writes_it():
    """A function of its own, whose backward pass is the inverse; and what is written into a caller's tensor counts as a change of it."""
    plan = PLANS["next"]

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos):
            ctx.save_for_backward(pos)
            return akvq.rotary_rows(plan, pos, x)[0]

        @staticmethod
        def backward(ctx, g):
            return akvq.rotary_rows(plan, ctx.saved_tensors[0], g.contiguous(), inverse=True)[0], None

    pos = torch.randint(0, 9000, (3, 4), dtype=torch.int32, device="cuda")
    x, g = (torch.randn(4, 3, 128, device="cuda").half() for _ in range(2))
    leaf = x.clone().requires_grad_()
    y = Turn.apply(leaf, pos)
    y.backward(g)
    assert torch.equal(y.detach(), akvq.rotary_rows(plan, pos, x)[0])
    assert torch.equal(leaf.grad, akvq.rotary_rows(plan, pos, g, inverse=True)[0])
    x = torch.randn(4, HQ + 2 * HKV, 128, device="cuda").half()
    w = torch.ones(HQ + 2 * HKV, 128, dtype=torch.float16, device="cuda", requires_grad=True)
    kept = (x * w).float().sum()
    cache = akvq.PagedCache(1, HKV, 128, 2, 2, fill=0, bits=4)
    starts = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    q, k, v = parts(x)
    akvq.paged_append_rotary(cache, plan, pos, q, k, v, starts, 4, CLIP, q_out=q, k_out=k)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    torch.cuda.synchronize()


def test_calls_on_another_stream():
    """The current stream's, not the default one's: what is queued there in front is seen."""
    plan, side = PLANS["half"], torch.cuda.Stream()
    a, b = (sequences([10, 40], [33, 1], HKV, 64, 32, Hq=HQ, seed=2) for _ in range(2))
    pos = torch.randint(0, 9000, (3, a.n), dtype=torch.int32, device="cuda")
    for s in (a, b):
        s.cache.seq_len.copy_(torch.tensor([10, 40], dtype=torch.int32))
    want = akvq.paged_append_rotary(a.cache, plan, pos, a.q, a.k, a.v, a.row_start, 33, CLIP)
    x = b.x.clone()
    b.x.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(10):
            big = big @ big * 1e-3
        b.x.copy_(x)
        got = akvq.paged_append_rotary(b.cache, plan, pos, b.q, b.k, b.v, b.row_start, 33, CLIP)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for name in POOLS:
        assert torch.equal(getattr(a.cache, name), getattr(b.cache, name)), name


def test_selection_into_pages_of_4_bit_codes():
    """select_salient writes the lists of such a cache as of any other."""
    T = 300
    g = torch.Generator(device="cuda").manual_seed(5)
    k, tail = torch.randn(2, 2, T, 128, generator=g, device="cuda").half(), torch.randn(2, 4, 64, 128, generator=g, device="cuda").half()
    caches = [akvq.PagedCache(2, 2, 128, 12, 5, 64, S_cap=64, bits=bits) for bits in (2, 4)]
    for c in caches:
        akvq.select_salient(c, mode=akvq.MODE_PSA, q_tail=tail, k=k, top_k=12, sm_scale=SM)
    torch.cuda.synchronize()
    assert torch.equal(caches[0].counts(), caches[1].counts()) and torch.equal(caches[0].sal_idx[:, :, :12], caches[1].sal_idx[:, :, :12])


def test_pools_of_another_kind_are_refused():
    s = sequences([10], [2], HKV, 128, Hq=HQ)
    two = Sequences([10], [2], HKV, 128, Hq=HQ).cache
    s.cache.k_codes = two.k_codes
    with pytest.raises(akvq.AkvqError, match="no pool of 4-bit codes"):
        akvq.paged_append(s.cache, s.k, s.v, s.row_start, 2, CLIP)
    with pytest.raises(akvq.AkvqError, match="no pool of 4-bit codes"):
        akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, 2, SM)


def test_pools_of_two_kinds_are_refused():
    s = sequences([10], [2], HKV, 128, Hq=HQ)
    s.cache.v_codes = Sequences([10], [2], HKV, 128, Hq=HQ).cache.v_codes
    pos = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(akvq.AkvqError, match="v_codes is no pool of 4-bit codes"):
        akvq.paged_append_rotary(s.cache, PLANS["half"], pos, s.q, s.k, s.v, s.row_start, 2, CLIP)
    with pytest.raises(akvq.AkvqError, match="v_codes is no pool of 4-bit codes"):
        akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, 2, SM)


def test_a_cache_that_describes_itself():
    """... is asked, and says how many bits a code has."""
    class Own(akvq.PagedCache):
        def paged_struct(self):
            asked.append(self)
            return super().paged_struct()

    asked = []
    s = sequences([70, 3], [2, 1], HKV, 128, Hq=HQ).fill_pages(clip=1.0)
    call = lambda: akvq.paged_attention(s.cache, s.q, s.k, s.v, s.row_start, 2, SM)
    want = call()
    s.cache.__class__ = Own
    assert torch.equal(call(), want) and asked == [s.cache]
