"""The chunk operators as a server uses them: positions put into a chunk's rows, attention over the pages and the chunk, the rows
written behind what is cached, the lengths advanced; prompts in chunks of unequal length, then generated tokens, eager and captured."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, check_attention

pytestmark = pytest.mark.gpu
SM, CLIP = 1 / math.sqrt(128), 0.8
AXES = akvq.RopeAxes.sections(1e6, (16, 24, 24))
B, HQ, HKV = 3, 8, 2


class Server:
    """Sequences whose rows arrive chunk by chunk (Sequences draws them all at once, as new rows, and owns the pages)."""

    def __init__(self, totals, G, seed=0):
        self.s = Sequences([0] * B, totals, HKV, G, 64, Hq=HQ, salient=[0, 1, 2, 30, 31, 90, 91, 140], seed=seed)
        self.totals = totals
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


def step(cache, x, pos, row_start, max_rows, out):
    q, k, v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
    akvq.rope_axes(AXES, pos, q, k, q_out=q, k_out=k)
    akvq.paged_attention(cache, q, k, v, row_start, max_rows, SM, out=out)
    akvq.paged_append(cache, k, v, row_start, max_rows, CLIP)
    cache.seq_len.add_(row_start[1:] - row_start[:-1])


def _view(srv, x, take, lens):
    """What the oracle looks at: the pages as they were, and the chunk with its positions in."""
    v = Sequences.__new__(Sequences)
    v.__dict__.update(srv.s.__dict__)
    starts = [0]
    for n in take:
        starts.append(starts[-1] + n)
    v.lens, v.rows, v.starts, v.n, v.x = lens, take, starts, starts[-1], x
    v.q, v.k, v.v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
    return v


@pytest.mark.parametrize("G", [128, 64])
def test_chunks_then_tokens(G):
    srv = Server([150, 97, 40], G)
    cache = srv.s.cache
    for take in ([40, 97, 0], [33, 0, 37], [70, 0, 1], [1, 0, 1], [1, 0, 1]):
        x, pos, starts = srv.chunk(take)
        lens = cache.seq_len.tolist()
        out = torch.zeros(x.shape[0], HQ, 128, dtype=torch.float16, device="cuda")
        step(cache, x, pos, starts, max(take), out)
        torch.cuda.synchronize()
        assert cache.seq_len.tolist() == [a + b for a, b in zip(lens, take)]
        check_attention(_view(srv, x, take, lens), out, None, SM, str(take))  # (rows behind lens have changed: none of them is read)
        again = torch.zeros_like(out)  # attention after the rows are stored, lengths not yet advanced: the same
        cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        akvq.paged_attention(cache, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], starts, max(take), SM, out=again)
        cache.seq_len.add_(starts[1:] - starts[:-1])
        torch.cuda.synchronize()
        assert torch.equal(again, out)
    # the pages now hold what one append of every sequence's rows would have written
    whole = Server([150, 97, 40], G)
    x = whole.s.x.clone()
    k = x[:, HQ:HQ + HKV]
    akvq.rope_axes(AXES, whole.pos, None, k, k_out=k)
    rows = [r for b, n in enumerate(cache.seq_len.tolist()) for r in range(whole.s.starts[b], whole.s.starts[b] + n)]
    starts = torch.tensor([0, 145, 242, 282], dtype=torch.int32, device="cuda")
    assert cache.seq_len.tolist() == [145, 97, 40]
    packed = x[rows]
    akvq.paged_append(whole.s.cache, packed[:, HQ:HQ + HKV], packed[:, HQ + HKV:], starts, 150, CLIP)
    torch.cuda.synchronize()
    for name in ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal"):
        assert torch.equal(getattr(cache, name), getattr(whole.s.cache, name)), name


def test_tokens_in_a_graph():
    """The step of one token captured once, with its split attention, and replayed while pages fill up: every replay against the eager
    step, with eager work in between."""
    eager, srv = (Server([1300, 700, 40], 64, seed=3) for _ in range(2))
    n = 6
    first = [1300 - n, 700 - n, 40 - n]
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    outs = []
    for x in (eager, srv):
        data, pos, rs = x.chunk(first)
        step(x.s.cache, data, pos, rs, max(first), torch.empty(data.shape[0], HQ, 128, dtype=torch.float16, device="cuda"))
    for _ in range(n):
        data, pos, _ = eager.chunk([1] * B)
        out = torch.zeros(B, HQ, 128, dtype=torch.float16, device="cuda")
        step(eager.s.cache, data, pos, starts, 1, out)
        outs.append(out)
    torch.cuda.synchronize()
    assert akvq.lib().akvq_paged_default_splits(akvq.C.byref(srv.s.cache.paged_struct()), HQ, 1) > 1
    data, pos, _ = srv.chunk([1] * B)
    x_in, pos_in, out = torch.empty_like(data), torch.empty_like(pos), torch.zeros(B, HQ, 128, dtype=torch.float16, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(srv.s.cache, x_in, pos_in, starts, 1, out)
    for i in range(n):
        data, pos, _ = srv.chunk([1] * B)
        x_in.copy_(data)
        pos_in.copy_(pos)
        out.fill_(float("nan"))
        torch.randn(1 << 20, device="cuda").sum().item()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, outs[i]), i
    for name in ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal", "seq_len"):
        assert torch.equal(getattr(srv.s.cache, name), getattr(eager.s.cache, name)), name


def test_selection_into_a_paged_cache():
    """select_salient fills a PagedCache's lists as it fills a contiguous cache's, text positions and pivots."""
    T = 300
    g = torch.Generator(device="cuda").manual_seed(5)
    k = torch.randn(2, 2, T, 128, generator=g, device="cuda").half()
    k[:, :, ::37] *= 6
    tail = torch.randn(2, 4, 64, 128, generator=g, device="cuda").half()
    text = (torch.rand(2, T, generator=g, device="cuda") < 0.1).to(torch.uint8)
    paged, plain = akvq.PagedCache(2, 2, 128, 12, 5, 64, S_cap=64), akvq.Cache(2, 2, 128, 320, 64)
    for args in (dict(mode=akvq.MODE_TSA, is_text=text), dict(mode=akvq.MODE_PSA, q_tail=tail, k=k, top_k=12, sm_scale=SM)):
        for c in (paged, plain):
            akvq.select_salient(c, **args)
        torch.cuda.synchronize()
        assert torch.equal(paged.counts(), plain.counts())
        n = int(plain.counts().max())
        for b in range(2):
            for h in range(2):
                m = int(plain.counts()[b, h])
                assert m <= n and torch.equal(paged.sal_idx[b, h, :m], plain.sal_idx[b, h, :m])
