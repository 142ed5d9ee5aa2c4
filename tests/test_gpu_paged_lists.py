"""What the documentation of the cache in pages leaves to the caller: pages that sequences share, and salient lists of prompts that differ in
length or come in pieces."""
import math

import pytest
import torch

from paper_2501_15021_amd import binding as akvq
from paged_inputs import Sequences, check_attention

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
ALL = ("k_codes", "v_codes", "k_meta", "v_meta", "k_sal", "v_sal")


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_pages_that_sequences_share(rows):
    """Lists that agree on the shared rows and differ behind them; the 16-bit rows copied."""
    s = Sequences([128, 200], [rows, 7], 2, 64, Hq=4, salient=[3, 31, 64, 127, 150, 199], seed=rows).fill_pages()
    p = s.cache
    p.table[0, :2] = p.table[1, :2]
    p.k_sal[0] = p.k_sal[1]
    p.v_sal[0] = p.v_sal[1]
    p.sal_idx[0, :, 4:6] = torch.tensor([129, 131], dtype=torch.int32)  # of rows to come
    for n_split in (1, 3):
        out, lse = torch.zeros(s.n, 4, 128, dtype=torch.float16, device="cuda"), torch.zeros(s.n, 4, device="cuda")
        akvq.paged_attention(p, s.q, s.k, s.v, s.row_start, s.max_rows, SM, n_split=n_split, out=out, lse=lse)
        torch.cuda.synchronize()
        check_attention(s, out, lse, SM, f"n_split {n_split}")


@pytest.mark.parametrize("G", [128, 64])
def test_pivots_of_unequal_prompts_in_pieces(G):
    """Each prompt's pivots selected into a cache of its own, its list copied, its rows appended piece by piece: what the contiguous path holds."""
    lens, Hkv, Hq = [300, 117, 64], 2, 4
    s = Sequences([0] * 3, lens, Hkv, G, 32, Hq=Hq, seed=G, S_cap=64)
    want = []
    for b, t in enumerate(lens):
        k, v = (x[s.starts[b]:s.starts[b + 1]].transpose(0, 1)[None].contiguous() for x in (s.k, s.v))
        k[:, :, 5:t:23] *= 6
        s.k[s.starts[b]:s.starts[b + 1]] = k[0].transpose(0, 1)
        c = akvq.Cache(1, Hkv, G, (s.cache.max_pages * 32 + 63) // 64 * 64, 64, fill=0)
        akvq.select_salient(c, akvq.MODE_PSA, q_tail=s.q[s.starts[b + 1] - 16:s.starts[b + 1]].transpose(0, 1)[None].contiguous(), k=k, top_k=9, sm_scale=SM)
        s.cache.sal_idx[b] = c.sal_idx[0]
        s.cache.counts()[b] = c.counts()[0]
        akvq.quantize_append(c, k, v, 0.8)
        want.append(c)
    s.cache.seq_len.zero_()
    at = [0, 0, 0]
    for piece in (40, 33, 1, 226):
        take = [min(piece, t - a) for t, a in zip(lens, at)]
        rows = [r for b in range(3) for r in range(s.starts[b] + at[b], s.starts[b] + at[b] + take[b])]
        x = s.x[rows]
        starts = torch.tensor([0, take[0], take[0] + take[1], sum(take)], dtype=torch.int32, device="cuda")
        akvq.paged_append(s.cache, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], starts, max(take), 0.8)
        s.cache.seq_len.add_(starts[1:] - starts[:-1])
        at = [a + n for a, n in zip(at, take)]
    torch.cuda.synchronize()
    assert at == lens and int(s.cache.counts().min()) == 9
    for b, c in enumerate(want):
        got = s.contiguous(b)
        for name in ALL:
            assert torch.equal(getattr(got, name), getattr(c, name)), (b, name)
