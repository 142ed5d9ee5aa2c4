"""Flags that do not fit the C ABI's 32 bits are refused, not cut off (on the host, before devices are looked at)."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq


@pytest.mark.parametrize("flags", [1 << 32, (1 << 32) | akvq.K_PREROTATED, -1, -(1 << 33)])
def test_flags_that_do_not_fit(flags):
    c = akvq.PagedCache(1, 2, 128, 2, 2, device="cpu", fill=0)
    x, start = torch.zeros(3, 2, 128, dtype=torch.float16), torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(akvq.AkvqError, match="flags"):
        akvq.paged_append(c, x, x, start, 3, 0.8, flags)
    with pytest.raises(akvq.AkvqError, match="flags"):
        akvq.paged_attention(c, x, x, x, start, 3, 0.1, flags=flags)
    with pytest.raises(akvq.AkvqError, match="current device"):
        akvq.paged_append(c, x, x, start, 3, 0.8, akvq.K_PREROTATED)
