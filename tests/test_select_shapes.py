"""select_salient reads query and key rows of every sequence of the cache: tensors of fewer are refused before anything is launched, for
contiguous caches and caches in pages (on the host)."""
import pytest
import torch

from paper_2501_15021_amd import binding as akvq


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("q,k,mass", [
    ((1, 4, 16, 128), (1, 2, 64, 128), None), ((3, 4, 16, 128), (2, 2, 64, 128), None), ((2, 4, 16, 128), (3, 2, 64, 128), None),
    ((3, 4, 16, 128), (3, 1, 64, 128), None), ((3, 4, 16, 64), (3, 2, 64, 128), None), ((3, 4, 16, 128), (3, 2, 64, 64), None),
    ((3, 4, 16, 128), (3, 2, 64, 128), 3 * 2 * 63)])
def test_rows_of_other_sequences(q, k, mass, paged, monkeypatch):
    c = akvq.PagedCache(3, 2, 128, 4, 2, device="cpu", fill=0) if paged else akvq.Cache(3, 2, 128, 64, 64, device="cpu", fill=0)
    asked = []
    monkeypatch.setattr(akvq, "_stream", lambda: asked.append(1))  # what a launch would need last
    with pytest.raises(AssertionError):
        akvq.select_salient(c, akvq.MODE_PSA, q_tail=torch.zeros(q, dtype=torch.float16), k=torch.zeros(k, dtype=torch.float16), top_k=4, sm_scale=0.1,
                            mass_out=None if mass is None else torch.zeros(mass))
    assert not asked
