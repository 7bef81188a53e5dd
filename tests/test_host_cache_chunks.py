"""The references of the attention over caches say the same query by query and by chunks."""
import pytest
import torch

from cache_chunks import attend_chunk
from cache_reference import attend


@pytest.mark.parametrize("window,n_first", [(0, 0), (5, 0), (5, 3), (1, 40), (200, 2)])
@pytest.mark.parametrize("L,m", [(30, 30), (30, 7), (5, 9), (1, 1), (0, 2), (17, 16), (17, 0), (0, 0)])
def test_by_chunks_and_by_queries(L, m, window, n_first):
    gen = torch.Generator().manual_seed(L * 100 + m)
    q, K, V = (torch.randn(s, generator=gen) for s in ((m, 4, 64), (L, 64), (L, 64)))
    out, w, out_off, w_off, by_size = attend_chunk(q, K, V, L - m, window, n_first)
    total, total_off = torch.zeros(L).double(), torch.zeros(L).double()
    for r in range(m):
        o, x, o_off, x_off = attend(q[r], K, V, L - m + r, window, n_first)
        assert torch.allclose(out[r], o, rtol=1e-12, atol=1e-14) and torch.allclose(out_off[r], o_off, rtol=1e-9, atol=1e-20)
        assert (by_size[r] >= o.abs() - 1e-12).all()
        total, total_off = total + x, total_off + x_off
    assert torch.allclose(w, total, rtol=1e-12, atol=1e-14) and torch.allclose(w_off, total_off, rtol=1e-9, atol=1e-20)
