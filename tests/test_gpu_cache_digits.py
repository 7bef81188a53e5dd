"""Digits of the attention over fp32 caches: as many as the definition has when it is computed by plain products, exponentials and sums in 32 bits.
Errors against 64 bits, root mean square over all outputs of a call, at most 1.5 times the plain computation's: both are sums of as many terms with
roundings of one size, which differ by the order of the sums."""
import math

import pytest
import torch

from cache_reference import Cache

pytestmark = pytest.mark.gpu


def _attend(q, K, V, p, window, n_first, dtype):
    """q [n][m][g][d] at positions p [m] of caches [n][L][d], all computed in `dtype`."""
    n, m, g, d = q.shape
    q, K, V = (x.to(dtype) for x in (q, K, V))
    j = torch.arange(K.shape[1], device=K.device)[None, :]
    seen = j <= p[:, None]
    if window:
        seen &= (j > p[:, None] - window) | (j < n_first)
    w = torch.matmul(q.reshape(n, m * g, d), K.transpose(1, 2).contiguous()).view(n, m, g, -1) * (1.0 / math.sqrt(d))
    w = w.masked_fill(~seen[None, :, None, :], -math.inf)
    w = (w - w.amax(-1, keepdim=True)).exp()
    w = w / w.sum(-1, keepdim=True)
    return torch.matmul(w.view(n, m * g, -1), V).view(n, m, g, d)


@pytest.mark.parametrize("window", [0, 3])
@pytest.mark.parametrize("L", [40, 500, 2049])
@pytest.mark.parametrize("d,g", [(64, 1), (64, 8), (128, 1), (128, 4)])
@pytest.mark.parametrize("m", [1, 33])
def test_digits_of_fp32(m, d, g, L, window):
    import paper_2502_04077_amd as ap
    n, window, n_first = 32, window and L // window, 4
    c = Cache(n, (L + 15) // 16 * 16, d, 16, torch.float32, False, L + d)
    q = (2 * torch.randn((n, m, g, d), generator=torch.Generator().manual_seed(L + g))).to("cuda:0")
    ctx = c.context(g, ap)
    length = torch.full((n,), L, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(ctx.cache_workspace_bytes(m, False), dtype=torch.uint8, device="cuda:0")
    out = torch.zeros_like(q)
    if m == 1:
        ctx.cache_decode(q[:, 0].contiguous(), c.gK, c.gV, length, window, n_first, out.view(n, g, d), None, ws)
    else:
        ctx.cache_prefill(q, None, c.gK, c.gV, length, window, n_first, out, None, ws)
    p = torch.arange(L - m, L, device="cuda:0")
    exact, plain = (_attend(q, c.gK[:, :L], c.gV[:, :L], p, window, n_first, t) for t in (torch.float64, torch.float32))
    rms = lambda x: ((x.double() - exact).square().mean() / exact.square().mean()).sqrt().item()  # noqa: E731
    assert rms(out) <= 1.5 * rms(plain), (rms(out), rms(plain))
