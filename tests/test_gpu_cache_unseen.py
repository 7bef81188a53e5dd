"""Rows of a cache that hold no numbers, seen by some queries of a chunk and not by others: what a query does not see does not matter, whatever it holds.
Bounds as in cache_reference.py."""
import math

import pytest
import torch

from cache_reference import HALF, Cache, attend, seen

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

SHAPES = [
    # g, d, dtype, block, paged, t_cap, m, window, n_first, lens
    (4, 128, "bf16", 8, True, 304, 12, 0, 0, [12, 130, 200, 301]),                     # one tile of rows of q, in splits
    (4, 128, "bf16", 16, True, 704, 150, 60, 3, [150, 151, 400, 700]),                 # tiles at both ends of a window
    (1, 64, "bf16", 8, False, 304, 40, 100, 0, [40, 64, 300]),
    (8, 64, "f32", 8, True, 304, 24, 0, 0, [24, 100, 301]),
    (2, 128, "f32", 32, True, 320, 70, 33, 5, [70, 90, 320]),
    (4, 64, "f32", 64, False, 256, 100, 0, 0, [100, 256]),
    (4, 128, "bf16", 16, True, 208, 20, 50, 4, [20 + 2 * i for i in range(94)] * 6),   # a workgroup goes over all of a tile's rows
]


def _case(shape, bad, whole):
    """Caches with bad rows among the chunk's own and around the ends of its windows: all of them, or one number."""
    g, d, dt, block, paged, t_cap, m, window, n_first, lens = SHAPES[shape]
    c = Cache(len(lens), t_cap, d, block, DT[dt], paged, shape)
    for i, L in enumerate(lens):
        rows = {L - 2, L - m // 2, L - m + 1}
        if window:
            rows |= {r for r in (L - window - 1, L - m - window + 3, L - window - m // 2) if r >= n_first}
        for x, r in enumerate(sorted(r for r in rows if 0 <= r < L)):
            at = c.V[i, r] if (x + i) % 3 else c.K[i, r]
            if whole:
                at.fill_(bad)
            else:
                at[(7 * x + 11 * i) % d] = bad
        c.K[i, L:], c.V[i, L:] = math.nan, math.nan        # rows that nobody wrote
    c.upload()
    q = 2 * torch.randn((c.n, m, g, d), generator=torch.Generator().manual_seed(shape + 9))
    return c, q.to(DT[dt])


@pytest.mark.parametrize("how", ["alone", "weights", "shared"])
@pytest.mark.parametrize("whole", [True, False], ids=["row", "number"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_what_a_query_does_not_see_does_not_matter(shape, bad, whole, how):
    import paper_2502_04077_amd as ap
    g, d, dt, block, paged, t_cap, m, window, n_first, lens = SHAPES[shape]
    c, q = _case(shape, bad, whole)
    ctx, length = c.context(g, ap), torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    out = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0")
    acc = torch.zeros((c.n, t_cap), device="cuda:0")
    buffer = lambda b: torch.full((max(16, b),), 255, dtype=torch.uint8, device="cuda:0")  # noqa: E731
    if how == "shared":                                    # (chunks of so many rows of q read every instance's own)
        plan = buffer(ctx.cache_share_bytes())
        ctx.cache_share(torch.full_like(length, -1), torch.zeros_like(length), plan)
        ctx.cache_prefill_shared(q.cuda(), None, c.gK, c.gV, length, plan, window, n_first, out, buffer(ctx.cache_shared_workspace_bytes(m)))
    else:
        ctx.cache_prefill(q.cuda(), None, c.gK, c.gV, length, window, n_first, out, acc if how == "weights" else None,
                          buffer(ctx.cache_workspace_bytes(m, how == "weights")))
    out, acc, half, clean, seen_bad = out.cpu().double(), acc.cpu().double(), HALF[DT[dt]], 0, 0
    for i, L in list(enumerate(lens))[::max(1, len(lens) // 12)]:
        total, total_off, spoiled = torch.zeros(L, dtype=torch.float64), torch.zeros(L, dtype=torch.float64), torch.zeros(L, dtype=torch.bool)
        for r in range(m):
            p = L - m + r
            j = seen(p, L, window, n_first)
            if not torch.isfinite(c.K[i, j]).all():
                spoiled[j] = True
                continue
            good = torch.isfinite(c.V[i, j]).all(0)        # dims that no number spoils
            K, V = c.K[i, :L].nan_to_num(0, 0, 0), c.V[i, :L].nan_to_num(0, 0, 0)
            ref, w, off, w_off = attend(q[i, r], K, V, p, window, n_first)
            rounded = off + (half * V.double().abs().max() if dt == "bf16" else 0) + half * ref.abs() * (1 + 2 * half)
            assert ((out[i, r] - ref).abs() <= rounded)[:, good].all(), (i, r)
            assert not torch.isfinite(out[i, r][:, ~good]).any(), (i, r)
            total, total_off = total + w, total_off + w_off + (m * g + 16) * HALF[torch.float32] * w      # (a sum over the chunk)
            clean += int(good.any())
            seen_bad += int((~good).any())
        if how == "weights":
            assert ((acc[i, :L] - total).abs() <= total_off)[~spoiled].all(), i
    assert clean > 0 and seen_bad > 0
