"""Caches with lengths of their own at the ends of their ranges: the most instances, the smallest caches, nothing but empty ones, weights
that are no numbers, and calls of two contexts at a time on two streams."""
import math

import pytest
import torch

from cache_chunks import attend_chunk
from cache_reference import HALF, Cache, attend, evict

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def _ws(ctx, q_cap, weights):
    return torch.full((max(16, ctx.cache_workspace_bytes(q_cap, weights)),), 255, dtype=torch.uint8, device="cuda:0")


def _all_calls(c, g, q_cap, lens, budget, check):
    """append, prefill, decode and eviction of a cache, checked for the instances of `check`; lens: behind the append."""
    import paper_2502_04077_amd as ap
    n, d, t_cap, dt = c.n, c.d, c.t_cap, c.K.dtype
    gen = torch.Generator().manual_seed(n)
    ctx, L = c.context(g, ap), _i32(lens)
    new = [min(L_, q_cap) for L_ in lens]
    k, v = (torch.randn((n, q_cap, d), generator=gen).to(dt) for _ in range(2))
    q = torch.randn((n, q_cap, g, d), generator=gen).to(dt)
    ctx.cache_append(k.to("cuda:0"), v.to("cuda:0"), _i32(new), L, c.gK, c.gV)
    chunk, out = torch.full(q.shape, 7.0, dtype=dt, device="cuda:0"), torch.full((n, g, d), 7.0, device="cuda:0")
    acc, ws = torch.zeros((n, t_cap), device="cuda:0"), _ws(ctx, q_cap, True)
    ctx.cache_prefill(q.to("cuda:0"), _i32(new), c.gK, c.gV, L, 0, 0, chunk, acc, ws)
    ctx.cache_decode(q[:, 0].contiguous().to("cuda:0"), c.gK, c.gV, L, 0, 0, out, acc, ws)
    before = acc.cpu()
    kept = torch.full((n, budget), -5, dtype=torch.int32, device="cuda:0")
    for i in check:
        if new[i]:
            c.K[i, lens[i] - new[i]:lens[i]], c.V[i, lens[i] - new[i]:lens[i]] = k[i, :new[i]], v[i, :new[i]]
    K, V = c.get(c.gK), c.get(c.gV)
    ctx.cache_evict(c.gK, c.gV, acc, L, budget, 0, 1, acc, L, kept)
    K2, V2, acc, L, kept, chunk, out = c.get(c.gK), c.get(c.gV), acc.cpu(), L.tolist(), kept.cpu(), chunk.cpu(), out.cpu()
    half = HALF[dt]
    for i in check:
        m, x = lens[i], new[i]
        assert torch.equal(K[i], c.K[i]) and torch.equal(V[i], c.V[i]), i
        ref, w, off, w_off, by_size = attend_chunk(q[i, :x], c.K[i, :m], c.V[i, :m], m - x, 0, 0)
        off = off + half * ref.abs() * (1 + 2 * half) + (half * by_size if dt == torch.bfloat16 else 0)
        assert ((chunk[i, :x].double() - ref).abs() <= off).all() and (chunk[i, x:] == 7).all(), i
        ref, w1, off, w1_off = attend(q[i, 0], c.K[i, :m], c.V[i, :m], m - 1, 0, 0)
        assert ((out[i].double() - ref).abs() <= off).all(), i
        assert ((before[i, :m].double() - w - w1).abs() <= w_off + w1_off + (x * g + 3) * HALF[torch.float32] * (w + w1)).all(), i
        assert not before[i, m:].any(), i
        stay = evict(before[i], m, budget, 0, 1)
        s = len(stay)
        assert L[i] == s and kept[i, :s].tolist() == stay and (kept[i, s:] == -5).all(), i
        assert torch.equal(K2[i, :s], K[i, stay]) and torch.equal(V2[i, :s], V[i, stay]) and torch.equal(K2[i, s:], K[i, s:]), i
        assert torch.equal(acc[i, :s], before[i, stay]) and not acc[i, s:].any(), i


@pytest.mark.parametrize("paged", [False, True])
def test_the_most_instances(paged):
    n = 65535
    c = Cache(n, 16, 64, 8, torch.bfloat16, paged, 1)
    _all_calls(c, 1, 3, [(i * 7) % 17 for i in range(n)], 9, list(range(0, n, 1311)) + [n - 1, n - 2, 65279, 65280])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,g,paged", [(64, 8, False), (128, 1, True)])
@pytest.mark.parametrize("lens", [[8], [1], [0], [7, 8, 0, 3], [0] * 9])
def test_caches_of_one_block(dt, d, g, paged, lens):
    c = Cache(len(lens), 8, d, 8, DT[dt], paged, 2)
    _all_calls(c, g, 5, lens, 4, range(len(lens)))


@pytest.mark.parametrize("t_cap,L,budget", [(1024, 1000, 300), (5120, 5000, 1200), (65536 + 64, 65540, 2000)])
def test_weights_that_are_no_numbers(t_cap, L, budget):
    """Which rows stay is open, but as many as the budget, in order, the forced ones among them, and what is moved is theirs."""
    import paper_2502_04077_amd as ap
    n, d, n_first, n_last = 3, 64, 8, 16
    c = Cache(n, t_cap, d, 16, torch.bfloat16, True, 3)
    acc = torch.rand((n, t_cap), generator=torch.Generator().manual_seed(4))
    acc[0, ::3] = math.nan
    acc[1] = math.nan
    acc[2, 1::2] = torch.tensor([-1], dtype=torch.int32).view(torch.float32)       # a NaN with every bit set
    a, lens, kept = acc.to("cuda:0"), _i32([L] * n), torch.full((n, budget), -5, dtype=torch.int32, device="cuda:0")
    c.context(2, ap).cache_evict(c.gK, c.gV, a, lens, budget, n_first, n_last, a, lens, kept)
    K, V, kept = c.get(c.gK), c.get(c.gV), kept.cpu().long()
    assert lens.tolist() == [budget] * n
    for i in range(n):
        assert (kept[i, 1:] > kept[i, :-1]).all() and kept[i, 0] >= 0 and kept[i, -1] < L
        assert kept[i, :n_first].tolist() == list(range(n_first)) and kept[i, -n_last:].tolist() == list(range(L - n_last, L))
        assert torch.equal(K[i, :budget], c.K[i, kept[i]]) and torch.equal(V[i, :budget], c.V[i, kept[i]])


def test_two_contexts_at_a_time():
    """Decodes without weights, whose pieces are counted in the workspace, prefills and evictions of two contexts on two streams."""
    import paper_2502_04077_amd as ap
    n, t_cap, g, d = 5, 2048, 4, 128
    lens = [[2000, 1, 1500, 130, 0], [129, 2048, 640, 0, 1999]]
    gen = torch.Generator().manual_seed(6)
    caches = [Cache(n, t_cap, d, 16, torch.bfloat16, x == 0, 10 + x) for x in range(2)]
    ctx = [c.context(g, ap) for c in caches]
    q = [[torch.randn((n, g, d), generator=gen).to(torch.bfloat16).to("cuda:0") for _ in range(20)] for _ in range(2)]
    chunk = [torch.randn((n, 90, g, d), generator=gen).to(torch.bfloat16).to("cuda:0") for _ in range(2)]
    acc0 = [torch.rand((n, t_cap), generator=gen).to("cuda:0") for _ in range(2)]

    def work(x):
        L, ws, outs = _i32(lens[x]), _ws(ctx[x], 90, False), []
        K, V, acc = caches[x].gK.clone(), caches[x].gV.clone(), acc0[x].clone()
        kept = torch.zeros((n, 500), dtype=torch.int32, device="cuda:0")
        for i in range(20):
            outs.append(torch.full((n, g, d), 7.0, device="cuda:0"))
            ctx[x].cache_decode(q[x][i], K, V, L, 0, 0, outs[-1], None, ws)
            if i % 6 == 5:
                outs.append(torch.zeros_like(chunk[x]))
                ctx[x].cache_prefill(chunk[x], None, K, V, L, 300, 5, outs[-1], None, ws)
            if i == 12:
                ctx[x].cache_evict(K, V, acc, L, 500, 4, 4, acc, L, kept)
        return outs + [K, V, acc, L, kept]
    alone = [work(x) for x in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for x in range(2):
            with torch.cuda.stream(streams[x]):
                got.append(work(x))
        torch.cuda.synchronize()
        for x in range(2):
            for i, (a, b) in enumerate(zip(alone[x], got[x])):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (x, i)       # (bytes: pages of nobody hold NaN)
