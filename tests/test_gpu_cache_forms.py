"""Caches with lengths of their own: the forms of the kernels that only many instances or long chunks reach, for every type, head size and
group, against the definitions in 64 bits.  Rows that nobody sees hold NaN."""
import math

import pytest
import torch

from cache_chunks import attend_chunk
from cache_reference import HALF, Cache, attend, evict

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMS = [(dt, d, g) for dt in ("bf16", "f32") for d in (64, 128) for g in (1, 2, 4, 8)]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def _ws(ctx, q_cap, weights):
    return torch.full((max(16, ctx.cache_workspace_bytes(q_cap, weights)),), 255, dtype=torch.uint8, device="cuda:0")


def _hide(c, lens, first_p, window, n_first):
    """NaN into every row of the caches that no query sees: queries lie at positions first_p[i] .. lens[i] - 1."""
    j = torch.arange(c.t_cap)
    for i, L in enumerate(lens):
        lo = max(0, max(0, first_p[i]) - window + 1) if window > 0 else 0
        shown = (j < L) & ((j >= lo) | (j < n_first))
        c.K[i, ~shown] = math.nan
        c.V[i, ~shown] = math.nan
    c.upload()


# Chunks of more workgroups of 128 rows of q than there are CUs: n instances of t_cap rows, chunks of q_cap.
def _chunks(g, n=48, tiles=6):
    return dict(n=n, q_cap=(tiles * 128 - 60) // g, t_cap=(tiles * 128 // g + 64) // 64 * 64 + 128)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("n", [48, 30])                    # 288 workgroups; 180, and two splits of each
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_prefill_of_many_workgroups(form, n, weights):
    import paper_2502_04077_amd as ap
    dt, d, g = FORMS[form]
    x = _chunks(g, n)
    q_cap, t_cap = x["q_cap"], x["t_cap"]
    window, n_first = [(0, 0), (q_cap // 2, 5), (37, 70), (0, 0), (1, 0)][(form + n) % 5]
    paged, b = [(True, 8), (False, 16), (True, 64), (True, 16)][form % 4]
    lens = [t_cap if i == 0 else (i * 97 + 31 * form) % (t_cap + 1) for i in range(n)]
    lens[3], lens[4] = 0, 1
    n_q = [q_cap if i % 3 == 0 else (i * 59) % (q_cap + 1) for i in range(n)]
    c = Cache(n, t_cap, d, b, DT[dt], paged, form)
    _hide(c, lens, [L - m for L, m in zip(lens, n_q)], window, n_first)
    gen = torch.Generator().manual_seed(400 + form)
    q = (2 * torch.randn((n, q_cap, g, d), generator=gen)).to(DT[dt])
    for i, m in enumerate(n_q):
        q[i, m:] = math.nan
    acc0 = torch.rand((n, t_cap), generator=gen)
    ctx = c.context(g, ap)
    out, acc = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0"), acc0.to("cuda:0")
    ctx.cache_prefill(q.to("cuda:0"), _i32(n_q), c.gK, c.gV, _i32(lens), window, n_first, out, acc if weights else None, _ws(ctx, q_cap, weights))
    out, acc, half = out.cpu(), acc.cpu(), HALF[DT[dt]]
    for i, (L, m) in enumerate(zip(lens, n_q)):
        ref, w, off, w_off, by_size = attend_chunk(q[i, :m], c.K[i, :L], c.V[i, :L], L - m, window, n_first)
        # bf16: probabilities and outputs are rounded
        off = off + half * ref.abs() * (1 + 2 * half) + (half * by_size if dt == "bf16" else 0)
        assert ((out[i, :m].double() - ref).abs() <= off).all(), (i, L, m)
        assert (out[i, m:] == 7).all(), i
        if weights:
            now = acc0[i].double()
            now[:L] += w
            bound = (m * g + 2) * HALF[torch.float32] * now
            bound[:L] += w_off
            assert ((acc[i].double() - now).abs() <= bound).all(), (i, L, m)
        else:
            assert torch.equal(acc[i], acc0[i])


# Workgroups of a decode call: instances beyond as many, all of them short, go a wave each.
def _workgroups(dt, d, g):
    pieces = d * (2 if dt == "bf16" else 4) // 16
    return 256 * ({8: 3 if g == 8 else 4, 16: 2, 32: 1}[pieces])


@pytest.mark.parametrize("over", [0, 1, 301])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_decode_of_many_short_instances(form, over):
    import paper_2502_04077_amd as ap
    dt, d, g = FORMS[form]
    n, t_cap = _workgroups(dt, d, g) + over, 192
    window, n_first = [(0, 0), (20, 3), (0, 0), (50, 17)][(form + over) % 4]
    paged, b = [(True, 16), (False, 16), (True, 8), (True, 64)][form % 4]
    lens = [(0, 192, 1, (i * 37) % 193, (i * 11) % 40)[i % 5] for i in range(n)]
    c = Cache(n, t_cap, d, b, DT[dt], paged, form)
    _hide(c, lens, [L - 1 for L in lens], window, n_first)
    gen = torch.Generator().manual_seed(500 + form)
    q = (2 * torch.randn((n, g, d), generator=gen)).to(DT[dt])
    acc0 = torch.rand((n, t_cap), generator=gen)
    ctx = c.context(g, ap)
    outs, acc = [torch.full((n, g, d), 7.0, device="cuda:0") for _ in range(2)], acc0.to("cuda:0")
    for out, a in zip(outs, (acc, None)):
        ctx.cache_decode(q.to("cuda:0"), c.gK, c.gV, _i32(lens), window, n_first, out, a, _ws(ctx, 0, a is not None))
    outs, acc = [x.cpu().double() for x in outs], acc.cpu().double()
    for i, L in enumerate(lens):
        ref, w, off, w_off = attend(q[i], c.K[i, :L], c.V[i, :L], L - 1, window, n_first)
        assert all(((x[i] - ref).abs() <= off).all() for x in outs), (i, L)
        now = acc0[i].double()
        now[:L] += w
        bound = HALF[torch.float32] * now
        bound[:L] += w_off
        assert ((acc[i] - now).abs() <= bound).all(), (i, L)


# Instances from which on an eviction moves columns of 128 bytes, and one fewer.
@pytest.mark.parametrize("fewer", [0, 1])
@pytest.mark.parametrize("d,dt,paged,b,n", [(128, "bf16", True, 16, 128), (128, "bf16", False, 16, 128), (64, "bf16", True, 8, 256),
                                            (128, "f32", True, 64, 64), (64, "f32", False, 16, 128)])
def test_evict_of_many_instances(d, dt, paged, b, n, fewer):
    import paper_2502_04077_amd as ap
    n, t_cap, budget, n_first, n_last = n - fewer, 1024, 700, 30, 100
    lens = [(1024, 701, 700, (i * 131) % 1025, 1000 - i)[i % 5] for i in range(n)]
    c = Cache(n, t_cap, d, b, DT[dt], paged, n)
    gen = torch.Generator().manual_seed(n)
    acc = torch.exp(2 * torch.randn((n, t_cap), generator=gen))
    a, L, kept = acc.to("cuda:0"), _i32(lens), torch.full((n, budget), -5, dtype=torch.int32, device="cuda:0")
    c.context(2, ap).cache_evict(c.gK, c.gV, a, L, budget, n_first, n_last, a, L, kept)
    K, V, a, left, kept = c.get(c.gK), c.get(c.gV), a.cpu(), L.tolist(), kept.cpu()
    for i, m in enumerate(lens):
        stay = evict(acc[i], m, budget, n_first, n_last)
        k = len(stay)
        assert left[i] == k and kept[i, :k].tolist() == stay and (kept[i, k:] == -5).all(), (i, m)
        for got, was in ((K, c.K), (V, c.V)):
            ref = was[i].clone()
            ref[:k] = was[i, stay]
            assert torch.equal(got[i], ref), (i, m)
        ref = acc[i].clone()
        ref[:k] = acc[i, stay]
        ref[k:m] = 0
        assert torch.equal(a[i], ref), (i, m)


# ------------------------------------------------------------------------------------------------------------------
# One workspace for calls whose lengths change, eager and replayed: without weights the pieces of an instance are counted in it.
# ------------------------------------------------------------------------------------------------------------------
LENGTHS = [[2000, 1, 1500, 130, 0, 129], [128, 2000, 1999, 0, 640, 16], [2048] * 6, [0, 0, 0, 2048, 0, 1], [700, 300, 2000, 150, 260, 1024]]


@pytest.mark.parametrize("dt,d,g", [("bf16", 128, 4), ("f32", 64, 1), ("bf16", 64, 8)])
@pytest.mark.parametrize("between", ["nothing", "fill", "prefill"])
def test_replays_of_a_decode_without_weights(dt, d, g, between):
    import paper_2502_04077_amd as ap
    n, t_cap = 6, 2048
    c = Cache(n, t_cap, d, 16, DT[dt], True, 1)
    ctx = c.context(g, ap)
    gen = torch.Generator().manual_seed(2)
    q = torch.randn((n, g, d), generator=gen).to(DT[dt]).to("cuda:0")
    chunk = torch.randn((n, 4, g, d), generator=gen).to(DT[dt]).to("cuda:0")
    L, out, chunk_out = _i32(LENGTHS[0]), torch.zeros((n, g, d), device="cuda:0"), torch.zeros_like(chunk)
    ws = torch.zeros(ctx.cache_workspace_bytes(4, False), dtype=torch.uint8, device="cuda:0")
    ctx.cache_decode(q, c.gK, c.gV, L, 0, 0, out, None, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.cache_decode(q, c.gK, c.gV, L, 0, 0, out, None, ws)
    torch.cuda.synchronize()
    for i in range(3 * len(LENGTHS)):
        L.copy_(_i32(LENGTHS[i % len(LENGTHS)]))
        q.copy_(torch.randn((n, g, d), generator=gen).to(DT[dt]))
        if between == "fill":
            ws.fill_((0, 255, 37)[i % 3])
        if between == "prefill":
            ctx.cache_prefill(chunk, None, c.gK, c.gV, L, 0, 0, chunk_out, None, ws)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        fresh = torch.full_like(out, 7.0)
        ctx.cache_decode(q, c.gK, c.gV, L, 0, 0, fresh, None, _ws(ctx, 0, False))
        again = torch.full_like(out, 7.0)
        ctx.cache_decode(q, c.gK, c.gV, L, 0, 0, again, None, ws)      # the workspace of the replays, eagerly
        assert torch.equal(out, fresh) and torch.equal(again, fresh), i
        for x, m in enumerate(LENGTHS[i % len(LENGTHS)]):
            ref, _, off, _ = attend(q[x].cpu(), c.K[x, :m], c.V[x, :m], m - 1, 0, 0)
            assert ((out[x].cpu().double() - ref).abs() <= off).all(), (i, x)


def test_eager_decodes_share_a_workspace():
    """Lengths, windows and calls with weights between them, one workspace: what a call finds there says nothing."""
    import paper_2502_04077_amd as ap
    n, t_cap, g, d = 6, 2048, 4, 128
    c = Cache(n, t_cap, d, 16, torch.bfloat16, False, 3)
    ctx = c.context(g, ap)
    gen = torch.Generator().manual_seed(4)
    ws = _ws(ctx, 0, True)
    for i in range(20):
        L, q = _i32(LENGTHS[i % 5]), torch.randn((n, g, d), generator=gen).to(torch.bfloat16).to("cuda:0")
        window = (0, 700, 1300)[i % 3]
        outs = [torch.full((n, g, d), 7.0, device="cuda:0") for _ in range(2)]
        accs = [torch.zeros((n, t_cap), device="cuda:0") if i % 4 == 3 else None for _ in range(2)]
        ctx.cache_decode(q, c.gK, c.gV, L, window, 3, outs[0], accs[0], ws)
        ctx.cache_decode(q, c.gK, c.gV, L, window, 3, outs[1], accs[1], _ws(ctx, 0, True))
        assert torch.equal(*outs) and (accs[0] is None or torch.equal(*accs)), i
        for x, m in enumerate(LENGTHS[i % 5]):
            ref, _, off, _ = attend(q[x].cpu(), c.K[x, :m], c.V[x, :m], m - 1, window, 3)
            assert ((outs[0][x].cpu().double() - ref).abs() <= off).all(), (i, x)
