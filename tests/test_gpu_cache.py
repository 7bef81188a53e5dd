"""Caches with lengths of their own: append, decode, prefill and eviction against the definitions in 64 bits (cache_reference.py, which
also says how the bounds come about), at lengths, windows, types and layouts where they can go wrong.  Rows that nobody sees hold NaN."""
import math

import pytest
import torch

from cache_reference import HALF, Cache, attend, evict, seen

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ws(ctx, q_cap, weights):
    return torch.full((max(16, ctx.cache_workspace_bytes(q_cap, weights)),), 255, dtype=torch.uint8, device="cuda:0")


def _hide(c, lens, first_p, window, n_first):
    """NaN into every row of the caches that no query sees: queries lie at positions first_p[i] .. lens[i] - 1."""
    for i, L in enumerate(lens):
        hidden = torch.ones(c.t_cap, dtype=torch.bool)
        for p in range(max(0, first_p[i]), L):
            hidden[seen(p, L, window, n_first)] = False
        c.K[i, hidden] = math.nan
        c.V[i, hidden] = math.nan
    c.upload()


DECODE = [
    # g, d, b, dtype, paged, t_cap, window, n_first, lens
    (4, 128, 16, "bf16", True, 400, 0, 0, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 399, 400]),
    (4, 128, 16, "bf16", False, 400, 37, 5, [0, 1, 36, 37, 38, 42, 43, 50, 64, 399, 400]),
    (8, 128, 8, "bf16", True, 1016, 100, 33, [1016, 1009, 7, 100, 101, 133, 134, 200, 0, 513]),
    (8, 64, 8, "bf16", False, 72, 0, 0, [72, 71, 8, 9, 1, 0, 0, 0, 33]),
    (1, 64, 64, "bf16", True, 2048, 1, 0, [2048, 1, 2, 1000]),
    (2, 64, 32, "bf16", True, 2048, 5, 2047, [2048, 5, 6, 1000]),
    (1, 128, 16, "bf16", True, 8192, 0, 0, [8190, 3, 4097]),
    (4, 64, 16, "f32", False, 2064, 0, 0, [2049]),
    (4, 128, 16, "f32", True, 320, 64, 4, [320, 0, 64, 65, 69, 300, 17]),
    (8, 128, 8, "f32", False, 264, 0, 0, [264, 1, 263, 129]),
    (1, 64, 32, "f32", True, 256, 200, 300, [256, 255, 201, 200]),
    (2, 128, 16, "f32", True, 96, 3, 1, [96, 5, 4, 3]),
    (4, 64, 16, "bf16", True, 96, 2147483647, 2147483647, [96, 5, 0]),
]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(case, weights):
    import paper_2502_04077_amd as ap
    g, d, b, dt, paged, t_cap, window, n_first, lens = DECODE[case]
    c = Cache(len(lens), t_cap, d, b, DT[dt], paged, case)
    _hide(c, lens, [L - 1 for L in lens], window, n_first)
    gen = torch.Generator().manual_seed(100 + case)
    q = (2 * torch.randn((c.n, g, d), generator=gen)).to(DT[dt])
    acc0 = torch.rand((c.n, t_cap), generator=gen)
    ctx = c.context(g, ap)
    out, acc = torch.full((c.n, g, d), 7.0, device="cuda:0"), acc0.to("cuda:0")
    ctx.cache_decode(q.to("cuda:0"), c.gK, c.gV, torch.tensor(lens, dtype=torch.int32, device="cuda:0"), window, n_first, out,
                     acc if weights else None, _ws(ctx, 0, weights))
    out, acc = out.cpu().double(), acc.cpu().double()
    for i, L in enumerate(lens):
        ref, w, out_off, w_off = attend(q[i], c.K[i, :L], c.V[i, :L], L - 1, window, n_first)
        assert ((out[i] - ref).abs() <= out_off).all(), (i, L, (out[i] - ref).abs().max())
        now = acc0[i].double()
        if weights:
            now[:L] += w
            off = torch.zeros_like(now)
            off[:L] = w_off + HALF[torch.float32] * now[:L]
            assert ((acc[i] - now).abs() <= off).all(), (i, L, (acc[i] - now).abs().max())
        else:
            assert torch.equal(acc[i], now)


@pytest.mark.parametrize("n,t_cap,lens", [
    (700, 64, lambda i: (i * 37) % 65),                   # more instances than threads of a workgroup, empty ones among them
    (1500, 32, lambda i: 0 if i != 777 else 31),          # one that is not empty
    (40, 4096, lambda i: 4096 if i == 39 else i % 5),     # nearly all of the rows in the last one
    (3, 16384, lambda i: 16383 - i),                      # pieces of one instance in many workgroups
    (2500, 64, lambda i: (i * 37) % 65),                  # more instances than workgroups, short: a wave each
    (1300, 1040, lambda i: 1024 if i % 97 == 0 else i % 3),   # the longest that a wave takes, and many empty ones
    (1300, 1040, lambda i: 1025 if i == 700 else 16),     # one row longer
    (6000, 32, lambda i: 32 if i > 5000 else 0),          # all in the last ones
])
def test_decode_shares(n, t_cap, lens):
    """Rows dealt to workgroups regardless of where instances begin: every kind of piece, weights and outputs."""
    import paper_2502_04077_amd as ap
    g, d = 2, 64
    lens = [lens(i) for i in range(n)]
    c = Cache(n, t_cap, d, 16, torch.bfloat16, True, n)
    gen = torch.Generator().manual_seed(n)
    q = torch.randn((n, g, d), generator=gen).to(torch.bfloat16)
    ctx = c.context(g, ap)
    out, acc = torch.full((n, g, d), 7.0, device="cuda:0"), torch.zeros((n, t_cap), device="cuda:0")
    ctx.cache_decode(q.to("cuda:0"), c.gK, c.gV, torch.tensor(lens, dtype=torch.int32, device="cuda:0"), 0, 0, out, acc, _ws(ctx, 0, True))
    alone = torch.full_like(out, 7.0)
    ctx.cache_decode(q.to("cuda:0"), c.gK, c.gV, torch.tensor(lens, dtype=torch.int32, device="cuda:0"), 0, 0, alone, None, _ws(ctx, 0, False))
    out, acc, alone = out.cpu().double(), acc.cpu().double(), alone.cpu().double()
    for i, L in enumerate(lens):
        ref, w, out_off, w_off = attend(q[i], c.K[i, :L], c.V[i, :L], L - 1, 0, 0)
        assert ((out[i] - ref).abs() <= out_off).all() and ((alone[i] - ref).abs() <= out_off).all(), (i, L)
        assert ((acc[i, :L] - w).abs() <= w_off + HALF[torch.float32] * w).all(), (i, L)
        assert not acc[i, L:].any()


PREFILL = [
    # g, d, b, dtype, paged, t_cap, q_cap, window, n_first, lens, n_q
    (4, 128, 16, "bf16", True, 400, 65, 0, 0, [400, 65, 1, 0, 64, 33, 30, 200], [65, 65, 1, 5, 32, 0, 65, 33]),
    (4, 128, 16, "bf16", False, 304, 40, 37, 5, [304, 40, 41, 78, 100, 37], [40, 40, 39, 40, 1, 17]),
    (8, 128, 8, "bf16", True, 1016, 130, 100, 70, [1016, 131, 90, 500], [130, 130, 90, 77]),
    (8, 64, 8, "bf16", False, 72, 72, 0, 0, [72, 71, 8, 1, 0], [72, 71, 7, 72, 3]),
    (1, 64, 64, "bf16", True, 640, 300, 1, 0, [640, 300, 299], [300, 300, 150]),
    (2, 64, 32, "bf16", True, 640, 200, 5, 2047, [640, 200, 7], [200, 199, 7]),
    (1, 128, 16, "bf16", True, 704, 513, 0, 0, [700, 513], [513, 129]),
    (2, 128, 16, "bf16", False, 1024, 3, 64, 64, [1024, 129, 128, 130], [3, 3, 2, 1]),
    (4, 64, 16, "f32", False, 208, 100, 0, 0, [201, 100, 3], [100, 99, 3]),
    (4, 128, 16, "f32", True, 320, 50, 64, 4, [320, 0, 64, 70, 100], [50, 1, 50, 33, 50]),
    (8, 128, 8, "f32", False, 136, 33, 0, 0, [136, 33, 20], [33, 33, 33]),
    (1, 64, 32, "f32", True, 256, 140, 20, 33, [256, 140], [140, 129]),
    (2, 128, 16, "f32", True, 96, 96, 3, 1, [96, 5], [96, 5]),
    (2, 64, 16, "bf16", True, 96, 40, 2147483647, 2147483647, [96, 5, 30], [40, 40, 40]),
    # few queries behind long caches, which are cut into splits
    (2, 128, 16, "bf16", True, 8192, 3, 0, 0, [8190, 5000, 2, 0], [3, 2, 2, 1]),
    (4, 128, 32, "bf16", False, 2048, 101, 0, 0, [2040, 517, 64], [101, 77, 3]),
    (8, 64, 8, "bf16", True, 5000, 9, 1300, 200, [4999, 1309, 1200], [9, 9, 8]),
    (2, 64, 32, "f32", True, 4096, 4, 1500, 70, [4096, 3001, 4], [4, 4, 3]),
    (1, 128, 16, "f32", False, 2048, 5, 0, 0, [2047, 1], [5, 1]),
]


def _prefill(case, weights, lens, n_q, q_rows=None):
    import paper_2502_04077_amd as ap
    g, d, b, dt, paged, t_cap, q_cap, window, n_first = PREFILL[case][:9]
    c = Cache(len(lens), t_cap, d, b, DT[dt], paged, case)
    _hide(c, lens, [L - m for L, m in zip(lens, n_q)], window, n_first)
    gen = torch.Generator().manual_seed(200 + case)
    q = (2 * torch.randn((c.n, q_cap, g, d), generator=gen)).to(DT[dt])
    for i, m in enumerate(n_q):
        q[i, m:] = math.nan
    acc0 = torch.rand((c.n, t_cap), generator=gen)
    ctx = c.context(g, ap)
    out, acc = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0"), acc0.to("cuda:0")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")  # noqa: E731
    ctx.cache_prefill(q.to("cuda:0"), i32(n_q), c.gK, c.gV, i32(lens), window, n_first, out, acc if weights else None, _ws(ctx, q_cap, weights))
    return c, q, acc0, out.cpu(), acc.cpu()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("case", range(len(PREFILL)))
def test_prefill(case, weights):
    g, d, b, dt, paged, t_cap, q_cap, window, n_first, lens, n_q = PREFILL[case]
    c, q, acc0, out, acc = _prefill(case, weights, lens, n_q)
    half = HALF[DT[dt]]
    for i, (L, m) in enumerate(zip(lens, n_q)):
        now, off = acc0[i].double(), torch.zeros(t_cap, dtype=torch.float64)
        for r in range(m):
            ref, w, out_off, w_off = attend(q[i, r], c.K[i, :L], c.V[i, :L], L - m + r, window, n_first)
            if dt == "bf16":                               # probabilities and outputs are rounded to bf16
                j = seen(L - m + r, L, window, n_first)
                P = torch.softmax(q[i, r].double() @ c.K[i, j].double().T / math.sqrt(d), dim=1) if len(j) else torch.zeros(g, 0).double()
                out_off = out_off + half * (P @ c.V[i, j].double().abs()) + half * ref.abs() * (1 + 2 * half)
            else:
                out_off = out_off + half * ref.abs()
            got = out[i, r].double()
            assert ((got - ref).abs() <= out_off).all(), (i, L, r, (got - ref).abs().max())
            now[:L] += w
            off[:L] += w_off
        assert (out[i, m:] == 7).all(), i
        if weights:
            off += (m * g + 2) * HALF[torch.float32] * now
            assert ((acc[i].double() - now).abs() <= off).all(), (i, L, (acc[i].double() - now).abs().max())
        else:
            assert torch.equal(acc[i], acc0[i])


def test_one_query_of_prefill_is_decode():
    """The same attention by both calls: outputs within their bounds of each other, weights too."""
    import paper_2502_04077_amd as ap
    g, d, t_cap, lens = 4, 128, 512, [512, 100, 1, 77]
    c = Cache(4, t_cap, d, 16, torch.bfloat16, True, 9)
    q = torch.randn((4, 1, g, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to("cuda:0")
    L = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    ctx = c.context(g, ap)
    o1, o2 = torch.zeros((4, 1, g, d), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((4, g, d), device="cuda:0")
    a1, a2 = torch.zeros((4, t_cap), device="cuda:0"), torch.zeros((4, t_cap), device="cuda:0")
    ctx.cache_prefill(q, None, c.gK, c.gV, L, 50, 3, o1, a1, _ws(ctx, 1, True))
    ctx.cache_decode(q[:, 0].contiguous(), c.gK, c.gV, L, 50, 3, o2, a2, _ws(ctx, 0, True))
    assert (o1[:, 0].float() - o2).abs().max() <= 2 * HALF[torch.bfloat16] * c.V.float().abs().max()
    assert (a1 - a2).abs().max() <= 1e-5


EVICT = [
    # d, b, dtype, paged, t_cap, budget, n_first, n_last, lens
    (128, 16, "bf16", True, 400, 64, 4, 16, [400, 399, 65, 64, 63, 1, 0, 200]),
    (128, 8, "bf16", False, 2104, 1031, 64, 256, [2104, 1032, 1031, 2000, 5]),
    (64, 32, "bf16", True, 1024, 300, 0, 0, [1024, 301, 999]),
    (64, 16, "f32", False, 256, 17, 8, 9, [256, 18, 17, 100]),     # nothing of the middle stays
    (128, 16, "f32", True, 512, 300, 300, 0, [512, 301, 4]),
    (128, 64, "bf16", True, 5120, 1, 0, 1, [5120, 2, 1, 0]),
    (64, 8, "bf16", True, 3000, 2900, 1, 1, [3000, 2901, 2950]),
    (64, 16, "bf16", False, 65536 + 128, 5000, 33, 70, [65536 + 128, 65536 + 103, 65535, 5001, 10000]),
    (64, 64, "bf16", True, 140032, 1024, 64, 64, [140000, 131072, 70000]),
]


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("kind", ["spread", "ties", "signs"])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_evict(case, kind, same):
    import paper_2502_04077_amd as ap
    d, b, dt, paged, t_cap, budget, n_first, n_last, lens = EVICT[case]
    c = Cache(len(lens), t_cap, d, b, DT[dt], paged, case)
    gen = torch.Generator().manual_seed(300 + case)
    acc = torch.exp(2 * torch.randn((c.n, t_cap), generator=gen))
    if kind == "ties":
        acc = torch.floor(2 * torch.rand((c.n, t_cap), generator=gen)) + 1.0
    if kind == "signs":
        acc = torch.randn((c.n, t_cap), generator=gen).round() * torch.where(torch.rand((c.n, t_cap), generator=gen) < 0.5, 0.0, 1.0)
        acc[:, ::7] = math.inf
        acc[:, 3::11] = -math.inf
        acc[:, 5::13] = -0.0
    ctx = c.context(2, ap)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    a = acc.to("cuda:0")
    a_out, L_out = (a, L) if same else (torch.full_like(a, 7.0), torch.full_like(L, -1))
    kept = torch.full((c.n, budget), -5, dtype=torch.int32, device="cuda:0")
    ctx.cache_evict(c.gK, c.gV, a, L, budget, n_first, n_last, a_out, L_out, kept)
    K, V, a_out, L_out, kept = c.get(c.gK), c.get(c.gV), a_out.cpu(), L_out.tolist(), kept.cpu()
    for i, n in enumerate(lens):
        stay = evict(acc[i], n, budget, n_first, n_last)
        m = len(stay)
        assert L_out[i] == m and kept[i, :m].tolist() == stay and (kept[i, m:] == -5).all(), (i, n)
        K_ref, V_ref = c.K[i].clone(), c.V[i].clone()
        K_ref[:m], V_ref[:m] = c.K[i, stay], c.V[i, stay]
        assert torch.equal(K[i], K_ref) and torch.equal(V[i], V_ref), (i, n)
        a_ref = acc[i].clone() if same else torch.full((t_cap,), 7.0)
        a_ref[:m] = acc[i, stay]
        a_ref[m:n] = 0
        assert torch.equal(a_out[i], a_ref), (i, n)


@pytest.mark.parametrize("d,b,dt,paged,q_cap,lens,n_new", [
    (128, 16, "bf16", True, 1, [1, 16, 17, 96, 0, 97, 50], None),
    (128, 8, "bf16", False, 7, [7, 6, 96, 100, 40, 0, -3], [7, 7, 0, 7, 3, 2, 1]),
    (64, 32, "bf16", True, 40, [96, 33, 40, 97, 200], [40, 40, 39, 4, 1]),
    (64, 16, "f32", True, 33, [96, 33, 1, 5], [33, 32, 33, 99]),
    (128, 64, "f32", False, 2, [64, 2, 128], [2, -1, 1]),
])
def test_append(d, b, dt, paged, q_cap, lens, n_new):
    import paper_2502_04077_amd as ap
    t_cap = 128 if b == 64 else 96
    c = Cache(len(lens), t_cap, d, b, DT[dt], paged, q_cap)
    gen = torch.Generator().manual_seed(q_cap)
    k, v = (torch.randn((c.n, q_cap, d), generator=gen).to(DT[dt]) for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    c.context(4, ap).cache_append(k.to("cuda:0"), v.to("cuda:0"), None if n_new is None else i32(n_new), i32(lens), c.gK, c.gV)
    for i, L in enumerate(lens):
        m = q_cap if n_new is None else max(0, min(q_cap, n_new[i]))
        for r in range(m):
            if 0 <= L - m + r < t_cap:
                c.K[i, L - m + r], c.V[i, L - m + r] = k[i, r], v[i, r]
    assert torch.equal(c.get(c.gK), c.K) and torch.equal(c.get(c.gV), c.V)


def test_pages_outside_the_pool():
    """Table entries outside the pool: rows there are not written, and reads stay inside the pool."""
    import paper_2502_04077_amd as ap
    c = Cache(2, 64, 64, 16, torch.bfloat16, True, 3)
    pool = c.gK.clone()
    c.gK.nan_to_num_(0.0), c.gV.nan_to_num_(0.0), pool.nan_to_num_(0.0)
    c.table[0, 1], c.table[0, 2], c.table[1, 0] = -1, c.n_pages, 1 << 30
    ctx = c.context(4, ap)
    L = torch.tensor([48, 16], dtype=torch.int32, device="cuda:0")
    new = torch.full((2, 32, 64), 5.0, dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_append(new, new, torch.tensor([32, 16], dtype=torch.int32, device="cuda:0"), L, c.gK, c.gV)
    assert torch.equal(c.gK, pool)
    q = torch.randn((2, 1, 4, 64), device="cuda:0").to(torch.bfloat16)
    out, chunk = torch.zeros((2, 4, 64), device="cuda:0"), torch.zeros((2, 1, 4, 64), dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_decode(q[:, 0].contiguous(), c.gK, c.gV, L, 0, 0, out, None, _ws(ctx, 0, False))
    ctx.cache_prefill(q, None, c.gK, c.gV, L, 0, 0, chunk, None, _ws(ctx, 1, False))
    acc, kept = torch.rand((2, 64), device="cuda:0"), torch.zeros((2, 8), dtype=torch.int32, device="cuda:0")
    ctx.cache_evict(c.gK, c.gV, acc, L, 8, 2, 2, acc, L, kept)
    assert torch.isfinite(out).all() and torch.isfinite(chunk).all() and L.tolist() == [8, 8]


@pytest.mark.parametrize("paged", [False, True])
def test_run_under_a_budget(paged):
    """Prompts of different lengths in two chunks, an eviction, then decode steps with evictions, against a model of all of it in 64 bits.
    Evictions are checked on the GPU's own weights: equal choices need equal inputs."""
    from paper_2502_04077_amd.runner import CacheRun
    from workloads import CONFIGS
    dev = torch.device("cuda:0")
    w = CONFIGS["cfg1"].with_(kv_heads=2, batch=3, t0=150, steps=58, budget_tokens=96, n_sink=1, n_local=2, g=4)
    n, cap = w.n_inst, w.t_cap
    nb = cap // w.block
    table = torch.randperm(n * nb, generator=torch.Generator().manual_seed(4)).to(torch.int32).view(n, nb).to(dev) if paged else None
    run = CacheRun(w, dev, q_cap=80, evict_every=16, table=table, n_pages=n * nb)
    gen = torch.Generator().manual_seed(5)
    draw = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16)  # noqa: E731
    K, V, acc = [torch.zeros((0, 128), dtype=torch.bfloat16)] * n, [torch.zeros((0, 128), dtype=torch.bfloat16)] * n, [torch.zeros(0).double()] * n

    def weights_agree():
        got = run.acc.cpu().double()
        for i in range(n):
            m = len(acc[i])
            assert run.len[i].item() == m and (got[i, :m] - acc[i]).abs().max() <= 1e-4 * max(1.0, acc[i].max().item()), i
            assert not got[i, m:].any()

    def evict_all():
        before = run.acc.cpu()
        lens = run.len.tolist()
        run.evict()
        for i in range(n):
            stay = evict(before[i], lens[i], w.budget_tokens, 16, 32)
            K[i], V[i], acc[i] = K[i][stay], V[i][stay], acc[i][stay]

    for new in ([80, 13, 80, 1, 64, 0], [70, 80, 2, 0, 79, 5]):
        q, k, v = 2 * draw(n, 80, 4, 128), draw(n, 80, 128), draw(n, 80, 128)
        out = run.prefill(q.to(dev), k.to(dev), v.to(dev), torch.tensor(new, dtype=torch.int32, device=dev)).cpu().double()
        for i, m in enumerate(new):
            K[i], V[i] = torch.cat([K[i], k[i, :m]]), torch.cat([V[i], v[i, :m]])
            acc[i] = torch.cat([acc[i], torch.zeros(m).double()])
            for r in range(m):
                ref, wt, off, _ = attend(q[i, r], K[i], V[i], len(K[i]) - m + r, 0, 0)
                acc[i] += wt
                assert (out[i, r] - ref).abs().max() <= 2.5 * HALF[torch.bfloat16] * V[i].double().abs().max() + off.max(), (i, r)
    weights_agree()
    evict_all()
    for step in range(48):
        q, k, v = 2 * draw(n, 4, 128), draw(n, 128), draw(n, 128)
        evicts = (run.steps_done + 1) % run.evict_every == 0
        run.evict_every = 10 ** 9                          # (the eviction of the step is made here, on the weights before it)
        out = run.step(q.to(dev), k.to(dev), v.to(dev)).cpu().double()
        run.evict_every = 16
        for i in range(n):
            K[i], V[i], acc[i] = torch.cat([K[i], k[i:i + 1]]), torch.cat([V[i], v[i:i + 1]]), torch.cat([acc[i], torch.zeros(1).double()])
            ref, wt, off, _ = attend(q[i], K[i], V[i], len(K[i]) - 1, 0, 0)
            acc[i] += wt
            assert ((out[i] - ref).abs() <= off).all(), (step, i)
        weights_agree()
        if evicts:
            evict_all()
    assert run.longest >= max(run.len.tolist())
    full = run.K.view(n, cap, 128) if not paged else run.K[table.long().view(-1)].view(n, cap, 128)
    for i in range(n):
        assert torch.equal(full[i, :len(K[i])].cpu(), K[i])


def test_far_rows():
    """Caches of 12 million rows: offsets pass 32 bits, in rows' bytes and in the pool's; only a window and a few rows are seen or kept."""
    import paper_2502_04077_amd as ap
    n, t_cap, d, b, window, n_first, lens = 2, 12_000_000, 128, 64, 50, 5, [12_000_000, 11_999_989]
    dev = torch.device("cuda:0")
    ctx = ap.Context(n_inst=n, g=1, head_dim=d, block=b, hist_len=1, t_cap=t_cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    K, V = (torch.empty((n, t_cap, d), dtype=torch.bfloat16, device=dev) for _ in range(2))
    gen = torch.Generator().manual_seed(3)
    rows = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16)  # noqa: E731
    L = torch.tensor(lens, dtype=torch.int32, device=dev)
    head_k, head_v, tail_k, tail_v = rows(n, n_first, d), rows(n, n_first, d), rows(n, 60, d), rows(n, 60, d)
    K[:, :n_first], V[:, :n_first] = head_k.to(dev), head_v.to(dev)
    ctx.cache_append(tail_k.to(dev), tail_v.to(dev), None, L, K, V)
    for i in range(n):
        assert torch.equal(K[i, lens[i] - 60:lens[i]].cpu(), tail_k[i]) and torch.equal(V[i, lens[i] - 60:lens[i]].cpu(), tail_v[i])
    q, out, acc = rows(n, 3, 1, d), torch.zeros((n, 1, d), device=dev), torch.zeros((n, t_cap), device=dev)
    chunk = torch.zeros((n, 3, 1, d), dtype=torch.bfloat16, device=dev)
    ctx.cache_prefill(q.to(dev), None, K, V, L, window, n_first, chunk, None, _ws(ctx, 3, False))
    ctx.cache_decode(q[:, 2].contiguous().to(dev), K, V, L, window, n_first, out, acc, _ws(ctx, 0, True))
    for i in range(n):
        for r in range(3):
            k, v = (torch.cat([h[i], t[i, 10 - 2 + r:58 + r]]) for h, t in ((head_k, tail_k), (head_v, tail_v)))
            ref, w, off, w_off = attend(q[i, r], k, v, len(k) - 1, 0, 0)
            assert (chunk[i, r].cpu().double() - ref).abs().max() <= 2.5 * HALF[torch.bfloat16] * v.double().abs().max() + off.max(), (i, r)
        assert ((out[i].cpu().double() - ref).abs() <= off).all(), i
        got = torch.cat([acc[i, :n_first], acc[i, lens[i] - 50:lens[i]]]).cpu().double()
        assert ((got - w).abs() <= w_off + HALF[torch.float32] * w).all() and abs(acc[i].double().sum().item() - 1) < 1e-5, i
    far = [7, 4_000_000, 8_388_608, 9_000_001, 11_000_000]
    acc.zero_()
    acc[:, far] = 3.0
    for i in range(n):
        K[i, far] = V[i, far] = rows(len(far), d).to(dev)
    kept = torch.zeros((n, 20), dtype=torch.int32, device=dev)
    want = [torch.cat([K[i, :n_first], K[i, far], K[i, lens[i] - 10:lens[i]]]).clone() for i in range(n)]
    ctx.cache_evict(K, V, acc, L, 20, n_first, 10, acc, L, kept)
    for i in range(n):
        assert kept[i].tolist() == list(range(n_first)) + far + list(range(lens[i] - 10, lens[i]))
        assert torch.equal(K[i, :20], want[i]) and acc[i].count_nonzero().item() == len(far)
