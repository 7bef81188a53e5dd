"""Attention over beginnings in common, and calls on pages, at the ends of their ranges: scores of any size that 32 bits hold (as in
test_gpu_cache_scores.py, which says why the definition gives equal weights there), the digits of fp32 (as in test_gpu_cache_digits.py), the most
instances, empty ones, pools beyond 32-bit offsets, many groups and many windows, two contexts at a time, and the device that is not current."""
import math

import pytest
import torch

from cache_reference import HALF, attend
from page_reference import Device, Pool
from test_gpu_cache_digits import _attend
from test_gpu_cache_scores import BELOW, DT, SIZES
from test_gpu_shared import Shared, _i32, _plan, _ws

pytestmark = pytest.mark.gpu

SHAPES = [
    # g, d, dtype, layout, t_cap, q_cap, window, n_first, group, shared, lens
    (4, 128, "bf16", "shared", 400, 5, 0, 0, [0, 0, 0, 1, 1, -1], [100, 100, 100, 17, 17, 0], [400, 101, 110, 17, 200, 130]),
    (8, 64, "bf16", "flat", 304, 4, 37, 5, [0, 0, 0], [200, 200, 200], [304, 201, 230]),
    (1, 64, "f32", "own", 2064, 3, 0, 0, [5, 5], [1000, 1000], [2049, 1003]),
    (2, 128, "f32", "shared", 320, 9, 64, 4, [1, 0, 1, 0], [64] * 4, [320, 73, 75, 300]),
    (4, 128, "bf16", "shared", 1040, 8, 0, 0, [0] * 40, [900] * 40, [908 + 3 * i for i in range(40)]),      # tiles of a workgroup, joined
]


def _inputs(shape, size, n_q):
    g, d, dt, layout, t_cap, q_cap, window, n_first, group, shared, lens = SHAPES[shape]
    k, sign = size
    gen = torch.Generator().manual_seed(shape)
    n = len(lens)
    c = Shared(lens, group, shared, t_cap, d, 16, DT[dt], "flat", shape, [0] * n, 0, 0)
    c.V = torch.randn((n, t_cap, d), generator=gen).to(DT[dt])
    c.K = torch.randn((n, t_cap, d), generator=gen).to(DT[dt])
    step = torch.randint(1, 5, (n, t_cap), generator=gen).float()
    if k == BELOW:
        step = torch.full((n, t_cap), -2.0 ** 20)
        for i, L in enumerate(lens):
            step[i, max(0, L - 1):L] = 0.0
            step[i, max(0, L - n_q - 2):max(0, L - n_q)] = 0.0
    c.K[:, :, 0] = step
    for i in range(n):                                     # rows in common are the lowest member's
        if group[i] >= 0:
            of, S = group.index(group[i]), min(shared[j] for j in range(n) if group[j] == group[i])
            c.K[i, :S], c.V[i, :S] = c.K[of, :S], c.V[of, :S]
    c.layout = layout
    if layout == "flat":
        c.gK, c.gV = c.K.to(c.dev), c.V.to(c.dev)
    else:
        nb = t_cap // 16
        c.n_pages = n * nb + 3
        names = torch.randperm(c.n_pages, generator=gen)[:n * nb].view(n, nb)
        if layout == "shared":
            for i in range(n):
                if group[i] >= 0:
                    names[i, :min(shared[j] for j in range(n) if group[j] == group[i]) // 16] = names[group.index(group[i]), :min(shared[j] for j in range(n) if group[j] == group[i]) // 16]
        pool = [torch.full((c.n_pages, 16, d), math.nan, dtype=DT[dt]) for _ in range(2)]
        for x, y in zip(pool, (c.K, c.V)):
            x[names.view(-1)] = y.view(-1, 16, d)
        c.gK, c.gV = (x.to(c.dev) for x in pool)
        c.table = names.to(torch.int32).to(c.dev)
    q = torch.zeros((n, n_q, g, d))
    q[..., 0] = sign * 2.0 ** (120 if k == BELOW else k)
    return c, q.to(DT[dt])


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_scores_of_any_size(shape, size):
    import paper_2502_04077_amd as ap
    g, d, dt, layout, t_cap, q_cap, window, n_first, group, shared, lens = SHAPES[shape]
    half = HALF[DT[dt]]
    for m in (1, q_cap):
        c, q = _inputs(shape, size, m)
        ctx, L32 = c.context(g, ap), _i32(lens)
        plan = _plan(ctx, group, shared)
        outs = [torch.full((c.n, m, g, d), 7.0, dtype=DT[dt], device="cuda:0")]
        ctx.cache_prefill_shared(q.to("cuda:0"), None, c.gK, c.gV, L32, plan, window, n_first, outs[0], _ws(ctx, m))
        if m == 1:
            outs.append(torch.full((c.n, m, g, d), 7.0, device="cuda:0"))
            ctx.cache_decode_shared(q[:, 0].to("cuda:0").contiguous(), c.gK, c.gV, L32, plan, window, n_first, outs[1].view(c.n, g, d), _ws(ctx))
        outs = [x.cpu().double() for x in outs]
        for i, L in enumerate(lens):
            for r in range(m):
                ref, w, _, _ = attend(q[i, r], c.K[i, :L], c.V[i, :L], L - m + r, window, n_first)
                terms = (w[None, :] / g) @ c.V[i, :L].double().abs()
                if size[0] == BELOW and w.any() and c.K[i, :L, 0][w > 0].min() < 0:
                    ref, terms = torch.zeros_like(ref), torch.zeros_like(terms)          # nothing that has a weight in 32 bits
                base = (2 * L + 16) * HALF[torch.float32] * terms
                rounded = base + (half * terms if dt == "bf16" else 0) + half * ref.abs() * (1 + 2 * half)
                for out, off in zip(outs, (rounded, base)):
                    assert ((out[i, r] - ref).abs() <= off).all(), (m, i, L, r, (out[i, r] - ref).abs().max())


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_scores_above_32_bits_make_nan_of_their_head(shape):
    """The first head's scores of the newest token pass 32 bits at the newest row: NaN there, in whatever form, and the others as without it."""
    import paper_2502_04077_amd as ap
    g, d, dt, layout, t_cap, q_cap, window, n_first, group, shared, lens = SHAPES[shape]
    c, _ = _inputs(shape, (20, 1), 1)
    q = torch.randn((c.n, q_cap, g, d), generator=torch.Generator().manual_seed(shape)).to(DT[dt])
    at = c.gK.view(-1, d) if c.table is None else c.gK
    hit = [L > (min(shared[j] for j in range(c.n) if group[j] == group[i]) if group[i] >= 0 else 0) for i, L in enumerate(lens)]
    for i, L in enumerate(lens):
        if hit[i]:                                         # (its own row)
            row = at[i * t_cap + L - 1] if c.table is None else at[c.table[i, (L - 1) // 16].item(), (L - 1) % 16]
            row.zero_()
            row[0] = 2.0 ** 20
    big = q.clone()
    big[:, -1, 0] = 0.0
    big[:, -1, 0, 0] = 2.0 ** 120
    ctx, L32, got = c.context(g, ap), _i32(lens), []
    plan = _plan(ctx, group, shared)
    for x in (q, big):
        out, one = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0"), torch.full((c.n, g, d), 7.0, device="cuda:0")
        ctx.cache_prefill_shared(x.to("cuda:0"), None, c.gK, c.gV, L32, plan, window, n_first, out, _ws(ctx, q_cap))
        ctx.cache_decode_shared(x[:, -1].contiguous().to("cuda:0"), c.gK, c.gV, L32, plan, window, n_first, one, _ws(ctx))
        got.append((out.cpu(), one.cpu()))
    (out, one), (big_out, big_one) = got
    assert torch.equal(out[:, :-1], big_out[:, :-1]) and torch.equal(out[:, -1, 1:], big_out[:, -1, 1:]) and torch.equal(one[:, 1:], big_one[:, 1:])
    assert torch.isfinite(out).all() and torch.isfinite(one).all()
    for i in range(c.n):
        if hit[i]:
            assert big_out[i, -1, 0].isnan().all() and big_one[i, 0].isnan().all(), i


@pytest.mark.parametrize("window", [0, 3])
@pytest.mark.parametrize("L", [40, 500, 2049])
@pytest.mark.parametrize("d,g", [(64, 1), (64, 8), (128, 1), (128, 4)])
@pytest.mark.parametrize("m,each", [(1, 4), (1, 32), (8, 2), (8, 16)])
def test_digits_of_fp32(m, each, d, g, L, window):
    import paper_2502_04077_amd as ap
    n, window, n_first = 32, window and L // window, 4
    gen = torch.Generator().manual_seed(L + g)
    S = L * 3 // 4
    group = [i % (n // each) for i in range(n)]
    cap = (L + 15) // 16 * 16
    K, V = (torch.randn((n, cap, d), generator=gen) for _ in range(2))
    for i in range(n):
        K[i, :S], V[i, :S] = K[group[i], :S], V[group[i], :S]
    K, V, q = K.to("cuda:0"), V.to("cuda:0"), (2 * torch.randn((n, m, g, d), generator=gen)).to("cuda:0")
    ctx = ap.Context(n_inst=n, g=g, head_dim=d, block=16, hist_len=1, t_cap=cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="f32")
    length, out, plan = _i32([L] * n), torch.zeros_like(q), _plan(ctx, group, [S] * n)
    if m == 1:
        ctx.cache_decode_shared(q[:, 0].contiguous(), K, V, length, plan, window, n_first, out.view(n, g, d), _ws(ctx))
    else:
        ctx.cache_prefill_shared(q, None, K, V, length, plan, window, n_first, out, _ws(ctx, m))
    p = torch.arange(L - m, L, device="cuda:0")
    exact, plain = (_attend(q, K[:, :L], V[:, :L], p, window, n_first, t) for t in (torch.float64, torch.float32))
    rms = lambda x: ((x.double() - exact).square().mean() / exact.square().mean()).sqrt().item()  # noqa: E731
    assert rms(out) <= 1.5 * rms(plain), (rms(out), rms(plain))


@pytest.mark.parametrize("n,groups", [(65535, 1), (65535, 20000), (65533, 65533), (3, 1), (1, 1)])
def test_numbers_of_instances_and_groups(n, groups):
    """The most instances, all in one group, in many or each in its own; values of some of them."""
    import paper_2502_04077_amd as ap
    g, d, t_cap, S = 2, 64, 24, 9
    lens = [(i * 7) % 16 + 9 if i % 11 else (i // 11) % 9 for i in range(n)]      # (some have not all that is shared; the first one of all none)
    lens[:groups] = [10 + i % 15 for i in range(groups)]
    group, shared = [i % groups for i in range(n)], [S + i % 3 for i in range(n)]
    gen = torch.Generator().manual_seed(n + groups)
    K, V = (torch.randn((n, t_cap, d), generator=gen).to(torch.bfloat16) for _ in range(2))
    lead = torch.tensor(group)
    K[:, :S], V[:, :S] = K[lead, :S], V[lead, :S]
    if n < 10:
        shared = [S] * n
    else:
        K[:, S:S + 2], V[:, S:S + 2] = K[lead, S:S + 2], V[lead, S:S + 2]          # (of groups whose members all say more)
    q = torch.randn((n, 2, g, d), generator=gen).to(torch.bfloat16)
    ctx = ap.Context(n_inst=n, g=g, head_dim=d, block=8, hist_len=1, t_cap=t_cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    plan, L32 = _plan(ctx, group, shared), _i32(lens)
    one, two = torch.full((n, g, d), 7.0, device="cuda:0"), torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_decode_shared(q[:, 0].contiguous().cuda(), K.cuda(), V.cuda(), L32, plan, 0, 0, one, _ws(ctx))
    new = [min(2, L) for L in lens]
    ctx.cache_prefill_shared(q.cuda(), _i32(new), K.cuda(), V.cuda(), L32, plan, 5, 3, two, _ws(ctx, 2))
    one, two, half = one.cpu().double(), two.cpu().double(), HALF[torch.bfloat16]
    for i in sorted(set(range(0, n, max(1, n // 300))) | {0, 1, n - 2, n - 1} & set(range(n))):
        L = lens[i]
        ref, _, off, _ = attend(q[i, 0], K[i, :L], V[i, :L], L - 1, 0, 0)
        assert ((one[i] - ref).abs() <= off).all(), i
        for r in range(new[i]):
            ref, _, off, _ = attend(q[i, r], K[i, :L], V[i, :L], L - new[i] + r, 5, 3)
            assert ((two[i, r] - ref).abs() <= off + half * V[i, :L].double().abs().max() + half * ref.abs() * (1 + 2 * half)).all(), (i, r)
        assert (two[i, new[i]:] == 7).all()


@pytest.mark.parametrize("n", [1023, 1024, 1025, 1500, 5000])
def test_many_groups_and_windows(n):
    """More sources than the threads of a workgroup hold at once, most of them of no or few tiles, with windows that leave some beginnings."""
    import paper_2502_04077_amd as ap
    g, d, t_cap = 1, 64, 200
    rng = torch.Generator().manual_seed(n)
    group = torch.randint(-2, n // 3, (n,), generator=rng).tolist()
    shared = torch.randint(0, 150, (n,), generator=rng).tolist()
    lens = torch.randint(0, t_cap + 1, (n,), generator=rng).tolist()
    c = Shared(lens, group, shared, t_cap, d, 8, torch.bfloat16, "shared", n, [L - 3 for L in lens], 40, 6)
    q = torch.randn((n, 3, g, d), generator=rng).to(torch.bfloat16)
    ctx = c.context(g, ap)
    plan, L32 = _plan(ctx, group, shared), _i32(lens)
    one, three = torch.full((n, g, d), 7.0, device="cuda:0"), torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_decode_shared(q[:, 0].contiguous().cuda(), c.gK, c.gV, L32, plan, 40, 6, one, _ws(ctx))
    new = [min(3, L) for L in lens]
    ctx.cache_prefill_shared(q.cuda(), _i32(new), c.gK, c.gV, L32, plan, 40, 6, three, _ws(ctx, 3))
    one, three, half = one.cpu().double(), three.cpu().double(), HALF[torch.bfloat16]
    for i in range(0, n, 7):
        L = lens[i]
        ref, _, off, _ = attend(q[i, 0], c.K[i, :L], c.V[i, :L], L - 1, 40, 6)
        assert ((one[i] - ref).abs() <= off).all(), i
        for r in range(new[i]):
            ref, _, off, _ = attend(q[i, r], c.K[i, :L], c.V[i, :L], L - new[i] + r, 40, 6)
            big = c.V[i, :L].double().nan_to_num(0).abs().max()
            assert ((three[i, r] - ref).abs() <= off + half * big + half * ref.abs() * (1 + 2 * half)).all(), (i, r)


def test_pools_beyond_32_bit_offsets():
    """Pages whose elements and bytes lie behind 2^32, reached by every call."""
    import paper_2502_04077_amd as ap
    n, b, d, g, nb = 4, 64, 128, 4, 4
    n_pages = (1 << 32) // (b * d) + 70
    gen = torch.Generator().manual_seed(8)
    K, V = (torch.empty((n_pages, b, d), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    ctx = ap.Context(n_inst=n, g=g, head_dim=d, block=b, hist_len=1, t_cap=nb * b, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    last = n_pages - 1
    table = _i32([[last, last - 3, last - 5, -1], [last, last - 3, last - 9, -1], [7, 5, -1, -1], [-1] * 4])
    ctx.set_block_table(table, n_pages)
    lens = [170, 150, 128, 0]
    rows = torch.randn((2, 8, b, d), generator=gen).to(torch.bfloat16)
    for x, page in enumerate((last, last - 3, last - 5, last - 9, 7, 5)):
        K[page], V[page] = rows[0, x].cuda(), rows[1, x].cuda()
    seqs = [[0, 1, 2], [0, 1, 3], [4, 5], []]
    flat = [[torch.cat([rows[y, x] for x in s])[:L] if s else rows[y, 0, :0] for s, L in zip(seqs, lens)] for y in range(2)]
    state = torch.zeros(ctx.pages_state_bytes(n_pages) // 4, dtype=torch.int32, device="cuda:0")
    ws = torch.full((ctx.pages_workspace_bytes(n_pages),), 255, dtype=torch.uint8, device="cuda:0")
    info = _i32([-1, -1])
    plan = _plan(ctx, [3, 3, -1, -1], [128, 128, 0, 0])
    q = torch.randn((n, g, d), generator=gen).to(torch.bfloat16)

    def check(lens, flat):
        out = torch.full((n, g, d), 7.0, device="cuda:0")
        ctx.cache_decode_shared(q.cuda(), K, V, _i32(lens), plan, 0, 0, out, _ws(ctx))
        out = out.cpu().double()
        for i, L in enumerate(lens):
            ref, _, off, _ = attend(q[i], flat[0][i], flat[1][i], L - 1, 0, 0)
            assert ((out[i] - ref).abs() <= off).all(), i
    ctx.pages_count(table, n_pages, state)
    assert state[:n_pages].sum() == 8 and state[n_pages:].sum() == n_pages - 6
    check(lens, flat)
    L32 = _i32(lens)
    ctx.pages_fork(K, V, table, state, _i32([0, 1, 2, 0]), L32, L32, info, ws)          # a copy from the pool's end
    assert table[3].tolist() == [last, last - 3, 0, -1] and info.tolist() == [n_pages - 7, 0] and L32.tolist() == [170, 150, 128, 170]
    flat = [x[:3] + [x[0]] for x in flat]
    check([170, 150, 128, 170], flat)
    ctx.pages_resize(K, V, table, state, _i32([170, 150, 129, 170]), _i32([0, 40, 0, 0]), 40, info, ws)
    assert table.tolist() == [[last, last - 3, last - 5, -1], [last, 1, last - 9, -1], [7, 5, 2, -1], [last, last - 3, 0, -1]]
    check(lens[:3] + [170], flat)
    other = [torch.empty((6, b, d), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    ctx.pages_copy(K, V, _i32([last, last - 9]), *other, _i32([4, 0]))
    assert torch.equal(other[0][4], K[last]) and torch.equal(other[1][0], V[last - 9])
    other[0].fill_(3.0)
    ctx.pages_copy(*other, _i32([1]), K, V, _i32([last - 1]))
    assert (K[last - 1] == 3).all()
    ctx.pages_compact(K, V, table, state, info, ws)
    assert info.tolist() == [n_pages - 9, 4] and table.max() == 8 and state[:9].min() > 0 and state[9:n_pages].max() == 0
    check(lens[:3] + [170], flat)


def test_two_contexts_at_a_time():
    """Both kinds of calls of two contexts on two streams."""
    import paper_2502_04077_amd as ap
    gen = torch.Generator().manual_seed(6)
    n, g, d, b, cap = 24, 4, 128, 16, 1040
    lens = [[900 + 5 * i for i in range(n)], [40 * i for i in range(n)]]
    group = [[i % 2 for i in range(n)], [i // 5 for i in range(n)]]
    shared = [[850] * n, [200 * (i // 5) for i in range(n)]]
    c = [Shared(lens[x], group[x], shared[x], cap, d, b, torch.bfloat16, "shared", x, [0] * n, 0, 0) for x in range(2)]
    ctx = [y.context(g, ap) for y in c]
    q = torch.randn((2, 20, n, g, d), generator=gen).to(torch.bfloat16).cuda()
    chunk = torch.randn((2, n, 6, g, d), generator=gen).to(torch.bfloat16).cuda()

    def work(x):
        plan, ws, outs = _plan(ctx[x], group[x], shared[x]), _ws(ctx[x], 6), []
        table, K, V, L = c[x].table.clone(), c[x].gK, c[x].gV, _i32(lens[x])
        state = torch.zeros(ctx[x].pages_state_bytes(c[x].n_pages) // 4, dtype=torch.int32, device="cuda:0")
        pws, info = torch.zeros(ctx[x].pages_workspace_bytes(c[x].n_pages), dtype=torch.uint8, device="cuda:0"), _i32([0, 0])
        ctx[x].pages_count(table, c[x].n_pages, state)
        K2, V2 = K.clone(), V.clone()
        for i in range(20):
            outs.append(torch.full((n, g, d), 7.0, device="cuda:0"))
            ctx[x].cache_decode_shared(q[x, i], K, V, L, plan, 0, 0, outs[-1], ws)
            if i % 6 == 5:
                outs.append(torch.zeros_like(chunk[x]))
                ctx[x].cache_prefill_shared(chunk[x], None, K, V, L, plan, 300, 5, outs[-1], ws)
                ctx[x].pages_resize(K2, V2, table, state, L - i, None, 1, info, pws)
                ctx[x].pages_compact(K2, V2, table, state, info, pws)
        return outs + [table, state, K2, V2]
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
            for i, (a, y) in enumerate(zip(alone[x], got[x])):
                assert torch.equal(a.view(torch.uint8), y.view(torch.uint8)), (x, i)


@pytest.mark.parametrize("n", [1, 2, 7])
def test_pools_of_one_and_two_pages(n):
    """The smallest pools and tables: one block an instance."""
    gen = torch.Generator().manual_seed(n)
    for n_pages in (1, 2):
        K, V = (torch.randn((n_pages, 8, 64), generator=gen) for _ in range(2))
        pool = Pool([[-1]] * n, n_pages, 8, K, V)
        dev = Device(__import__("paper_2502_04077_amd"), pool, 8, 64)
        for length, new, cap in (([0] * n, None, 0), ([8] + [0] * (n - 1), None, 8), ([1] * n, None, 1), ([0] * n, [5] * n, 9)):
            assert pool.resize(length, new, cap) == dev.resize(length, new, cap)
            dev.same(pool)
        assert pool.resize([3] + [0] * (n - 1), None, 3) == dev.resize([3] + [0] * (n - 1), None, 3)
        for parent in ([0] * n, list(range(n)), [n] * n):
            assert pool.fork(parent, [3] + [0] * (n - 1)) == dev.fork(parent, [3] + [0] * (n - 1))
            dev.same(pool)
        assert pool.compact() == dev.compact()
        dev.same(pool)


@pytest.mark.parametrize("dt,d,g", [("bf16", 128, 4), ("bf16", 64, 1), ("f32", 64, 2), ("f32", 128, 1)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_query_does_not_see_does_not_matter(dt, d, g, bad):
    """Rows that hold no numbers, seen by some of a group or chunk and not by others, whose outputs are those of the definition."""
    import paper_2502_04077_amd as ap
    t_cap, window, n_first, m = 304, 60, 3, 4
    lens = [130, 200, 300, 150] + [260 + 3 * i for i in range(12)]
    n = len(lens)
    c = Shared(lens, [0] * n, [120] * n, t_cap, d, 8, DT[dt], "shared", d + g, [0] * n, 0, 0)
    c.K, c.V = c.K.nan_to_num(0.5), c.V.nan_to_num(0.5)
    c.gK, c.gV = c.gK.nan_to_num(0.25), c.gV.nan_to_num(0.25)
    for i, row, K in [(0, 75, True), (0, 110, False)] + [(i, lens[i] - 2, i % 2 == 0) for i in range(1, n, 3)]:
        page = c.table[i, row // 8].item()
        (c.gK if K else c.gV)[page, row % 8] = bad
        for j in range(n) if row < 120 else [i]:
            (c.K if K else c.V)[j, row] = bad
    q = torch.randn((n, m, g, d), generator=torch.Generator().manual_seed(3)).to(DT[dt])
    ctx, L32 = c.context(g, ap), _i32(lens)
    plan = _plan(ctx, [0] * n, [120] * n)
    one, out = torch.full((n, g, d), 7.0, device="cuda:0"), torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0")
    ctx.cache_decode_shared(q[:, -1].contiguous().cuda(), c.gK, c.gV, L32, plan, window, n_first, one, _ws(ctx))
    ctx.cache_prefill_shared(q.cuda(), None, c.gK, c.gV, L32, plan, window, n_first, out, _ws(ctx, m))
    one, out, half, clean = one.cpu().double(), out.cpu().double(), HALF[DT[dt]], 0
    for i, L in enumerate(lens):
        for r in range(m):
            p = L - m + r
            j = [x for x in range(p + 1) if x > p - window or x < n_first]
            if not (torch.isfinite(c.K[i, j]).all() and torch.isfinite(c.V[i, j]).all()):
                continue
            clean += 1
            K, V = c.K[i, :L].nan_to_num(0, 0, 0), c.V[i, :L].nan_to_num(0, 0, 0)
            ref, _, off, _ = attend(q[i, r], K, V, p, window, n_first)
            rounded = off + (half * V.double().abs().max() if dt == "bf16" else 0) + half * ref.abs() * (1 + 2 * half)
            assert ((out[i, r] - ref).abs() <= rounded).all(), (i, r)
            if r == m - 1:
                assert ((one[i] - ref).abs() <= off).all(), i
    assert clean > n


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("where", ["q", "K", "V", "K first", "V first"])
def test_what_holds_no_numbers_costs_little(where, dt, d):
    """A sequence whose q, or a row of whose cache, holds no numbers: NaN for those that see it, the same bytes for the others, and in about the time."""
    import paper_2502_04077_amd as ap
    n, g, L, S = 16, 4, 16000, 15000
    gen = torch.Generator(device="cuda:0").manual_seed(d)
    K, V, q = (torch.randn(s, generator=gen, device="cuda:0").to(DT[dt]) for s in ((n, L, d), (n, L, d), (n, g, d)))
    ctx = ap.Context(n_inst=n, g=g, head_dim=d, block=16, hist_len=1, t_cap=L, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype=dt)
    length, plan, ws = _i32([L] * n), _plan(ctx, [0] * n, [S] * n), _ws(ctx)

    def timed():
        out, best = torch.full((n, g, d), 7.0, device="cuda:0"), math.inf
        for _ in range(5):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            for _ in range(4):
                ctx.cache_decode_shared(q, K, V, length, plan, 0, 0, out, ws)
            end.record()
            torch.cuda.synchronize()
            best = min(best, begin.elapsed_time(end))
        return out, best
    good, usual = timed()
    for at in {"q": [q[3, 1]], "K": [K[3, L - 2]], "V": [V[3, L - 2]], "K first": K[:, 5], "V first": V[:, 5]}[where]:
        at.fill_(math.nan)
    bad, slow = timed()
    hit = torch.full((n, g), "first" in where, device="cuda:0")
    hit[3, 1 if where == "q" else slice(None)] = True
    assert bad[hit].isnan().all() and torch.equal(bad[~hit], good[~hit])
    # (Rows of q that go over all rows of the cache one after the other take some 5 ms, the call some 40 us.)
    assert slow < 5 * usual, (usual, slow)
