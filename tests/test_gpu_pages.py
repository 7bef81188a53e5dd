"""Pages that instances share: taken, given back, copied before they are written, forked, compacted and copied, against the definitions
(page_reference.py), all of it bit by bit.  Workspaces start with anything."""
import random

import pytest
import torch

from page_reference import Device, Pool

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _pool(n, nb, n_pages, b, d, dtype, seed, table=None):
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn((n_pages, b, d), generator=g).to(DT[dtype]) for _ in range(2))
    return Pool(table if table is not None else [[-1] * nb for _ in range(n)], n_pages, b, K, V)


SHAPES = [  # n, nb, n_pages, b, d, dtype
    (1, 1, 1, 8, 64, "bf16"),
    (3, 4, 9, 8, 64, "f32"),
    (5, 9, 40, 16, 128, "bf16"),
    (70, 3, 150, 64, 64, "bf16"),
    (4, 130, 600, 8, 64, "bf16"),          # rows of a table longer than a wave
    (300, 8, 1500, 8, 64, "bf16"),         # more instances than threads of a workgroup, pages in two segments
    (6, 400, 2049, 8, 64, "bf16"),         # one page in the third segment
    (700, 7, 3500, 8, 64, "bf16"),         # more instances than a fourth of the threads of a large workgroup
    (1270, 4, 4000, 8, 64, "bf16"),        # more than all of them
    (1200, 8, 7000, 8, 64, "bf16"),
    (13, 300, 3000, 8, 64, "bf16"),        # tables longer than half a wave looks at together
    (17, 256, 2500, 16, 64, "f32"),
    (50, 30, 900, 8, 64, "bf16"),
    (32, 11, 250, 8, 64, "bf16"),          # as many instances as one workgroup takes, and one more
    (33, 11, 250, 8, 64, "bf16"),
    (3, 2100, 4100, 8, 64, "bf16"),        # rows of a table longer than a workgroup looks at together
]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_life_of_a_pool(shape):
    """Random lengths, forks and compactions, one after the other; pages run short now and then."""
    import paper_2502_04077_amd as ap
    n, nb, n_pages, b, d, dtype = SHAPES[shape]
    rng, pool = random.Random(shape), _pool(n, nb, n_pages, b, d, dtype, shape)
    gpu, lens = Device(ap, pool, nb * b, d), [0] * n
    gpu.same(pool)
    for step in range(24):
        what = rng.choice(["grow", "grow", "grow", "shrink", "fork", "fork", "compact"])
        if what == "grow":
            q = rng.choice([1, 3, b, 3 * b])
            new = [rng.choice([0, 1, q, rng.randint(0, q)]) for _ in range(n)] if rng.random() < 0.7 else None
            want = [min(nb * b, x + (q if new is None else new[i])) for i, x in enumerate(lens)]
            told = None if new is None else [w - x for w, x in zip(want, lens)]
            info = pool.resize(want, told, q)
            assert gpu.resize(want, told, q) == info
            lens = want if info[1] == 0 else lens
        elif what == "shrink":
            lens = [rng.choice([0, x, max(0, x - 1), rng.randint(0, x)]) for x in lens]
            assert gpu.resize(lens, None, 0) == pool.resize(lens, None, 0)
        elif what == "fork":
            parent = [rng.choice([i, i, rng.randrange(n), rng.randrange(n), -1, n]) for i in range(n)]
            now, info = pool.fork(parent, lens)
            assert gpu.fork(parent, lens, in_place=rng.random() < 0.5) == (now, info)
            lens = now
        else:
            assert gpu.compact() == pool.compact()
        gpu.same(pool)


def test_rows_about_to_be_written_are_own():
    """Three instances share pages; rows go back into them: the rows in front are copied, those behind are not, and who writes nothing keeps its pages."""
    import paper_2502_04077_amd as ap
    table = [[4, 2, 7, -1], [4, 2, 7, -1], [4, 2, -1, -1], [9, -1, -1, -1]]
    pool = _pool(4, 4, 12, 8, 64, "bf16", 1, table)
    gpu = Device(ap, pool, 32, 64)
    for length, new, q in (([17, 24, 16, 3], [6, 0, 1, 2], 8), ([13, 17, 16, 3], [4, 5, 16, 0], 16), ([8, 8, 8, 8], None, 8), ([24, 1, 9, 0], None, 1)):
        assert gpu.resize(length, new, q) == pool.resize(length, new, q)
        gpu.same(pool)


def test_all_or_nothing():
    import paper_2502_04077_amd as ap
    pool = _pool(3, 4, 5, 8, 64, "f32", 2)
    gpu = Device(ap, pool, 32, 64)
    assert gpu.resize([16, 8, 9], None, 0) == pool.resize([16, 8, 9], None, 0) == [0, 0]
    gpu.same(pool)
    # Six pages for five; the third instance would give two up.
    assert gpu.resize([24, 8, 0], None, 0) == pool.resize([24, 8, 0], None, 0) == [0, 1]
    gpu.same(pool)
    assert gpu.fork([0, 0, 2], [16, 8, 9]) == pool.fork([0, 0, 2], [16, 8, 9]) == ([16, 16, 9], [1, 0])
    gpu.same(pool)
    assert gpu.fork([2, 2, 2], [16, 16, 9]) == pool.fork([2, 2, 2], [16, 16, 9]) == ([16, 16, 9], [1, 1])
    assert gpu.fork([2, 2, 2], [16, 16, 9], in_place=False) == ([16, 16, 9], [1, 1])
    gpu.same(pool)


def test_beams_move_among_each_other():
    """A permutation with repeats: everybody's table is somebody else's next one."""
    import paper_2502_04077_amd as ap
    n = 9
    pool = _pool(n, 6, 120, 16, 128, "bf16", 3)
    gpu, lens = Device(ap, pool, 96, 128), [5 + 11 * i for i in range(n)]
    lens[8] = 96
    assert gpu.resize(lens, None, 0) == pool.resize(lens, None, 0)
    for parent in ([1, 2, 3, 4, 5, 6, 7, 8, 0], [8, 8, 8, 0, 0, 5, 5, 7, 7], [0] * 9, [8, 7, 6, 5, 4, 3, 2, 1, 0], [-1, 9, -7, 3, 3, 2147483647, 6, 6, -2147483648]):
        now, info = pool.fork(parent, lens)
        assert gpu.fork(parent, lens) == (now, info)
        lens = now
        gpu.same(pool)


def test_lengths_and_entries_out_of_range():
    import paper_2502_04077_amd as ap
    table = [[3, 99, -7, 5], [2147483647, 1, -2147483648, 12]]
    pool = _pool(2, 4, 12, 8, 64, "bf16", 4, table)
    gpu = Device(ap, pool, 32, 64)
    gpu.same(pool)
    for length, new, q in (([17, 40], [-3, 99], 5), ([-5, 2147483647], None, 0), ([2147483647, -2147483648], [2147483647, 1], 2147483647)):
        assert gpu.resize(length, new, q) == pool.resize(length, new, q)
        gpu.same(pool)


def test_a_state_that_does_not_belong_to_the_table_stays_in_the_pool():
    """Counts of anything: whatever is taken, named or moved, no row outside the pool is written (the pools lie inside larger buffers)."""
    import paper_2502_04077_amd as ap
    rng = random.Random(5)
    for case in range(6):
        pool = _pool(6, 5, 40, 8, 64, "f32", case, [[rng.choice([-1, rng.randrange(40)]) for _ in range(5)] for _ in range(6)])
        gpu = Device(ap, pool, 40, 64)
        wide = [torch.full((120, 8, 64), 3.0, device="cuda:0") for _ in range(2)]
        gpu.K, gpu.V = (w[40:80] for w in wide)
        gpu.state[:40] = gpu.i32([rng.choice([0, 0, 1, 2, -1, 2147483647]) for _ in range(40)])
        gpu.state[40:] = rng.choice([0, 17, 40, 2147483647, -2147483648])
        for _ in range(3):
            gpu.resize([rng.randint(0, 40) for _ in range(6)], None, rng.choice([0, 3]))
            gpu.fork([rng.randrange(-1, 6) for _ in range(6)], [rng.randint(0, 40) for _ in range(6)])
            gpu.compact()
        for w in wide:
            assert (w[:40] == 3).all() and (w[80:] == 3).all()


@pytest.mark.parametrize("d,b,dtype", [(64, 8, "bf16"), (128, 16, "bf16"), (128, 64, "f32"), (64, 32, "f32")])
def test_copy(d, b, dtype):
    import paper_2502_04077_amd as ap
    g = torch.Generator().manual_seed(b)
    src, dst = ([torch.randn((p, b, d), generator=g).to(DT[dtype]) for _ in range(2)] for p in (37, 50))
    ctx = Device(ap, _pool(2, 2, 3, b, d, dtype, 1), 2 * b, d).ctx
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for a, c, n in (([5, 36, 0, 7, 7], [49, 0, 3, 12, 13], None), ([3, -1, 37, 2147483647, 4, 6], [1, 2, 3, 4, 50, -1], None), ([8], [8], None), ([], [], None),
                    (None, [40, 30, 20], None), ([9, 1], None, None), (None, None, 37), (None, None, 0), (list(range(37)), list(range(37, 0, -1)), None)):
        on = [x.to("cuda:0") for x in dst]
        ctx.pages_copy(src[0].to("cuda:0"), src[1].to("cuda:0"), None if a is None else i32(a), *on, None if c is None else i32(c), n)
        count = n if n is not None else len(a if a is not None else c)
        for x, y, z in zip(src, dst, on):
            want = y.clone()
            for k in range(count):
                s, t = k if a is None else a[k], k if c is None else c[k]
                if 0 <= s < 37 and 0 <= t < 50:
                    want[t] = x[s]
            assert torch.equal(z.cpu(), want)


def test_copy_to_pinned_memory_and_back():
    import paper_2502_04077_amd as ap
    dev = Device(ap, _pool(4, 6, 30, 16, 128, "bf16", 7), 96, 128)
    dev.resize([96, 50, 7, 0], None, 0)
    K, V = dev.K.clone(), dev.V.clone()
    pages = dev.table[:2][dev.table[:2] >= 0].contiguous()
    host = [torch.zeros((pages.numel(), 16, 128), dtype=torch.bfloat16, pin_memory=True) for _ in range(2)]
    dev.ctx.pages_copy(dev.K, dev.V, pages, *host, None)
    torch.cuda.synchronize()
    assert torch.equal(host[0], K[pages.long()].cpu()) and torch.equal(host[1], V[pages.long()].cpu())
    dev.K.zero_()
    dev.V.zero_()
    dev.ctx.pages_copy(*host, None, dev.K, dev.V, pages)
    assert torch.equal(dev.K[pages.long()], K[pages.long()]) and torch.equal(dev.V[pages.long()], V[pages.long()])
    assert not dev.K[[p for p in range(30) if p not in pages.tolist()]].any()


def test_many_pages():
    """Segments that are full, half full and empty, and more of them than workgroups look for free pages; lists as long as the pool."""
    import paper_2502_04077_amd as ap
    n, nb, n_pages = 20, 5000, 99000
    rng = torch.Generator().manual_seed(9)
    ctx = ap.Context(n_inst=n, g=1, head_dim=64, block=8, hist_len=1, t_cap=nb * 8, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    K = torch.arange(n_pages, device="cuda:0", dtype=torch.int32).view(-1, 1, 1).expand(-1, 8, 32).contiguous().view(torch.bfloat16)      # a page's number, in its bits
    V = K.clone()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")  # noqa: E731
    table = torch.full((n, nb), -1, dtype=torch.int32, device="cuda:0")
    state = torch.zeros(ctx.pages_state_bytes(n_pages) // 4, dtype=torch.int32, device="cuda:0")
    ws, info = torch.full((ctx.pages_workspace_bytes(n_pages),), 255, dtype=torch.uint8, device="cuda:0"), torch.zeros(2, dtype=torch.int32, device="cuda:0")
    ctx.pages_count(table, n_pages, state)

    def free():
        """Free pages by the table alone, which counts and segments agree with."""
        refs = torch.bincount(table[table >= 0].long(), minlength=n_pages)
        assert torch.equal(state[:n_pages].long(), refs)
        zero = torch.nn.functional.pad(refs == 0, (0, -n_pages % 1024)).view(-1, 1024).sum(1)
        assert torch.equal(state[n_pages:].long(), zero)
        return (refs == 0).nonzero()[:, 0].int()

    full = i32([nb * 8 - 8 * (i % 3) for i in range(n)])
    ctx.pages_resize(K, V, table, state, full, None, 0, info, ws)
    assert info.tolist() == [n_pages, sum((full // 8).tolist()) - n_pages] and (table == -1).all() and len(free()) == n_pages   # too few
    lens = i32([nb * 8 - 8 * (i % 3) if i != 7 else 8 for i in range(n)])
    ctx.pages_resize(K, V, table, state, lens, None, 0, info, ws)
    rows = [table[i, :lens[i] // 8] for i in range(n)]
    used = sum((lens // 8).tolist())
    assert torch.equal(torch.cat(rows), torch.arange(used, device="cuda:0", dtype=torch.int32)) and info.tolist() == [n_pages - used, 0]
    free()
    # Half of it goes, anywhere; then others take the lowest of what is free.
    lens = i32([(int(x) if i % 2 else int(torch.randint(0, int(x) + 1, (1,), generator=rng))) // 8 * 8 for i, x in enumerate(lens.tolist())])
    ctx.pages_resize(K, V, table, state, lens, None, 0, info, ws)
    was, before = free(), table.clone()
    grown = i32([int(x) if i % 2 else min(nb * 8, int(x) + 8 * 1700) for i, x in enumerate(lens.tolist())])
    ctx.pages_resize(K, V, table, state, grown, None, 0, info, ws)
    new = table[(table >= 0) & (before < 0)]
    assert info.tolist() == [len(was) - len(new), 0] and torch.equal(new, was[:len(new)])
    free()
    ctx.pages_resize(K, V, table, state, lens, None, 0, info, ws)
    before = table.clone()
    gone = free()
    live = n_pages - len(gone)
    ctx.pages_compact(K, V, table, state, info, ws)
    moved = int((gone < live).sum())
    assert info.tolist() == [len(gone), moved] and int(table.max()) == live - 1 and len(free()) == len(gone)
    assert torch.equal(table < 0, before < 0)
    there = table >= 0
    assert torch.equal(K.view(torch.int32)[:, 0, 0][table[there].long()], before[there]) and torch.equal(V[table[there].long()], V[before[there].long()])
    stay = there & (before < live)
    assert torch.equal(table[stay], before[stay])


def test_needs_beyond_32_bits():
    """Tables with more entries than 32 bits count: what lacks is said as far as there is room for it, and nothing is changed."""
    import paper_2502_04077_amd as ap
    n, nb, b, d, n_pages = 65535, 65538, 8, 64, 4
    ctx = ap.Context(n_inst=n, g=1, head_dim=d, block=b, hist_len=1, t_cap=nb * b, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    K, V = (torch.full((n_pages, b, d), x, dtype=torch.bfloat16, device="cuda:0") for x in (1.0, 2.0))
    table = torch.full((n, nb), -1, dtype=torch.int32, device="cuda:0")
    state = torch.zeros(ctx.pages_state_bytes(n_pages) // 4, dtype=torch.int32, device="cuda:0")
    ws, info = torch.empty(ctx.pages_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda:0"), torch.zeros(2, dtype=torch.int32, device="cuda:0")
    ctx.pages_count(table, n_pages, state)
    for needs in (2 ** 32 + 2, 2 ** 32 - 1, 2 ** 31, 2 ** 31 + 3, 2 ** 31 + 4, n * nb, 5, 3):
        lens = torch.zeros(n, dtype=torch.int32)
        lens[:needs // nb] = nb * b
        if needs % nb:
            lens[needs // nb] = needs % nb * b
        ctx.pages_resize(K, V, table, state, lens.cuda(), None, 0, info, ws)
        if needs > n_pages:
            assert info.tolist() == [n_pages, min(needs - n_pages, 2 ** 31 - 1)] and state.tolist() == [0] * 4 + [4], needs
            assert int(table.max()) == -1 and (K == 1).all() and (V == 2).all(), needs
    assert info.tolist() == [1, 0] and table[0, :4].tolist() == [0, 1, 2, -1] and state.tolist() == [1, 1, 1, 0, 1]


def test_the_longest_list_of_pages():
    """As many entries as a call takes, which all but for the first lie outside the pools."""
    import ctypes as C

    import paper_2502_04077_amd as ap
    ctx = Device(ap, _pool(2, 2, 3, 8, 64, "bf16", 1), 16, 64).ctx
    src, dst = ([torch.randn((p, 8, 64), device="cuda:0").to(torch.bfloat16) for _ in range(2)] for p in (5, 7))
    want = [torch.cat([s, x[5:]]) for s, x in zip(src, dst)]
    for n in (2 ** 31 - 1, 2 ** 31 - 4096, 2 ** 31 - 4097):
        on = [x.clone() for x in dst]
        p = [C.c_void_p(x.data_ptr()) for x in src + on]
        rc = ap.load_library().ap_pages_copy(ctx._h, p[0], p[1], 5, None, p[2], p[3], 7, None, n, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()
        assert torch.equal(on[0], want[0]) and torch.equal(on[1], want[1])


def test_copies_follow_lists_in_a_graph():
    """Captured copies to other pages, to pinned memory and back, replayed with lists and pages that change."""
    import paper_2502_04077_amd as ap
    ctx = Device(ap, _pool(2, 2, 3, 16, 128, "bf16", 1), 32, 128).ctx
    K, V, K2, V2 = (torch.zeros((40, 16, 128), dtype=torch.bfloat16, device="cuda:0") for _ in range(4))
    host = [torch.zeros((10, 16, 128), dtype=torch.bfloat16, pin_memory=True) for _ in range(2)]
    src, dst = (torch.zeros(10, dtype=torch.int32, device="cuda:0") for _ in range(2))

    def calls():
        ctx.pages_copy(K, V, src, *host, None)
        ctx.pages_copy(*host, None, K2, V2, dst)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    gen = torch.Generator().manual_seed(4)
    for _ in range(4):
        for x in (K, V, K2, V2):
            x.copy_(torch.randn(x.shape, generator=gen).to(torch.bfloat16))
        src.copy_(torch.randperm(40, generator=gen)[:10])
        dst.copy_(torch.randperm(40, generator=gen)[:10])
        want = K2.clone(), V2.clone()
        for x, y in zip(want, (K, V)):
            x[dst.long()] = y[src.long()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(K2, want[0]) and torch.equal(V2, want[1])
        assert torch.equal(host[0], K[src.long()].cpu()) and torch.equal(host[1], V[src.long()].cpu())
