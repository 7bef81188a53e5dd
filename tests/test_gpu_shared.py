"""Attention of instances whose first rows are the same, against the definitions in 64 bits (cache_reference.py, which says how the bounds come
about): groups of any size and order, beginnings that reach into tiles, windows that leave them, instances that are shorter than what they
share.  Rows that nobody sees hold NaN, workspaces and plans start with anything."""
import math

import pytest
import torch

from cache_reference import HALF, attend, seen

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Shared:
    """Caches [n][t_cap][d] whose groups begin alike, on the CPU, and the same on the GPU: contiguous, in pages of an instance's own, or with
    full pages of the rows in common shared."""

    def __init__(self, lens, group, shared, t_cap, d, b, dtype, layout, seed, first_p, window, n_first, dev="cuda:0"):
        gen = torch.Generator().manual_seed(seed)
        n = self.n = len(lens)
        self.t_cap, self.d, self.b, self.dtype, self.layout, self.dev = t_cap, d, b, dtype, layout, dev
        K, V = (torch.randn((n, t_cap, d), generator=gen).to(dtype) for _ in range(2))
        lead, common = {}, {}
        for i in range(n):
            if group[i] >= 0:
                lead.setdefault(group[i], i)
                common[group[i]] = min(common.get(group[i], t_cap), max(0, shared[i]))
        of = [lead[group[i]] if group[i] >= 0 else i for i in range(n)]
        S = [common[group[i]] if group[i] >= 0 else 0 for i in range(n)]
        for i in range(n):
            K[i, :S[i]], V[i, :S[i]] = K[of[i], :S[i]], V[of[i], :S[i]]
        # What nobody sees: in rows in common, nobody of the group.
        visible = torch.zeros((n, t_cap), dtype=torch.bool)
        for i, L in enumerate(lens):
            for p in range(max(0, first_p[i]), L):
                visible[i, seen(p, L, window, n_first)] = True
        for i in range(n):
            visible[of[i], :S[i]] |= visible[i, :S[i]]
        for i in range(n):
            visible[i, :S[i]] = visible[of[i], :S[i]]
        K[~visible], V[~visible] = math.nan, math.nan
        self.K, self.V, self.table = K, V, None
        if layout == "flat":
            self.gK, self.gV = K.to(dev), V.to(dev)
            return
        nb = t_cap // b
        self.n_pages = n * nb + 3
        names = torch.randperm(self.n_pages, generator=gen)[:n * nb].view(n, nb)
        if layout == "shared":
            for i in range(n):
                names[i, :S[i] // b] = names[of[i], :S[i] // b]
        pool = [torch.full((self.n_pages, b, d), math.nan, dtype=dtype) for _ in range(2)]
        for x, y in zip(pool, (K, V)):
            x[names.view(-1)] = y.view(-1, b, d)
        self.gK, self.gV = (x.to(dev) for x in pool)
        self.table = names.to(torch.int32).to(dev)

    def context(self, g, ap):
        x = ap.Context(n_inst=self.n, g=g, head_dim=self.d, block=self.b, hist_len=1, t_cap=self.t_cap, k_blocks=1, n_sink=0, n_local=0, c1=4,
                       c2=4, kv_dtype="bf16" if self.dtype == torch.bfloat16 else "f32")
        if self.table is not None:
            x.set_block_table(self.table, self.n_pages)
        return x


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda:0")


def _plan(ctx, group, shared):
    plan = torch.full((ctx.cache_share_bytes(),), 255, dtype=torch.uint8, device="cuda:0")
    ctx.cache_share(_i32(group), _i32(shared), plan)
    return plan


def _ws(ctx, q_cap=0):
    return torch.full((ctx.cache_shared_workspace_bytes(q_cap),), 255, dtype=torch.uint8, device="cuda:0")


def test_plan():
    """First member, place, number of members, rows in common, and the members one group after the other."""
    import paper_2502_04077_amd as ap
    gen = torch.Generator().manual_seed(1)
    for n, kinds in ((1, 1), (2, 1), (9, 4), (300, 7), (700, 500), (256, 1)):
        group = [int(x) - 1 for x in torch.randint(0, kinds + 1, (n,), generator=gen)]
        group = [2147483647 if x == 0 else -2147483648 if x == -1 else x for x in group]
        shared = [int(x) for x in torch.randint(-3, 60, (n,), generator=gen)]
        ctx = ap.Context(n_inst=n, g=1, head_dim=64, block=8, hist_len=1, t_cap=48, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
        words = _plan(ctx, group, shared).view(torch.int32).cpu()
        members = {}
        for i, x in enumerate(group):
            if x >= 0:
                members.setdefault(x, []).append(i)
        order, inst, pos = [], [[i, 0, 1, 0] for i in range(n)], [-1] * n
        for m in sorted((m for m in members.values() if len(m) > 1), key=lambda m: m[0]):
            for k, i in enumerate(m):
                inst[i] = [m[0], len(order), len(m), max(0, min(48, min(shared[x] for x in m)))]
                pos[i] = len(order) + k
            order += m
        groups = [inst[i] for i in range(n) if inst[i][0] == i and inst[i][2] > 1]
        assert words[:4 * n].view(n, 4).tolist() == inst and words[4 * n:8 * n].view(n, 4)[:len(groups)].tolist() == groups and words[8 * n] == len(groups)
        assert words[8 * n + 4:9 * n + 4].tolist() == pos and words[9 * n + 4:9 * n + 4 + len(order)].tolist() == order


def _many(n, f):
    return [f(i) for i in range(n)]


CASES = [
    # g, d, b, dtype, layout, t_cap, window, n_first, group, shared, lens
    (4, 128, 16, "bf16", "shared", 208, 0, 0, [5, 5, 5, 5, 5], [100] * 5, [101, 102, 150, 208, 117]),
    (4, 128, 16, "bf16", "own", 208, 0, 0, [0, -1, 1, 0, 1, 7, -3, 0], [64, 9, 33, 70, 40, 50, 1, 65], [65, 10, 208, 128, 41, 60, 0, 66]),
    (4, 128, 16, "bf16", "flat", 208, 0, 0, [3, 3, 3, 3, 3, 3], [90, 95, 90, 91, 200, 100], [90, 89, 200, 91, 0, 1]),      # no rows behind, and shorter than what is shared
    (2, 64, 8, "bf16", "flat", 200, 0, 0, [1, 1, 1], [150] * 3, [20, 190, 0]),                                             # the first is the shortest
    (8, 128, 8, "bf16", "shared", 400, 60, 0, [1, 0, 1, 0, 1, 1], [128, 200, 130, 200, 128, 140], [129, 201, 400, 230, 190, 187]),     # windows leave the beginning
    (8, 64, 32, "bf16", "shared", 416, 100, 37, [0, 0, 0, 0], [192] * 4, [193, 300, 416, 250]),
    (4, 128, 16, "bf16", "shared", 416, 10, 300, [0, 0, 0, 0], [200] * 4, [416, 380, 311, 250]),                            # first rows reach beyond the beginning
    (1, 128, 16, "bf16", "own", 416, 10, 5, [2, 2], [300, 300], [416, 390]),
    (1, 64, 64, "bf16", "shared", 256, 0, 0, [0, 0], [256, 256], [256, 256]),
    (4, 128, 16, "bf16", "shared", 304, 0, 0, [0] * 70, [260] * 70, _many(70, lambda i: 261 + (i * 7) % 44)),               # three tiles of queries
    (1, 128, 16, "bf16", "shared", 304, 0, 0, [0] * 129, [200] * 129, _many(129, lambda i: 200 + (i * 7) % 44)),            # one row in a second tile
    (2, 64, 8, "bf16", "shared", 64, 0, 0, _many(600, lambda i: i // 2 * 5), [40] * 600, _many(600, lambda i: 41 + i % 24)),  # many small groups
    (4, 64, 8, "bf16", "shared", 64, 30, 3, _many(300, lambda i: i % 7), _many(300, lambda i: 17 + i % 7), _many(300, lambda i: 24 + (i * 5) % 41)),
    (8, 128, 16, "bf16", "shared", 4112, 0, 0, [0, 0, 1, 1, -1], [4001, 4000, 3000, 3000, 0], [4100, 4001, 3007, 3001, 500]),  # pieces of many workgroups
    (2, 64, 8, "bf16", "flat", 40, 0, 0, _many(2600, lambda i: i % 50), [24] * 2600, _many(2600, lambda i: 24 + i % 17)),    # a wave an instance
    (4, 128, 16, "f32", "shared", 208, 0, 0, [5, 5, 5, 5, 5], [100] * 5, [101, 102, 150, 208, 117]),
    (8, 64, 8, "f32", "flat", 200, 50, 4, [1, 0, 1, 0, 1], [96, 64, 96, 64, 99], [97, 65, 130, 200, 96]),
    (1, 128, 32, "f32", "own", 608, 0, 0, [0] * 40, [500] * 40, _many(40, lambda i: 500 + i)),
    (2, 64, 16, "f32", "shared", 2064, 0, 0, [0, 0, -1, 4], [2000, 2000, 0, 70], [2001, 2064, 77, 70]),
    (4, 128, 16, "bf16", "shared", 112, 2147483647, 2147483647, [0, 0, 0], [80] * 3, [81, 112, 96]),
    (4, 64, 16, "bf16", "own", 48, 0, 0, [-1, -1, 6], [40, 40, 40], [48, 7, 30]),                                           # nobody shares
    (2, 128, 16, "bf16", "own", 48, 0, 0, [1, 1, 1], [0, -5, 40], [48, 7, 30]),                                             # a group without rows in common
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_decode(case):
    import paper_2502_04077_amd as ap
    g, d, b, dt, layout, t_cap, window, n_first, group, shared, lens = CASES[case]
    c = Shared(lens, group, shared, t_cap, d, b, DT[dt], layout, case, [L - 1 for L in lens], window, n_first)
    q = (2 * torch.randn((c.n, g, d), generator=torch.Generator().manual_seed(100 + case))).to(DT[dt])
    ctx = c.context(g, ap)
    out = torch.full((c.n, g, d), 7.0, device="cuda:0")
    ctx.cache_decode_shared(q.to("cuda:0"), c.gK, c.gV, _i32(lens), _plan(ctx, group, shared), window, n_first, out, _ws(ctx))
    out = out.cpu().double()
    for i, L in enumerate(lens):
        ref, _, off, _ = attend(q[i], c.K[i, :L], c.V[i, :L], L - 1, window, n_first)
        assert ((out[i] - ref).abs() <= off).all(), (i, L, (out[i] - ref).abs().max())


CHUNKS = [  # case, q_cap, n_q of instance i
    (0, 1, lambda i: 1), (0, 16, lambda i: [1, 2, 16, 0, 7][i]), (0, 60, lambda i: [1, 2, 50, 60, 17][i]),      # (rows in common lie in front of the new ones, or not)
    (1, 5, lambda i: 1 + i % 5), (2, 3, lambda i: 3 - i % 4 if i < 4 else 1), (3, 9, lambda i: 9),
    (4, 8, lambda i: 1 + i), (5, 7, lambda i: 7 - i), (6, 13, lambda i: 13), (7, 31, lambda i: 30 + i), (9, 2, lambda i: 1 + i % 2),
    (10, 33, lambda i: 1 + (i * 3) % 33), (11, 3, lambda i: i % 4), (13, 4, lambda i: 4 - i % 4), (15, 4, lambda i: 4), (16, 3, lambda i: 1 + i % 3),
    (17, 20, lambda i: 1 + i % 20), (18, 5, lambda i: 5), (19, 2, lambda i: 2), (20, 4, lambda i: 3), (21, 32, lambda i: 7),
]


@pytest.mark.parametrize("chunk", range(len(CHUNKS)))
def test_prefill(chunk):
    import paper_2502_04077_amd as ap
    case, q_cap, count = CHUNKS[chunk]
    g, d, b, dt, layout, t_cap, window, n_first, group, shared, lens = CASES[case]
    new = [max(0, min(q_cap, count(i))) for i in range(len(lens))]
    c = Shared(lens, group, shared, t_cap, d, b, DT[dt], layout, case, [L - m for L, m in zip(lens, new)], window, n_first)
    q = (2 * torch.randn((c.n, q_cap, g, d), generator=torch.Generator().manual_seed(200 + chunk))).to(DT[dt])
    for i, m in enumerate(new):
        q[i, m:] = math.nan
    ctx = c.context(g, ap)
    out = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0")
    ctx.cache_prefill_shared(q.to("cuda:0"), _i32(new) if chunk % 3 or min(new) < q_cap else None, c.gK, c.gV, _i32(lens), _plan(ctx, group, shared), window, n_first, out,
                             _ws(ctx, q_cap))
    out, half = out.cpu(), HALF[DT[dt]]
    for i, (L, m) in enumerate(zip(lens, new)):
        for r in range(m):
            p = L - m + r
            ref, _, off, _ = attend(q[i, r], c.K[i, :L], c.V[i, :L], p, window, n_first)
            if dt == "bf16":                               # probabilities and outputs are rounded to bf16
                j = seen(p, L, window, n_first)
                P = torch.softmax(q[i, r].double() @ c.K[i, j].double().T / math.sqrt(d), dim=1) if len(j) else torch.zeros(g, 0).double()
                off = off + half * (P @ c.V[i, j].double().abs()) + half * ref.abs() * (1 + 2 * half)
            else:
                off = off + half * ref.abs()
            assert ((out[i, r].double() - ref).abs() <= off).all(), (i, L, r, (out[i, r].double() - ref).abs().max())
        assert (out[i, m:] == 7).all(), i


def test_rows_without_tokens_hold_anything():
    """Queries that are none are NaN, and those of other members of their tile are not touched by it."""
    import paper_2502_04077_amd as ap
    lens, new = [70, 80, 75], [0, 2, 0]
    c = Shared(lens, [0, 0, 0], [64] * 3, 80, 64, 8, torch.bfloat16, "shared", 3, [70, 78, 75], 0, 0)
    q = torch.full((3, 4, 2, 64), math.nan, dtype=torch.bfloat16)
    q[1, :2] = torch.randn((2, 2, 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    ctx, out = c.context(2, ap), torch.full((3, 4, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_prefill_shared(q.to("cuda:0"), _i32(new), c.gK, c.gV, _i32(lens), _plan(ctx, [0, 0, 0], [64] * 3), 0, 0, out, _ws(ctx, 4))
    out = out.cpu()
    assert (out[0] == 7).all() and (out[2] == 7).all() and (out[1, 2:] == 7).all()
    for r in range(2):
        ref = attend(q[1, r], c.K[1, :80], c.V[1, :80], 78 + r, 0, 0)[0]
        assert (out[1, r].double() - ref).abs().max() <= 3 * HALF[torch.bfloat16] * c.V[1, :80].float().abs().max()


def test_shared_is_what_each_alone_is():
    """The same caches, by groups and alone: outputs within both bounds of each other, and the same whatever order the groups are in."""
    import paper_2502_04077_amd as ap
    lens, shared = [900 + 3 * i for i in range(24)], [880] * 24
    group = [i % 3 for i in range(24)]
    c = Shared(lens, group, shared, 1008, 128, 16, torch.bfloat16, "shared", 11, [L - 1 for L in lens], 0, 0)
    q = torch.randn((24, 4, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to("cuda:0")
    ctx, outs = c.context(4, ap), []
    for name in (group, [9 - x for x in group], [-1] * 24):
        out = torch.zeros((24, 4, 128), device="cuda:0")
        ctx.cache_decode_shared(q, c.gK, c.gV, _i32(lens), _plan(ctx, name, shared), 0, 0, out, _ws(ctx))
        outs.append(out)
    alone = torch.zeros((24, 4, 128), device="cuda:0")
    ctx.cache_decode(q, c.gK, c.gV, _i32(lens), 0, 0, alone, None, torch.zeros(ctx.cache_workspace_bytes(0, False), dtype=torch.uint8, device="cuda:0"))
    assert torch.equal(outs[0], outs[1])
    for i, L in enumerate(lens):
        off = attend(q[i].cpu(), c.K[i, :L], c.V[i, :L], L - 1, 0, 0)[2]
        for out in (outs[0], outs[2]):
            assert ((out[i].cpu().double() - alone[i].cpu().double()).abs() <= 2 * off).all()
