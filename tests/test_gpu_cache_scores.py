"""Scores of any size that 32 bits hold: attention over caches where one component of q and K makes them, as powers of two that every
product and sum holds exactly, up to 2^102, and below what 32 bits hold.  Neighbouring scores lie so far apart that the definition gives equal
weight to the rows with the largest one and none to the others, whatever the rounding of the scale."""
import pytest
import torch

from cache_reference import HALF, Cache, attend

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

SHAPES = [
    # g, d, dtype, paged, t_cap, q_cap, window, n_first, lens
    (4, 128, "bf16", True, 400, 5, 0, 0, [400, 17, 1, 0, 130]),
    (8, 64, "bf16", False, 304, 5, 37, 5, [304, 40, 5]),
    (1, 64, "f32", True, 2064, 3, 0, 0, [2049, 33]),
    (2, 128, "f32", False, 320, 9, 64, 4, [320, 70]),
    (4, 128, "bf16", True, 1040, 300, 0, 0, [1040] * 30 + [300, 301]),      # chunks in many workgroups
]
BELOW = "below"      # scores that 32 bits hold as -inf, in all rows but some of the last
SIZES = [(k, sign) for k in (20, 26, 31, 40, 100) for sign in (1, -1)] + [(BELOW, 1)]


def _inputs(shape, size, n_q):
    g, d, dt, paged, t_cap, q_cap, window, n_first, lens = SHAPES[shape]
    k, sign = size
    gen = torch.Generator().manual_seed(shape)
    c = Cache(len(lens), t_cap, d, 16, DT[dt], paged, shape)
    step = torch.randint(1, 5, (c.n, t_cap), generator=gen).float()
    if k == BELOW:
        step = torch.full((c.n, t_cap), -2.0 ** 20)
        for i, L in enumerate(lens):
            step[i, max(0, L - 1):L] = 0.0
            step[i, max(0, L - n_q - 2):max(0, L - n_q)] = 0.0
    c.K[:, :, 0] = step
    c.upload()
    q = torch.zeros((c.n, n_q, g, d))
    q[..., 0] = sign * 2.0 ** (120 if k == BELOW else k)
    return c, q.to(DT[dt])


def _ws(ctx, q_cap):
    return torch.full((ctx.cache_workspace_bytes(q_cap, True),), 255, dtype=torch.uint8, device="cuda:0")


def _expected(c, q, i, L, r, n_q, window, n_first):
    """Output, weights, and the sum of the outputs' terms by size."""
    p = L - n_q + r
    out, w, _, _ = attend(q[i, r], c.K[i, :L], c.V[i, :L], p, window, n_first)
    return out, w, (w[None, :] / q.shape[2]) @ c.V[i, :L].double().abs()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_decode(shape, size):
    import paper_2502_04077_amd as ap
    g, d, dt, paged, t_cap, _, window, n_first, lens = SHAPES[shape]
    c, q = _inputs(shape, size, 1)
    ctx = c.context(g, ap)
    L32 = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    both = []
    for weights in (True, False):
        out, acc = torch.full((c.n, g, d), 7.0, device="cuda:0"), torch.zeros((c.n, t_cap), device="cuda:0")
        ctx.cache_decode(q[:, 0].to("cuda:0").contiguous(), c.gK, c.gV, L32, window, n_first, out, acc if weights else None, _ws(ctx, 0))
        both.append(out.cpu().double())
        if weights:
            acc = acc.cpu().double()
            for i, L in enumerate(lens):
                _, w, _ = _expected(c, q, i, L, 0, 1, window, n_first)
                assert ((acc[i, :L] - w).abs() <= (2 * L + 16) * HALF[torch.float32] * w).all(), (i, L)
                assert not acc[i, L:].any()
    for i, L in enumerate(lens):
        ref, _, terms = _expected(c, q, i, L, 0, 1, window, n_first)
        for out in both:
            assert ((out[i] - ref).abs() <= (2 * L + 16) * HALF[torch.float32] * terms).all(), (i, L, (out[i] - ref).abs().max())


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefill(shape, size):
    import paper_2502_04077_amd as ap
    g, d, dt, paged, t_cap, q_cap, window, n_first, lens = SHAPES[shape]
    c, q = _inputs(shape, size, q_cap)
    ctx = c.context(g, ap)
    L32 = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    out, acc = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0"), torch.zeros((c.n, t_cap), device="cuda:0")
    ctx.cache_prefill(q.to("cuda:0"), None, c.gK, c.gV, L32, window, n_first, out, acc, _ws(ctx, q_cap))
    out, acc = out.cpu().double(), acc.cpu().double()
    half = HALF[DT[dt]]
    rows = range(q_cap) if q_cap < 20 else sorted(set(range(0, q_cap, 41)) | {q_cap - 1})
    for i, L in enumerate(lens):
        if i % 7 not in (0, 2, 3) and q_cap >= 20:
            continue
        total = torch.zeros(L, dtype=torch.float64)
        for r in range(q_cap):
            if r not in rows and q_cap >= 20 and i:
                continue
            ref, w, terms = _expected(c, q, i, L, r, q_cap, window, n_first)
            if size[0] == BELOW and len(w) and w.any() and c.K[i, :L, 0][w > 0].min() < 0:
                ref, w, terms = torch.zeros_like(ref), torch.zeros_like(w), torch.zeros_like(terms)      # nothing that has a weight in 32 bits
            total += w
            # as in test_gpu_cache.py: bf16 probabilities, equal ones, and one rounding of the output
            off = (2 * L + 16) * HALF[torch.float32] * terms + (half * terms if dt == "bf16" else 0) + half * ref.abs() * (1 + 2 * half)
            assert ((out[i, r] - ref).abs() <= off).all(), (i, L, r, (out[i, r] - ref).abs().max())
        if q_cap < 20 or i == 0:
            assert ((acc[i, :L] - total).abs() <= (2 * L + q_cap * g + 16) * HALF[torch.float32] * total).all(), (i, L)
            assert not acc[i, L:].any()


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_scores_above_32_bits_make_nan_of_their_head(shape):
    """The first head's scores pass 32 bits at the newest row: NaN there, in whatever form, and the other heads as without it."""
    import paper_2502_04077_amd as ap
    g, d, dt, paged, t_cap, q_cap, window, n_first, lens = SHAPES[shape]
    c, _ = _inputs(shape, (20, 1), 1)
    q = torch.randn((c.n, q_cap, g, d), generator=torch.Generator().manual_seed(shape)).to(DT[dt])
    for i, L in enumerate(lens):
        if L:
            c.K[i, L - 1] = 0.0
            c.K[i, L - 1, 0] = 2.0 ** 20
    c.upload()
    big = q.clone()
    big[:, -1, 0] = 0.0
    big[:, -1, 0, 0] = 2.0 ** 120
    ctx, L32, got = c.context(g, ap), torch.tensor(lens, dtype=torch.int32, device="cuda:0"), []
    for x in (q, big):
        out, one = torch.full(q.shape, 7.0, dtype=DT[dt], device="cuda:0"), torch.full((c.n, g, d), 7.0, device="cuda:0")
        ctx.cache_prefill(x.to("cuda:0"), None, c.gK, c.gV, L32, window, n_first, out, None, _ws(ctx, q_cap))
        ctx.cache_decode(x[:, -1].contiguous().to("cuda:0"), c.gK, c.gV, L32, window, n_first, one, None, _ws(ctx, 0))
        got.append((out.cpu(), one.cpu()))
    (out, one), (big_out, big_one) = got
    assert torch.equal(out[:, :-1], big_out[:, :-1]) and torch.equal(out[:, -1, 1:], big_out[:, -1, 1:]) and torch.equal(one[:, 1:], big_one[:, 1:])
    for i, L in enumerate(lens):
        if L:
            assert big_out[i, -1, 0].isnan().all() and big_one[i, 0].isnan().all(), (i, L)
        else:
            assert not big_out[i].any() and not big_one[i].any()
