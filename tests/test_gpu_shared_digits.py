"""Digits of chunks of few tokens behind beginnings in common, bf16: a chunk's output is off by the rounding of the output itself and by little else.

Probabilities go into the second product as two bf16 numbers each: the first is off by half a step, 2^-8 relative, the second, of what is left, by as much of
it, so that 2^-16 is.  The rest as in cache_reference.py."""
import pytest
import torch

from cache_reference import HALF, attend
from test_gpu_shared import Shared, _i32, _plan, _ws

pytestmark = pytest.mark.gpu

SHAPES = [
    # g, d, layout, t_cap, m, window, n_first, seqs, lens' step
    (4, 128, "shared", 704, 5, 0, 0, 20, 7),               # tiles of a workgroup, and of a wave behind them
    (8, 64, "own", 512, 4, 0, 0, 9, 11),
    (1, 128, "shared", 400, 8, 90, 3, 6, 5),               # a wave's alone
    (2, 64, "flat", 320, 16, 70, 2, 3, 30),                # two rows of 16
    (4, 64, "shared", 256, 2, 0, 0, 1, 0),
]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_probabilities_of_few_tokens_keep_their_digits(shape):
    import paper_2502_04077_amd as ap
    g, d, layout, t_cap, m, window, n_first, seqs, step = SHAPES[shape]
    S = t_cap // 2
    lens = [S + 10 + m + step * i for i in range(seqs)]
    group, shared = [0] * seqs, [S] * seqs
    c = Shared(lens, group, shared, t_cap, d, 16, torch.bfloat16, layout, shape, [0] * seqs, 0, 0)
    q = (2 * torch.randn((seqs, m, g, d), generator=torch.Generator().manual_seed(shape))).to(torch.bfloat16)
    ctx = c.context(g, ap)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda:0")
    ctx.cache_prefill_shared(q.cuda(), None, c.gK, c.gV, _i32(lens), _plan(ctx, group, shared), window, n_first, out, _ws(ctx, m))
    out, half = out.cpu().double(), HALF[torch.bfloat16]
    for i, L in enumerate(lens):
        K, V = c.K[i, :L].nan_to_num(0), c.V[i, :L].nan_to_num(0)
        for r in range(m):
            p = L - m + r
            ref, _, off, _ = attend(q[i, r], K, V, p, window, n_first)
            terms = attend(q[i, r], K, V.abs(), p, window, n_first)[0]
            off = off + 2.0 ** -16 * terms
            assert ((out[i, r] - ref).abs() <= off + half * (ref.abs() + off)).all(), (i, r, (out[i, r] - ref).abs().max())
