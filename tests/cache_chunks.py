"""The definition of cache_reference.attend for all queries of a chunk at a time, with the same bounds."""
import math

import torch

from cache_reference import HALF


def attend_chunk(q, K, V, base, window, n_first):
    """q [m][g][d], query r at position base + r, K and V [L][d]: outputs [m][g][d], weights summed over the queries [L], bounds of both.
    What no query sees may hold anything."""
    q, K, V = q.double(), K.double(), V.double()
    m, g, d = q.shape
    L = K.shape[0]
    j, p = torch.arange(L)[None, :], (base + torch.arange(m))[:, None]
    seen = j <= p
    if window > 0:
        seen &= (j > p - window) | (j < n_first)
    rows = seen.any(0)
    seen, K, V = seen[:, rows], K[rows], V[rows]
    count, nr = seen.sum(1), K.shape[0]
    x = (q.reshape(m * g, d) @ K.T).view(m, g, nr) / math.sqrt(d)
    P = torch.softmax(x.masked_fill(~seen[:, None, :], -math.inf), dim=2).nan_to_num(0.0)
    size = (q.reshape(m * g, d).abs() @ K.abs().T).view(m, g, nr).masked_fill(~seen[:, None, :], 0.0)
    size = size.flatten(1).amax(1) / math.sqrt(d) if size.numel() else torch.zeros(m, dtype=torch.float64)
    rel = 2 * (d + 4) * HALF[torch.float32] * size + (2 * count + 8) * HALF[torch.float32]
    w, w_off = torch.zeros(L, dtype=torch.float64), torch.zeros(L, dtype=torch.float64)
    w[rows], w_off[rows] = P.sum((0, 1)), (P.sum(1) * rel[:, None]).sum(0)
    by_size = (P.view(m * g, nr) @ V.abs()).view(m, g, d)
    return (P.view(m * g, nr) @ V).view(m, g, d), w, rel[:, None, None] * by_size, w_off, by_size
