"""Attention over caches with lengths of their own, and eviction, from their definitions in 64 bits, one instance at a time on the CPU;
and bounds on what the kernels' arithmetic may add, worked out from the numbers of the case."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


def seen(p, L, window, n_first):
    """Rows that a query at position p of a cache of L rows sees."""
    j = torch.arange(max(0, min(p + 1, L)))
    return j if window <= 0 else j[(j > p - window) | (j < n_first)]


def attend(q, K, V, p, window, n_first):
    """q [g][d], K and V [L][d]: output [g][d], weight of every row [L], bounds of both."""
    q, K, V = q.double(), K.double(), V.double()
    g, d = q.shape
    j = seen(p, K.shape[0], window, n_first)
    out, w = torch.zeros(g, d, dtype=torch.float64), torch.zeros(K.shape[0], dtype=torch.float64)
    out_off, w_off = torch.zeros_like(out), torch.zeros_like(w)
    if not len(j):
        return out, w, out_off, w_off
    P = torch.softmax(q @ K[j].T / math.sqrt(d), dim=1)
    out, w[j] = P @ V[j], P.sum(0)
    # A score is a sum of d products in 32 bits (exact ones for bf16, rounded once for fp32), times a constant, in an exponent: off by at
    # most d + 4 roundings of the sum of its terms' sizes.  A probability moves by that, relative, and by as much again with the sum it is
    # divided by; sums over n rows add n roundings of their terms' sizes, and the rest (exponential, division) at most 8.
    size = (q.abs() @ K[j].abs().T).max().item() / math.sqrt(d)
    rel = 2 * (d + 4) * HALF[torch.float32] * size + (2 * len(j) + 8) * HALF[torch.float32]
    out_off = rel * (P @ V[j].abs())
    w_off[j] = rel * P.sum(0)
    return out, w, out_off, w_off


def evict(acc, L, budget, n_first, n_last):
    """Indices of the rows that stay, ascending."""
    if L <= budget:
        return list(range(L))
    middle = sorted(range(n_first, L - n_last), key=lambda j: (-float(acc[j]) + 0.0, j))
    return sorted(list(range(n_first)) + middle[:budget - n_first - n_last] + list(range(L - n_last, L)))


class Cache:
    """A paged or contiguous cache on the GPU, and the same rows as one [n][t_cap][d] tensor on the CPU."""

    def __init__(self, n, t_cap, d, b, dtype, paged, seed, dev="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        self.n, self.t_cap, self.d, self.b, self.paged = n, t_cap, d, b, paged
        self.K, self.V = (torch.randn((n, t_cap, d), generator=g).to(dtype) for _ in range(2))
        self.table = self.table_cpu = None
        nb = t_cap // b
        if paged:
            self.n_pages = n * nb + 3
            self.table_cpu = torch.randperm(self.n_pages, generator=g)[:n * nb].view(n, nb)
            self.table = self.table_cpu.to(torch.int32).to(dev)
        self.dev = dev
        self.gK, self.gV = self.put(self.K), self.put(self.V)

    def put(self, x):
        if not self.paged:
            return x.to(self.dev)
        pool = torch.full((self.n_pages, self.b, self.d), math.nan, dtype=x.dtype)
        pool[self.table_cpu.view(-1)] = x.view(-1, self.b, self.d)
        return pool.to(self.dev)

    def get(self, x):
        x = x.cpu()
        return x if not self.paged else x[self.table_cpu.view(-1)].view(self.n, self.t_cap, self.d)

    def upload(self):
        self.gK, self.gV = self.put(self.K), self.put(self.V)

    def context(self, g, ap):
        x = ap.Context(n_inst=self.n, g=g, head_dim=self.d, block=self.b, hist_len=1, t_cap=self.t_cap, k_blocks=1, n_sink=0, n_local=0, c1=4,
                       c2=4, kv_dtype="bf16" if self.K.dtype == torch.bfloat16 else "f32")
        if self.paged:
            x.set_block_table(self.table, self.n_pages)
        return x
