"""PagedRun: calls on pages and attention over beginnings in common together, against a model of lists of rows in 64 bits (cache_reference.py,
which says how the bounds come about)."""
import math

import pytest
import torch

from cache_reference import HALF, attend, seen

pytestmark = pytest.mark.gpu
I32 = torch.int32


class Model:
    """A run, and the rows of every instance on the CPU."""

    def __init__(self, n_pages, dtype="bf16", window=0, seed=1, **kw):
        from paper_2502_04077_amd.runner import PagedRun
        from workloads import CONFIGS
        self.w = CONFIGS["cfg1"].with_(kv_heads=2, batch=4, t0=350, steps=50, budget_tokens=96, n_sink=1, n_local=2, g=4, kv_dtype=dtype, **kw)
        self.run = PagedRun(self.w, n_pages, "cuda:0", q_cap=120, window=window)
        self.run.K.fill_(math.nan)                         # rows that nobody wrote
        self.run.V.fill_(math.nan)
        self.n, self.g, self.d, self.window, self.first = self.w.n_inst, self.w.g, self.w.head_dim, window, self.run.n_first
        self.dt = self.w.torch_dtype()
        self.K, self.V = ([torch.zeros((0, self.d), dtype=self.dt)] * self.n for _ in range(2))
        self.gen = torch.Generator().manual_seed(seed)

    def i32(self, v):
        return torch.tensor(v, dtype=I32, device="cuda:0")

    def draw(self, *shape):
        return torch.randn(shape, generator=self.gen).to(self.dt)

    def _check(self, i, r, m, q, out, rounded):
        L = len(self.K[i])
        p = L - m + r
        ref, _, off, _ = attend(q, self.K[i], self.V[i], p, self.window, self.first)
        half = HALF[self.dt]
        if rounded and self.dt is torch.bfloat16:          # probabilities and outputs are rounded to bf16
            j = seen(p, L, self.window, self.first)
            P = torch.softmax(q.double() @ self.K[i][j].double().T / math.sqrt(self.d), dim=1)
            off = off + half * (P @ self.V[i][j].double().abs()) + half * ref.abs() * (1 + 2 * half)
        elif rounded:
            off = off + half * ref.abs()
        assert ((out.double() - ref).abs() <= off).all(), (i, r, (out.double() - ref).abs().max())

    def prefill(self, m, new):
        q, k, v = 2 * self.draw(self.n, m, self.g, self.d), self.draw(self.n, m, self.d), self.draw(self.n, m, self.d)
        out = self.run.prefill(q.cuda(), k.cuda(), v.cuda(), self.i32(new)).cpu()
        for i, x in enumerate(new):
            self.K[i], self.V[i] = torch.cat([self.K[i], k[i, :x]]), torch.cat([self.V[i], v[i, :x]])
            for r in range(x):
                self._check(i, r, x, q[i, r], out[i, r], True)
        self.whole()

    def step(self):
        q, k, v = 2 * self.draw(self.n, self.g, self.d), self.draw(self.n, self.d), self.draw(self.n, self.d)
        out = self.run.step(q.cuda(), k.cuda(), v.cuda()).cpu()
        for i in range(self.n):
            self.K[i], self.V[i] = torch.cat([self.K[i], k[i:i + 1]]), torch.cat([self.V[i], v[i:i + 1]])
            self._check(i, 0, 1, q[i], out[i], False)
        self.whole()

    def fork(self, parent):
        self.run.fork(self.i32(parent))
        none = torch.zeros((0, self.d), dtype=self.dt)
        self.K, self.V = ([x[p] if 0 <= p < self.n else none for p in parent] for x in (self.K, self.V))
        self.whole()

    def take_back(self, n):
        self.run.take_back(self.i32(n))
        self.K, self.V = ([x[:max(0, len(x) - max(0, m))] for x, m in zip(y, n)] for y in (self.K, self.V))
        self.whole()

    def end(self, which):
        self.run.end(torch.tensor([i in which for i in range(self.n)], device="cuda:0"))
        for i in which:
            self.K[i], self.V[i] = self.K[i][:0], self.V[i][:0]
        self.whole()

    def whole(self):
        """Lengths, rows, counts, and what groups say they have in common."""
        r, b = self.run, self.w.block
        table, lens, group, shared = r.table.cpu(), r.len.tolist(), r.group.tolist(), r.shared.tolist()
        assert lens == [len(x) for x in self.K]
        names = table[table >= 0].long()
        assert torch.equal(r.state[:r.n_pages].cpu().long(), torch.bincount(names, minlength=r.n_pages))
        K, V = r.K.cpu(), r.V.cpu()
        for i, L in enumerate(lens):
            pages = table[i, :-(-L // b)].long()
            assert torch.equal(K[pages].view(-1, self.d)[:L], self.K[i]) and torch.equal(V[pages].view(-1, self.d)[:L], self.V[i]), i
            if group[i] >= 0:
                lead, common = group.index(group[i]), min(shared[j] for j in range(self.n) if group[j] == group[i])
                assert torch.equal(self.K[i][:common], self.K[lead][:common]) and common <= L
        used = len(set(names.tolist()))
        assert r.free <= r.n_pages - used
        return used


@pytest.mark.parametrize("dtype,window,d", [("bf16", 0, 128), ("f32", 0, 64), ("bf16", 50, 64)])
def test_sequences_live_together(dtype, window, d):
    x = Model(150, dtype, window, head_dim=d)
    x.prefill(120, [120, 0, 0, 0, 77, 0, 1, 0])            # prompts
    x.prefill(120, [111, 0, 0, 0, 120, 0, 0, 0])
    x.fork([0, 0, 0, 0, 4, 4, 6, -1])                      # samples
    assert x.run.shared.tolist() == [231] * 4 + [197] * 2 + [0, 0]
    for _ in range(3):
        x.step()
    x.prefill(6, [6, 3, 0, 6, 1, 2, 6, 5])                 # drafts, and those not accepted
    x.take_back([2, 3, 0, 6, 0, 1, 9, 5])
    x.step()
    x.fork([1, 0, 0, 3, 5, 4, 6, 6])                       # beams change places
    x.step()
    away = x.run.set_aside([0, 4, 5])                      # sequences wait
    kept = [(x.K[i], x.V[i]) for i in (0, 4, 5)]
    for i in (0, 4, 5):
        x.K[i], x.V[i] = x.K[i][:0], x.V[i][:0]
    used = x.whole()
    x.run.compact()
    assert x.whole() == used and x.run.table.max() == used - 1
    x.step()
    x.end([0, 4, 5, 7])
    x.run.bring_back(away, [7, 0, 5])
    for i, (k, v) in zip((7, 0, 5), kept):
        x.K[i], x.V[i] = k, v
    x.whole()
    for _ in range(17):                                    # across an end of a page
        x.step()
    x.end([3])
    x.fork([2, 2, 2, 2, 7, 7, -1, 7])
    x.prefill(20, [20, 11, 0, 1, 20, 20, 20, 3])
    x.step()
    x.end(range(8))
    assert x.run.free_pages() == 150


def test_a_pool_that_is_full():
    x = Model(30)
    x.prefill(120, [120, 120, 120, 0, 0, 0, 0, 0])         # 8 pages each, the last one half full
    with pytest.raises(MemoryError):
        x.run.fork(x.i32([0] * 8))                         # 7 copies of a last page, and 6 are free
    assert x.whole() == 24
    x.end([2])
    x.fork([0] * 8)
    assert x.whole() == 7 + 8
    for _ in range(8 + 16):
        x.step()
    assert x.whole() == 7 + 16
    with pytest.raises(MemoryError):
        x.step()
    assert x.whole() == 23
    x.prefill(1, [1, 0, 1, 1, 1, 1, 1, 1])                 # 7 pages, just so
    assert x.whole() == 30
    x.end([1])
    assert x.whole() == 28
    x.step()
    assert x.whole() == 29


@pytest.mark.parametrize("number", [8, 15, 16, 1000, 2 ** 31 - 1])
def test_groups_of_any_number(number):
    """Groups that the caller names anew, by numbers that are no instance's, beside instances that stand alone."""
    x = Model(100)
    x.prefill(120, [100, 0, 0, 60, 50, 70, 0, 0])
    x.fork([0, 0, 0, 3, 4, 5, 0, -1])
    x.run.share(x.i32([number, number, -1, number - 8, -5, 2 ** 31 - 2, number, -1]), x.i32([100, 90, 100, 60, 50, 70, 95, 0]))
    assert x.run.group.tolist() == [0, 0, -1, -1, -1, -1, 0, -1] and x.run.shared.tolist() == [100, 90, 0, 0, 0, 0, 95, 0]
    x.step()
    x.fork([0, 1, 2, 3, 3, 5, 6, 3])
    assert x.run.group.tolist() == [0, 0, -1, 3, 3, -1, 0, 3] and x.run.shared.tolist() == [100, 90, 0, 61, 61, 0, 95, 61]
    x.step()
    x.end([0])
    assert x.run.group.tolist() == [-1, 1, -1, 3, 3, -1, 1, 3]
    x.prefill(7, [7, 7, 0, 7, 5, 7, 3, 1])
    x.take_back([0, 60, 0, 7, 5, 0, 0, 9])
    x.step()
