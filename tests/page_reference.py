"""Pages that instances share, from the definitions, on the CPU, page by page."""
import torch


def clamp(x, lo, hi):
    return max(lo, min(int(x), hi))


class Pool:
    """Tables, counts and rows of a pool: lists of whole numbers, and K, V [n_pages][b][d]."""

    def __init__(self, table, n_pages, b, K, V):
        self.table, self.n_pages, self.b, self.K, self.V = [list(r) for r in table], n_pages, b, K.clone(), V.clone()
        self.refs = [sum(r.count(p) for r in self.table) for p in range(n_pages)]

    def named(self, page):
        return 0 <= page < self.n_pages

    def free(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def copy(self, src, dst, rows):
        self.K[dst, :rows], self.V[dst, :rows] = self.K[src, :rows], self.V[src, :rows]

    def count_again(self):
        for p in range(self.n_pages):
            self.refs[p] = sum(r.count(p) for r in self.table)

    def resize(self, length, n_new, q_cap):
        """Returns info."""
        b, cap, needs = self.b, len(self.table[0]) * self.b, []
        for i, row in enumerate(self.table):
            L = clamp(length[i], 0, cap)
            n = min(L, q_cap if n_new is None else clamp(n_new[i], 0, q_cap))
            some = q_cap > 0 if n_new is None else clamp(n_new[i], 0, q_cap) > 0
            for k in range(-(-L // b)):
                mine = some and k >= (L - n) // b
                if not self.named(row[k]) or (mine and self.refs[row[k]] > 1):
                    needs.append((i, k, clamp(L - n - k * b, 0, b)))
        free = self.free()
        if len(needs) > len(free):
            return [len(free), len(needs) - len(free)]
        for (i, k, keep), page in zip(needs, free):
            if self.named(self.table[i][k]):
                self.copy(self.table[i][k], page, keep)
            self.table[i][k] = page
        for i, row in enumerate(self.table):
            for k in range(-(-clamp(length[i], 0, cap) // b), len(row)):
                row[k] = -1
        self.count_again()
        return [len(self.free()), 0]

    def fork(self, parent, length):
        """Returns the lengths and info."""
        n, b = len(self.table), self.b
        old, free, needs, now, lens = [list(r) for r in self.table], self.free(), [], [], []
        for j, p in enumerate(parent):
            if p == j:
                now.append(list(old[j]))
                lens.append(int(length[j]))
                continue
            L = clamp(length[p], 0, len(old[0]) * b) if 0 <= p < n else 0
            row = [old[p][k] if k < L // b else -1 for k in range(len(old[0]))]
            if L % b:
                last = old[p][L // b]
                heir = parent[p] != p and min(x for x in range(n) if parent[x] == p) == j
                row[L // b] = last
                if not heir and self.named(last):
                    needs.append((j, L // b, last, L % b))
            now.append(row)
            lens.append(L)
        if len(needs) > len(free):
            return [int(x) for x in length], [len(free), len(needs) - len(free)]
        for (j, k, last, rows), page in zip(needs, free):
            now[j][k] = page
            self.copy(last, page, rows)
        self.table = now
        self.count_again()
        return lens, [len(self.free()), 0]

    def compact(self):
        """Returns info."""
        live = self.n_pages - len(self.free())
        src = [p for p in range(live, self.n_pages) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        self.table = [[to.get(p, p) for p in r] for r in self.table]
        for a, c in to.items():
            self.copy(a, c, self.b)
        self.count_again()
        return [self.n_pages - live, len(to)]


class Device:
    """The same on the GPU, with the calls of a context."""

    def __init__(self, ap, pool, t_cap, d, g=1, dev="cuda:0"):
        self.n, self.b, self.n_pages, self.dev = len(pool.table), pool.b, pool.n_pages, dev
        self.ctx = ap.Context(n_inst=self.n, g=g, head_dim=d, block=self.b, hist_len=1, t_cap=t_cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4,
                              kv_dtype="bf16" if pool.K.dtype == torch.bfloat16 else "f32")
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        self.i32 = i32
        self.table, self.K, self.V = i32(pool.table), pool.K.to(dev), pool.V.to(dev)
        self.state = torch.full((self.ctx.pages_state_bytes(self.n_pages) // 4,), 77, dtype=torch.int32, device=dev)
        self.ws = torch.full((self.ctx.pages_workspace_bytes(self.n_pages),), 255, dtype=torch.uint8, device=dev)
        self.info = torch.full((2,), -5, dtype=torch.int32, device=dev)
        self.ctx.pages_count(self.table, self.n_pages, self.state)

    def resize(self, length, n_new, q_cap):
        self.ctx.pages_resize(self.K, self.V, self.table, self.state, self.i32(length), None if n_new is None else self.i32(n_new), q_cap, self.info, self.ws)
        return self.info.tolist()

    def fork(self, parent, length, in_place=True):
        len_in = self.i32(length)
        out = len_in if in_place else torch.full_like(len_in, -9)
        self.ctx.pages_fork(self.K, self.V, self.table, self.state, self.i32(parent), len_in, out, self.info, self.ws)
        return out.tolist(), self.info.tolist()

    def compact(self):
        self.ctx.pages_compact(self.K, self.V, self.table, self.state, self.info, self.ws)
        return self.info.tolist()

    def same(self, pool):
        """Asserts that tables, counts and every row are the reference's."""
        assert self.table.tolist() == pool.table
        assert self.state[:self.n_pages].tolist() == pool.refs
        free = [sum(pool.refs[p] == 0 for p in range(s, min(s + 1024, self.n_pages))) for s in range(0, self.n_pages, 1024)]
        assert self.state[self.n_pages:].tolist() == free
        bits = torch.int16 if pool.K.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(self.K.cpu().view(bits), pool.K.view(bits)) and torch.equal(self.V.cpu().view(bits), pool.V.view(bits))
