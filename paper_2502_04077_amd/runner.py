"""Device buffers and call sequencing for a Workload: allocation and bookkeeping only.

Holds the tensors one decode run needs (history ring, pred, idx, out, row, workspace) and drives
the C-ABI calls in the order of Algorithm 1.  No arithmetic of the method happens here.
"""
from __future__ import annotations

import torch

from .binding import AP_PRED_ADVANCE, AP_PRED_HOLD, AP_PRED_REBASE, AP_PRED_SKIP, AP_STEP_REUSE_SELECTION, Context


class DecodeRun:
    def __init__(self, w, device="cuda:0", incremental=True, rebase_every=512, flags=0, refresh_every=1):
        """incremental: carry the predictor's interior state across steps (ap_predict_incremental)
        and re-evaluate the full tile every `rebase_every` pushes; False evaluates the full tile
        on every step.  refresh_every: the selection is re-made on every refresh_every-th step and
        carried over (ap_refresh_selection) on the others (Sec. 3.3).  The predictor state then either
        advances on every step anyway, or - from skip_predictor_from steps between selections on - the
        predictor is left out on the steps in between and evaluates the full tile when it is needed
        (one full tile costs about as much as a dozen advances)."""
        self.w = w
        self.refresh_every = refresh_every
        self.skip_predictor_from = 12
        self.steps_done = 0
        self.incremental = incremental
        self.rebase_every = rebase_every
        self.state_n = None       # n_pushed the predictor state is valid for
        self.state_t = None       # t_cur of the call that wrote it
        self.dev = torch.device(device)
        self.ctx = Context(n_inst=w.n_inst, g=w.g, head_dim=w.head_dim, block=w.block, hist_len=w.hist_len,
                           t_cap=w.t_cap, k_blocks=w.k_blocks, n_sink=w.n_sink, n_local=w.n_local,
                           c1=w.c1, c2=w.c2, kv_dtype=w.kv_dtype, flags=flags)
        R, nbc = self.ctx.hist_slots(), self.ctx.nb_cap()
        self.R, self.nb_cap = R, nbc
        f32, i32 = torch.float32, torch.int32
        self.hist = torch.zeros((w.n_inst, R, nbc), dtype=f32, device=self.dev)
        self.pred = torch.zeros((w.n_inst, nbc), dtype=f32, device=self.dev)
        self.pstate = torch.zeros((w.n_inst, nbc), dtype=f32, device=self.dev)
        self.row = torch.zeros((w.n_inst, nbc), dtype=f32, device=self.dev)
        self.idx = torch.zeros((w.n_inst, w.k_blocks), dtype=i32, device=self.dev)
        self.cnt = torch.zeros((w.n_inst,), dtype=i32, device=self.dev)
        self.out = torch.zeros((w.n_inst, w.g, w.head_dim), dtype=f32, device=self.dev)
        self.ws = torch.zeros((max(16, self.ctx.workspace_bytes()),), dtype=torch.uint8, device=self.dev)
        self.n_pushed = 0

    def set_weights(self, blob):
        self.ctx.set_weights(blob)

    def nb(self, t):
        return (t + self.w.block - 1) // self.w.block

    def logical_history(self, instances=None) -> torch.Tensor:
        """The H-row window in logical order (index H-1 = newest) as a new tensor
        [len(instances) or n_inst][H][nb_cap]."""
        H, R = self.w.hist_len, self.R
        slots = torch.tensor([(self.n_pushed - H + r) % R for r in range(H)], device=self.dev)
        src = self.hist if instances is None else self.hist[torch.as_tensor(list(instances), device=self.dev)]
        h = src.index_select(1, slots)
        for r in range(H):
            if self.n_pushed - H + r < 0:
                h[:, r, :] = 0
        return h

    def warmup_calibrate(self, q, K, t):
        """Push the dense pooled row of (q, K[:t]) - used for the prefill tail and calibration."""
        self.ctx.calibrate(q, K, t, self.row, self.ws)
        self.ctx.update_history(self.hist, self.n_pushed, self.row)
        self.n_pushed += 1

    def _pred_mode(self, t):
        """Which predictor mode is valid now, and the bookkeeping for the next call."""
        if not self.incremental:
            return AP_PRED_REBASE
        n = self.n_pushed
        if self.state_n == n and self.state_t == t:
            mode = AP_PRED_HOLD
        elif self.state_n == n - 1 and self.state_t == t - 1 and n % self.rebase_every != 0:
            mode = AP_PRED_ADVANCE
        else:
            mode = AP_PRED_REBASE
        return mode

    def selects_now(self, t):
        """Whether the step at context length t re-makes the selection (else it carries the last one over)."""
        k = self.w.k_blocks
        return (self.steps_done % self.refresh_every == 0 or self.nb(t - 1) <= k < self.nb(t)
                or self.nb(t) <= k)

    def _step_mode(self, t, selects):
        """Predictor mode of this step; AP_PRED_SKIP on steps that carry the selection over under a long interval."""
        if not selects and self.refresh_every >= self.skip_predictor_from:
            return AP_PRED_SKIP
        return self._pred_mode(t)

    def step_unfused(self, q, K, V, t, calibrate=False):
        nb = self.nb(t)
        selects = self.selects_now(t)
        mode = self._step_mode(t, selects)
        if mode == AP_PRED_SKIP:
            pass
        elif self.incremental:
            self.ctx.predict_incremental(self.hist, self.n_pushed, nb, self.nb(max(t - 1, 1)), mode, self.pstate,
                                         self.pred, self.ws)
            self.state_n, self.state_t = self.n_pushed, t
        else:
            self.ctx.predict(self.hist, self.n_pushed, nb, self.pred, self.ws)
        if selects:
            self.ctx.select_topk(self.pred, nb, self.idx, self.cnt, self.ws)
        elif nb != self.nb(t - 1):
            self.ctx.refresh_selection(self.nb(t - 1), nb, self.idx, self.cnt)
        self.ctx.sparse_decode(q, K, V, t, self.idx, self.cnt, self.out, self.row, self.ws)
        if calibrate:
            self.ctx.calibrate(q, K, t, self.row, self.ws)
        self.ctx.update_history(self.hist, self.n_pushed, self.row)
        self.n_pushed += 1
        self.steps_done += 1
        return mode

    def step(self, q, K, V, t, calibrate=False):
        selects = self.selects_now(t)
        mode = self._step_mode(t, selects)
        flag = 0 if selects else AP_STEP_REUSE_SELECTION
        self.ctx.step(self.hist, self.n_pushed, q, K, V, t, self.out, self.idx, self.cnt, self.pred,
                      self.pstate if self.incremental else None, mode | flag, self.ws)
        if self.incremental and mode != AP_PRED_SKIP:
            self.state_n, self.state_t = self.n_pushed, t
        if calibrate:
            self.ctx.calibrate(q, K, t, self.row, self.ws)
            self.ctx.update_history(self.hist, self.n_pushed, self.row)
        self.n_pushed += 1
        self.steps_done += 1
        return mode


class DenseRun:
    """Layers that attend to the whole cache in every step (Sec. 4.1 keeps the first two layers uncompressed):
    the same attention kernel with a budget of all blocks, no history and no predictor."""

    def __init__(self, w, n_layers, device="cuda:0"):
        self.w = w
        self.dev = torch.device(device)
        self.n_inst = n_layers * w.batch * w.kv_heads
        self.ctx = Context(n_inst=self.n_inst, g=w.g, head_dim=w.head_dim, block=w.block, hist_len=w.hist_len,
                           t_cap=w.t_cap, k_blocks=w.nb_cap, n_sink=0, n_local=0, c1=w.c1, c2=w.c2,
                           kv_dtype=w.kv_dtype)
        f32, i32 = torch.float32, torch.int32
        nbc = self.ctx.nb_cap()
        self.idx = torch.zeros((self.n_inst, nbc), dtype=i32, device=self.dev)
        self.cnt = torch.zeros((self.n_inst,), dtype=i32, device=self.dev)
        self.row = torch.zeros((self.n_inst, nbc), dtype=f32, device=self.dev)
        self.out = torch.zeros((self.n_inst, w.g, w.head_dim), dtype=f32, device=self.dev)
        self.ws = torch.zeros((max(16, self.ctx.workspace_bytes()),), dtype=torch.uint8, device=self.dev)
        self.nb_listed = 0

    def step(self, q, K, V, t):
        nb = (t + self.w.block - 1) // self.w.block
        if nb != self.nb_listed:                          # all blocks: no scores are read
            self.ctx.select_topk(self.row, nb, self.idx, self.cnt, self.ws)
            self.nb_listed = nb
        self.ctx.sparse_decode(q, K, V, t, self.idx, self.cnt, self.out, self.row, self.ws)


class _Lengths:
    """Caches whose lengths `len` live on the device; the host only knows `longest`, which none exceeds."""

    def _grow(self, n, by):
        if self.longest + by > self.w.t_cap:
            raise ValueError(f"caches of up to {self.longest} rows have no room for {by} more (t_cap = {self.w.t_cap})")
        self.len += n
        self.longest += by

    def _grown(self, n, by, calls):
        """The calls on caches that are n rows longer.  If one of them is refused, the lengths are what they were: rows behind them
        hold nothing."""
        if self.longest + by > self.w.t_cap:
            # The bound counts every token of a chunk, the caches may be shorter: only now are the device's lengths asked, and waited for.
            self.longest, after = torch.stack([self.len.max(), (self.len + n).max()]).tolist()
            by = after - self.longest
        longest = self.longest
        self._grow(n, by)
        try:
            calls()
        except Exception:
            self.len -= n
            self.longest = longest
            raise


class CacheRun(_Lengths):
    """Layers whose caches have lengths of their own: prompts of different lengths go in by chunks, every token attends to its whole
    cache (or to a window and the first rows), and every `evict_every` steps caches beyond the budget lose the rows that gathered the
    least attention weight - the eviction that the predicted selection of DecodeRun is an alternative to.  The first n_sink and the last
    n_local blocks of the workload's budget stay, as there; no history and no predictor.

    Every instance starts empty.  The lengths live on the device, so the host only knows how long a cache can be at most; it asks for them
    where that is too long for what is to come."""

    def __init__(self, w, device="cuda:0", q_cap=1, window=0, evict_every=64, table=None, n_pages=0):
        """q_cap: most tokens of a chunk.  table: int32 [n_inst][nb_cap] into a pool of n_pages pages, every page an instance's own;
        None for the contiguous layout."""
        self.w, self.q_cap, self.window, self.evict_every = w, q_cap, window, evict_every
        self.dev = torch.device(device)
        self.ctx = Context(n_inst=w.n_inst, g=w.g, head_dim=w.head_dim, block=w.block, hist_len=w.hist_len, t_cap=w.t_cap,
                           k_blocks=w.k_blocks, n_sink=w.n_sink, n_local=w.n_local, c1=w.c1, c2=w.c2, kv_dtype=w.kv_dtype)
        self.table = table
        if table is not None:
            self.ctx.set_block_table(table, n_pages)
        self.n_first, self.n_last = w.n_sink * w.block, w.n_local * w.block
        shape = (w.n_inst, w.t_cap, w.head_dim) if table is None else (n_pages, w.block, w.head_dim)
        self.K = torch.zeros(shape, dtype=w.torch_dtype(), device=self.dev)
        self.V = torch.zeros_like(self.K)
        self.len = torch.zeros((w.n_inst,), dtype=torch.int32, device=self.dev)
        self.acc = torch.zeros((w.n_inst, w.t_cap), dtype=torch.float32, device=self.dev)
        self.kept = torch.zeros((w.n_inst, w.budget_tokens), dtype=torch.int32, device=self.dev)
        self.out = torch.zeros((w.n_inst, w.g, w.head_dim), dtype=torch.float32, device=self.dev)
        self.chunk_out = torch.zeros((w.n_inst, q_cap, w.g, w.head_dim), dtype=w.torch_dtype(), device=self.dev)
        size = max(16, self.ctx.cache_workspace_bytes(q_cap, True))
        self.ws = torch.zeros((size,), dtype=torch.uint8, device=self.dev)
        self.steps_done = 0
        self.longest = 0          # no cache is longer than this

    def prefill(self, q, k, v, n_new=None):
        """The next chunk of every prompt, q [n_inst][m][g][d] and k, v [n_inst][m][d] with m <= q_cap; n_new: int32 [n_inst], how many
        of the m tokens count.  Returns the outputs [n_inst][m][g][d], a buffer that the next chunk uses again; its rows from n_new[i]
        on hold nothing of this chunk."""
        m = q.shape[1]
        if m > self.q_cap:
            raise ValueError(f"a chunk has at most q_cap = {self.q_cap} tokens")
        if k.shape[:2] != q.shape[:2] or v.shape[:2] != q.shape[:2]:
            raise ValueError(f"{list(q.shape[:2])} queries and rows k, v of {list(k.shape[:2])}, {list(v.shape[:2])}")
        out = self.chunk_out.view(-1)[:q.numel()].view(q.shape)

        def calls():
            self.ctx.cache_append(k, v, n_new, self.len, self.K, self.V)
            self.ctx.cache_prefill(q, n_new, self.K, self.V, self.len, self.window, self.n_first, out, self.acc, self.ws)
        self._grown(m if n_new is None else n_new.clamp(0, m), m, calls)
        return out

    def step(self, q, k, v):
        """One decode step: q [n_inst][g][d], k and v [n_inst][d].  Returns the outputs, float [n_inst][g][d], a buffer that the
        next step uses again."""
        def calls():
            self.ctx.cache_append(k.unsqueeze(1), v.unsqueeze(1), None, self.len, self.K, self.V)
            self.ctx.cache_decode(q, self.K, self.V, self.len, self.window, self.n_first, self.out, self.acc, self.ws)
        self._grown(1, 1, calls)
        self.steps_done += 1
        if self.steps_done % self.evict_every == 0:
            self.evict()
        return self.out

    def evict(self):
        self.ctx.cache_evict(self.K, self.V, self.acc, self.len, self.w.budget_tokens, self.n_first, self.n_last, self.acc, self.len,
                             self.kept)
        self.longest = min(self.longest, self.w.budget_tokens)


class PagedRun(_Lengths):
    """Sequences whose pages come from one pool as they grow, and whose beginnings in common are held once and read once: samples and beams
    that go on from one another (`fork`), drafted tokens that are taken back (`take_back`), sequences that end (`end`) or wait in host memory
    (`set_aside`, `bring_back`).  Every token attends to its whole cache, or to a window and the first n_sink blocks of the workload's budget.

    Every instance starts empty and alone.  Lengths, tables and counts live on the device; the host knows how many pages are free at least,
    and asks only where that might not do.  What is refused, for want of pages too, leaves every cache as it was."""

    def __init__(self, w, n_pages, device="cuda:0", q_cap=1, window=0):
        """n_pages: of the pool, for all instances.  q_cap: most tokens of a chunk."""
        self.w, self.q_cap, self.window, self.n_pages = w, q_cap, window, n_pages
        self.dev = torch.device(device)
        self.ctx = Context(n_inst=w.n_inst, g=w.g, head_dim=w.head_dim, block=w.block, hist_len=w.hist_len, t_cap=w.t_cap,
                           k_blocks=w.k_blocks, n_sink=w.n_sink, n_local=w.n_local, c1=w.c1, c2=w.c2, kv_dtype=w.kv_dtype)
        self.n_first = w.n_sink * w.block
        new = lambda shape, dtype, value=0: torch.full(shape, value, dtype=dtype, device=self.dev)  # noqa: E731
        i32, u8, n = torch.int32, torch.uint8, w.n_inst
        self.table = new((n, w.t_cap // w.block), i32, -1)
        self.ctx.set_block_table(self.table, n_pages)
        self.K = new((n_pages, w.block, w.head_dim), w.torch_dtype())
        self.V = torch.zeros_like(self.K)
        self.state = new((self.ctx.pages_state_bytes(n_pages) // 4,), i32)
        self.info = new((2,), i32)
        self.pages_ws = new((max(16, self.ctx.pages_workspace_bytes(n_pages)),), u8)
        self.len = new((n,), i32)
        self.none_new = new((n,), i32)
        self.group, self.shared = new((n,), i32, -1), new((n,), i32)
        self.plan = new((max(16, self.ctx.cache_share_bytes()),), u8)
        self.ws = new((max(16, self.ctx.cache_shared_workspace_bytes(q_cap)),), u8)
        self.out = new((n, w.g, w.head_dim), torch.float32)
        self.chunk_out = new((n, q_cap, w.g, w.head_dim), w.torch_dtype())
        self.free = n_pages        # at least so many pages are free
        self.longest = 0           # no cache is longer than this
        self.ctx.pages_count(self.table, n_pages, self.state)
        self._share(self.group, self.shared)

    # -- pages ------------------------------------------------------------------------------------
    def _given(self, most, call):
        """A call that takes at most so many pages: where fewer may be free, what it says is waited for."""
        call()
        if most <= self.free:
            self.free -= most
        else:
            self.free, lacking = self.info.tolist()
            if lacking > 0:
                raise MemoryError(f"{self.free} of {self.n_pages} pages are free, {lacking} too few")

    def _resize(self, n_new, m):
        """The tables of caches of `len` rows, of which n_new (None: m) are about to be written; at most m each."""
        most = self.w.n_inst * ((m + self.w.block - 2) // self.w.block + 1) if m > 0 else 0
        self._given(most, lambda: self.ctx.pages_resize(self.K, self.V, self.table, self.state, self.len, n_new, m, self.info, self.pages_ws))

    def free_pages(self):
        """How many pages are free (waits for the device)."""
        self.free = int((self.state[:self.n_pages] == 0).sum())
        return self.free

    def compact(self):
        """Moves the pages in use to the pool's front."""
        self.ctx.pages_compact(self.K, self.V, self.table, self.state, self.info, self.pages_ws)

    # -- tokens -----------------------------------------------------------------------------------
    def prefill(self, q, k, v, n_new=None):
        """As CacheRun.prefill: the next chunk of every sequence, q [n_inst][m][g][d], k and v [n_inst][m][d]; n_new: int32 [n_inst]."""
        m = q.shape[1]
        if m > self.q_cap:
            raise ValueError(f"a chunk has at most q_cap = {self.q_cap} tokens")
        if k.shape[:2] != q.shape[:2] or v.shape[:2] != q.shape[:2]:
            raise ValueError(f"{list(q.shape[:2])} queries and rows k, v of {list(k.shape[:2])}, {list(v.shape[:2])}")
        out = self.chunk_out.view(-1)[:q.numel()].view(q.shape)

        def calls():
            self._resize(n_new, m)
            self.ctx.cache_append(k, v, n_new, self.len, self.K, self.V)
            self.ctx.cache_prefill_shared(q, n_new, self.K, self.V, self.len, self.plan, self.window, self.n_first, out, self.ws)
        self._grown(m if n_new is None else n_new.clamp(0, m), m, calls)
        return out

    def step(self, q, k, v):
        """One decode step: q [n_inst][g][d], k and v [n_inst][d].  Returns the outputs, float [n_inst][g][d], a buffer that the next step uses
        again.  (Where some sequences rest: prefill, with chunks of one token and counts.)"""
        def calls():
            self._resize(None, 1)
            self.ctx.cache_append(k.unsqueeze(1), v.unsqueeze(1), None, self.len, self.K, self.V)
            self.ctx.cache_decode_shared(q, self.K, self.V, self.len, self.plan, self.window, self.n_first, self.out, self.ws)
        self._grown(1, 1, calls)
        return self.out

    # -- sequences --------------------------------------------------------------------------------
    def share(self, group, shared):
        """Says which instances have how many first rows in common, int32 [n_inst] each (group < 0: none).  A group has any number; it is kept
        under its lowest member's."""
        self._check_each(group, torch.int32)
        self._check_each(shared, torch.int32)
        ordered, at = torch.sort(group, stable=True)
        begins = torch.ones_like(ordered)
        begins[1:] = ordered[1:] != ordered[:-1]
        number = torch.empty_like(at).scatter_(0, at, begins.cumsum(0) - 1)
        self._regroup(number, group >= 0, shared)

    def _share(self, group, shared):
        """The same of groups that have their lowest members' numbers; the others, that follow from them, count on it."""
        self.ctx.cache_share(group, shared, self.plan)
        self.group.copy_(group)
        self.shared.copy_(shared)

    def _regroup(self, number, members, shared):
        """Groups by numbers in [0, 2 n_inst): they are numbered anew, by their lowest members, and who is left alone is alone."""
        n = self.w.n_inst
        each = torch.arange(n, device=self.dev)
        number = torch.where(members, number, 2 * n)
        low = torch.full((2 * n + 1,), n, device=self.dev).scatter_reduce_(0, number, each, "amin")[number]
        high = torch.full((2 * n + 1,), -1, device=self.dev).scatter_reduce_(0, number, each, "amax")[number]
        grouped = members & (low < high)
        self._share(torch.where(grouped, low, -1).int(), torch.where(grouped, shared, 0).int())

    def fork(self, parent):
        """Instance j goes on from parent[j], int32 [n_inst]; one outside [0, n_inst) ends.  Those that go on from members of a group are a group,
        and have in common what it had; those that go on from one instance alone have all its rows in common."""
        n = self.w.n_inst
        before = self.len.clone()
        self._given(n, lambda: self.ctx.pages_fork(self.K, self.V, self.table, self.state, parent, before, self.len, self.info, self.pages_ws))
        members = (parent >= 0) & (parent < n)
        p = parent.clamp(0, n - 1).long()
        number = torch.where(self.group[p] < 0, n + p, self.group[p].long())
        at = torch.where(members, number, 2 * n)
        first = torch.full((2 * n + 1,), n, device=self.dev).scatter_reduce_(0, at, p, "amin")[number]
        last = torch.full((2 * n + 1,), -1, device=self.dev).scatter_reduce_(0, at, p, "amax")[number]
        self._regroup(number, members, torch.where(first == last, before[p], self.shared[p]))

    def _shorter(self, length):
        before = self.len.clone()
        self.len.copy_(length)
        try:
            self._resize(self.none_new, 0)
        except Exception:
            self.len.copy_(before)
            raise

    def take_back(self, n):
        """The last n tokens of every cache, int32 [n_inst], are taken back (drafts that were not accepted)."""
        self._check_each(n, torch.int32)
        self._shorter((self.len - n.clamp(min=0)).clamp(min=0))
        self._share(self.group, torch.minimum(self.shared, self.len))

    def end(self, which):
        """Sequences that end, bool [n_inst]: their pages are free, unless others have them too."""
        self._check_each(which, torch.bool)
        self._shorter(torch.where(which, 0, self.len))
        self._without(which)

    def _check_each(self, x, dtype):
        if x.dtype is not dtype or x.shape != self.len.shape or x.device != self.len.device:
            raise ValueError(f"expected {dtype} {list(self.len.shape)} on {self.len.device}")

    def _check_instances(self, instances):
        if not instances or len(set(instances)) != len(instances) or not all(0 <= i < self.w.n_inst for i in instances):
            raise ValueError(f"expected different instances out of {self.w.n_inst}, not {instances}")

    def _which(self, instances):
        which = torch.zeros(self.w.n_inst, dtype=torch.bool)
        which[instances] = True
        return which.to(self.dev)

    def _without(self, which):
        """These leave their groups."""
        self._regroup(self.group.clamp(min=0).long(), (self.group >= 0) & ~which, self.shared)

    def _pages_of(self, instances, pages):
        return torch.cat([self.table[i, :m] for i, m in zip(instances, pages)])

    def set_aside(self, instances):
        """Moves the caches of a list of instances to pinned host memory, and ends them: returns what bring_back takes.  Waits for the device."""
        self._check_instances(instances)
        lens = self.len[instances].tolist()
        pages = [-(-x // self.w.block) for x in lens]
        away = {"len": lens}
        if sum(pages):
            shape = (sum(pages), self.w.block, self.w.head_dim)
            away["K"], away["V"] = (torch.empty(shape, dtype=self.K.dtype, pin_memory=True) for _ in "KV")
            self.ctx.pages_copy(self.K, self.V, self._pages_of(instances, pages), away["K"], away["V"], None)
            torch.cuda.current_stream(self.dev).synchronize()
        self.end(self._which(instances))
        return away

    def bring_back(self, away, instances):
        """The caches of set_aside go on as these instances, which are empty, each alone.  Waits for the device."""
        self._check_instances(instances)
        if len(instances) != len(away["len"]) or max(self.len[instances].tolist()) > 0:
            raise ValueError(f"{len(away['len'])} caches need as many empty instances, not {instances}")
        if max(away["len"]) > self.w.t_cap:
            raise ValueError(f"a cache of {max(away['len'])} rows has no room here (t_cap = {self.w.t_cap})")
        pages = [-(-x // self.w.block) for x in away["len"]]
        for name in "KV" if sum(pages) else "":
            if away[name].dtype is not self.K.dtype or away[name].shape != (sum(pages),) + self.K.shape[1:]:
                raise ValueError(f"{name}: {sum(pages)} pages as this pool's, not {away[name].dtype} {list(away[name].shape)}")
        before, longest = self.len.clone(), self.longest
        self.len[instances] = torch.tensor(away["len"], dtype=torch.int32, device=self.dev)
        self.longest = max(self.longest, max(away["len"]))
        try:
            self._given(sum(pages), lambda: self.ctx.pages_resize(self.K, self.V, self.table, self.state, self.len, self.none_new, 0, self.info, self.pages_ws))
            if sum(pages):
                self.ctx.pages_copy(away["K"], away["V"], None, self.K, self.V, self._pages_of(instances, pages))
                torch.cuda.current_stream(self.dev).synchronize()
        except Exception:
            self.len.copy_(before)
            self.longest = longest
            raise
        self._without(self._which(instances))
