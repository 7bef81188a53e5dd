"""The predicted path (calibration, prediction, selection, attention over the selected blocks) over a table whose pages the page calls gave out, and which
sequences share: the same bytes as over contiguous caches."""
import pytest
import torch

from test_gpu_parity import _dev, _run, small
from workloads import kv_cache, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(t0=700), dict(t0=1500, g=1, kv_dtype="f32", head_dim=64)], ids=["bf16", "f32"])
def test_steps_over_pages_of_a_pool(kw):
    dev = _dev()
    w = small("pool", kv_heads=2, batch=3, hist_len=16, steps=20, calib_every=5, **kw)
    K, V = kv_cache(w, dev)
    n, H, d = w.n_inst, w.hist_len, w.head_dim
    S = w.t0 - H - 5                                       # the second and third sequence go on from the first
    for x in (K, V):
        x.view(w.batch, w.kv_heads, w.t_cap, d)[1:, :, :S] = x.view(w.batch, w.kv_heads, w.t_cap, d)[:1, :, :S]
    ref, pag = _run(w, dev), _run(w, dev)
    c, nb, n_pages = pag.ctx, w.t_cap // w.block, n * (w.t_cap // w.block) + 3
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    table = torch.full((n, nb), -1, dtype=torch.int32, device=dev)
    c.set_block_table(table, n_pages)
    Kp, Vp = (torch.zeros((n_pages, w.block, d), dtype=K.dtype, device=dev) for _ in range(2))
    state = torch.zeros(c.pages_state_bytes(n_pages) // 4, dtype=torch.int32, device=dev)
    ws, info = torch.zeros(c.pages_workspace_bytes(n_pages), dtype=torch.uint8, device=dev), i32([0, 0])
    c.pages_count(table, n_pages, state)
    first = [S if i < w.kv_heads else 0 for i in range(n)]
    length = i32(first)
    c.pages_resize(Kp, Vp, table, state, length, length, S, info, ws)
    c.cache_append(K[:, :S].contiguous(), V[:, :S].contiguous(), length.clone(), length, Kp, Vp)
    c.pages_fork(Kp, Vp, table, state, i32([i % w.kv_heads for i in range(n)]), length, length, info, ws)
    used = int((state[:n_pages] > 0).sum())
    assert length.tolist() == [S] * n and used == w.kv_heads * -(-S // w.block) + (n - w.kv_heads) * (S % w.block > 0)
    have = S

    def upto(t):
        nonlocal have
        m = t - have
        length.fill_(t)
        c.pages_resize(Kp, Vp, table, state, length, None, m, info, ws)
        c.cache_append(K[:, have:t].contiguous(), V[:, have:t].contiguous(), None, length, Kp, Vp)
        have = t
    for j in range(H):
        q, t = queries(w, j - H, dev), w.t0 - H + 1 + j
        upto(t)
        ref.warmup_calibrate(q, K, t)
        pag.warmup_calibrate(q, Kp, t)
    assert torch.equal(ref.hist, pag.hist)
    for s in range(w.steps):
        q, t, cal = queries(w, s, dev), w.t_at(s), w.is_calibration_step(s)
        upto(t)
        ref.step(q, K, V, t, calibrate=cal)
        pag.step(q, Kp, Vp, t, calibrate=cal)
        if s == 7:
            c.pages_compact(Kp, Vp, table, state, info, ws)
        assert torch.equal(ref.idx, pag.idx) and torch.equal(ref.out, pag.out) and torch.equal(ref.hist, pag.hist), s
    assert info[1] == 0 and int((state[:n_pages] > 1).sum()) == w.kv_heads * (S // w.block)
