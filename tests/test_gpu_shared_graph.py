"""Calls on pages and attention over beginnings in common, captured into a graph: a captured step follows lengths, tables, counts and groups on
the device, and every replay gives the bytes of the eager calls, with the program's own work in between; on a stream that is not the default
one; and two contexts at once."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _run(seed, dtype="bf16"):
    from paper_2502_04077_amd.runner import PagedRun
    from workloads import CONFIGS
    w = CONFIGS["cfg1"].with_(kv_heads=4, batch=8, t0=600, steps=40, n_sink=1, kv_dtype=dtype)
    run = PagedRun(w, 1400, "cuda:0", q_cap=6)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda:0").to(w.torch_dtype())  # noqa: E731
    n = w.n_inst
    # Every instance has a prompt of its own; then all of a sequence go on from a sequence's.
    run.len.copy_(200 + 7 * (torch.arange(n, device="cuda:0") % 13))
    run.longest = 300
    run.ctx.pages_resize(run.K, run.V, run.table, run.state, run.len, None, 0, run.info, run.pages_ws)
    run.K.copy_(draw(*run.K.shape))
    run.V.copy_(draw(*run.V.shape))
    return run, w, draw


def _step(run, parent, q, k, v, qc, kc, vc, n_new, n_back):
    """A fork, a decode step, drafts, drafts taken back, a compaction, as captured."""
    c = run.ctx
    before = run.len.clone()
    c.pages_fork(run.K, run.V, run.table, run.state, parent, before, run.len, run.info, run.pages_ws)
    # Groups of those that go on from one.
    run.group.copy_(parent)
    run.shared.copy_(run.len)
    c.cache_share(run.group, run.shared, run.plan)
    run.len += 1
    c.pages_resize(run.K, run.V, run.table, run.state, run.len, None, 1, run.info, run.pages_ws)
    c.cache_append(k, v, None, run.len, run.K, run.V)
    c.cache_decode_shared(q, run.K, run.V, run.len, run.plan, 0, 0, run.out, run.ws)
    run.len += n_new
    c.pages_resize(run.K, run.V, run.table, run.state, run.len, n_new, 6, run.info, run.pages_ws)
    c.cache_append(kc, vc, n_new, run.len, run.K, run.V)
    c.cache_prefill_shared(qc, n_new, run.K, run.V, run.len, run.plan, 100, 4, run.chunk_out, run.ws)
    run.len -= torch.minimum(n_back, n_new)
    c.pages_resize(run.K, run.V, run.table, run.state, run.len, run.none_new, 0, run.info, run.pages_ws)
    c.pages_compact(run.K, run.V, run.table, run.state, run.info, run.pages_ws)


def _state(run):
    return [run.table, run.state, run.len, run.info, run.K, run.V, run.out, run.chunk_out]


def _args(run, draw, seed):
    n, g, d, dev = run.w.n_inst, run.w.g, run.w.head_dim, "cuda:0"
    gen = torch.Generator().manual_seed(seed)
    num = lambda lo, hi: torch.randint(lo, hi, (n,), generator=gen, dtype=torch.int32).to(dev)  # noqa: E731
    return [num(0, n), draw(n, g, d), draw(n, 1, d), draw(n, 1, d), draw(n, 6, g, d), draw(n, 6, d), draw(n, 6, d), num(0, 7), num(0, 7)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replays_equal_eager_calls(dtype):
    eager, w, _ = _run(1, dtype)
    graph, _, draw = _run(1, dtype)
    args = _args(graph, draw, 0)
    args[0].copy_(torch.arange(w.n_inst, dtype=torch.int32))
    for run in (eager, graph):
        _step(run, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            _step(graph, *args)
    torch.cuda.synchronize()
    for i in range(5):
        for x, y in zip(args, _args(graph, draw, i + 1)):
            x.copy_(y)
        if i == 2:
            args[0].fill_(5)                               # all from one
        graph.ws.fill_(255)
        graph.pages_ws.fill_(255)
        graph.plan.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        _step(eager, *args)
        for a, b in zip(_state(graph), _state(eager)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        assert eager.info[0] > 0 and eager.len.min() > 0


def test_current_stream_is_used():
    a, _, draw = _run(2)
    b, _, _ = _run(2)
    args = [_args(a, draw, i) for i in range(3)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for x in args:
        _step(a, *x)
        with torch.cuda.stream(side):                      # (both at once, each with its own workspaces)
            _step(b, *x)
    torch.cuda.synchronize()
    for x, y in zip(_state(a), _state(b)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_one_workspace_for_two_graphs():
    """Two captured calls with one workspace and one plan, replayed in turn on one stream."""
    run, w, draw = _run(3)
    n = w.n_inst
    run.share(torch.arange(n, dtype=torch.int32, device="cuda:0") // 8, torch.full((n,), 0, dtype=torch.int32, device="cuda:0"))
    q, qc = draw(n, w.g, w.head_dim), draw(n, 6, w.g, w.head_dim)

    def decode():
        run.ctx.cache_decode_shared(q, run.K, run.V, run.len, run.plan, 0, 0, run.out, run.ws)

    def prefill():
        run.ctx.cache_prefill_shared(qc, None, run.K, run.V, run.len, run.plan, 0, 0, run.chunk_out, run.ws)
    graphs = []
    for f in (decode, prefill):
        f()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    for _ in range(4):
        q.copy_(draw(*q.shape))
        qc.copy_(draw(*qc.shape))
        for g in graphs:
            g.replay()
        got = run.out.clone(), run.chunk_out.clone()
        run.out.fill_(7)
        run.chunk_out.fill_(7)
        decode()
        prefill()
        assert torch.equal(got[0], run.out) and torch.equal(got[1], run.chunk_out)
        run.len += 3
        run.ctx.pages_resize(run.K, run.V, run.table, run.state, run.len, None, 0, run.info, run.pages_ws)
