"""Calls on caches with lengths of their own, captured into a graph: a captured step follows the lengths on the device, and every replay
gives the bytes of the eager calls, with the program's own work in between; and on a stream that is not the default one."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _run(seed):
    from paper_2502_04077_amd.runner import CacheRun
    from workloads import CONFIGS
    w = CONFIGS["cfg1"].with_(kv_heads=4, batch=2, t0=400, steps=40, budget_tokens=64, n_sink=1, n_local=1)
    run = CacheRun(w, "cuda:0", q_cap=96, evict_every=10 ** 9)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda:0").to(torch.bfloat16)  # noqa: E731
    return run, w, draw


def _step(run, q, k, v, qc, kc, vc, n_new):
    """A decode step, a chunk and an eviction, as captured: lengths go on by device work only."""
    run.len += 1
    run.ctx.cache_append(k, v, None, run.len, run.K, run.V)
    run.ctx.cache_decode(q, run.K, run.V, run.len, 0, 0, run.out, run.acc, run.ws)
    run.len += n_new
    run.ctx.cache_append(kc, vc, n_new, run.len, run.K, run.V)
    run.ctx.cache_prefill(qc, n_new, run.K, run.V, run.len, 100, 4, run.chunk_out, run.acc, run.ws)
    run.ctx.cache_evict(run.K, run.V, run.acc, run.len, 64, 16, 16, run.acc, run.len, run.kept)


def _state(run):
    return [run.out, run.chunk_out, run.acc, run.len, run.K, run.V, run.kept]


def test_replays_equal_eager_calls():
    eager, w, _ = _run(1)
    graph, _, draw = _run(1)
    n = w.n_inst
    q, k, v = draw(n, 4, 128), draw(n, 1, 128), draw(n, 1, 128)
    qc, kc, vc = draw(n, 96, 4, 128), draw(n, 96, 128), draw(n, 96, 128)
    n_new = torch.tensor([96, 1, 0, 50, 33, 64, 95, 2], dtype=torch.int32, device="cuda:0")
    for run in (eager, graph):
        _step(run, q, k, v, qc, kc, vc, n_new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            _step(graph, q, k, v, qc, kc, vc, n_new)
    torch.cuda.synchronize()
    for i in range(4):
        for x in (q, k, v, qc, kc, vc):
            x.copy_(draw(*x.shape))
        n_new.copy_((n_new * 7 + 13 * i) % 97)
        graph.ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        _step(eager, q, k, v, qc, kc, vc, n_new)
        for a, b in zip(_state(graph), _state(eager)):
            assert torch.equal(a, b), i


def test_current_stream_is_used():
    a, w, draw = _run(2)
    b, _, _ = _run(2)
    n = w.n_inst
    args = (draw(n, 4, 128), draw(n, 1, 128), draw(n, 1, 128), draw(n, 96, 4, 128), draw(n, 96, 128), draw(n, 96, 128),
            torch.full((n,), 90, dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        _step(a, *args)
        with torch.cuda.stream(side):
            _step(b, *args)
    torch.cuda.synchronize()
    for x, y in zip(_state(a), _state(b)):
        assert torch.equal(x, y)
