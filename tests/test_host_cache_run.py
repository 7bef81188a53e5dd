"""The bookkeeping of CacheRun, which the host does before and behind the calls: on the CPU, where the calls refuse every tensor, or with
calls that do nothing in their place."""
import pytest
import torch

from paper_2502_04077_amd.runner import CacheRun
from workloads import CONFIGS


def _run():
    """6 caches of at most 208 rows, on the CPU."""
    w = CONFIGS["cfg1"].with_(kv_heads=2, batch=3, t0=150, steps=58, budget_tokens=96, n_sink=1, n_local=2, g=4)
    assert w.n_inst == 6 and w.t_cap == 208
    return CacheRun(w, "cpu", q_cap=80, evict_every=16)


def _rows(m=None):
    lead = (6,) if m is None else (6, m)
    bf = torch.bfloat16
    return torch.zeros(lead + (4, 128), dtype=bf), torch.zeros(lead + (128,), dtype=bf), torch.zeros(lead + (128,), dtype=bf)


def _state(run):
    return run.len.tolist(), run.longest, run.steps_done


class _Nothing:
    """Calls that do nothing."""
    def __getattr__(self, name):
        return lambda *args: None


I32 = torch.int32
REFUSED = {   # name -> call that the library or torch refuses
    "step on the host": lambda run: run.step(*_rows()),
    "step, rows of another type": lambda run: run.step(_rows()[0], _rows()[1].float(), _rows()[2].float()),
    "prefill on the host": lambda run: run.prefill(*_rows(7)),
    "counts in 64 bits": lambda run: run.prefill(*_rows(7), torch.full((6,), 7)),
    "counts that are no whole numbers": lambda run: run.prefill(*_rows(7), torch.full((6,), 7.0)),
    "too few counts": lambda run: run.prefill(*_rows(7), torch.ones(5, dtype=I32)),
    "one count": lambda run: run.prefill(*_rows(7), torch.ones(1, dtype=I32)),
    "queries of more heads": lambda run: run.prefill(torch.zeros(6, 80, 5, 128, dtype=torch.bfloat16), *_rows(80)[1:], torch.ones(6, dtype=I32)),
    "fewer rows than queries": lambda run: run.prefill(_rows(7)[0], *_rows(5)[1:]),
    "more rows than queries": lambda run: run.prefill(_rows(5)[0], *_rows(7)[1:], torch.full((6,), 5, dtype=I32)),
    "a longer chunk than q_cap": lambda run: run.prefill(*_rows(81)),
}


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_a_refused_call_leaves_the_lengths(name):
    run = _run()
    run.len += torch.tensor([3, 0, 17, 90, 90, 1], dtype=I32)
    run.longest = 90
    before, kept = _state(run), run.len
    if "fewer" in name or "more rows" in name:
        run.ctx = _Nothing()                               # (what the run has to see by itself)
    with pytest.raises((ValueError, RuntimeError)):
        REFUSED[name](run)
    assert _state(run) == before and run.len is kept


@pytest.mark.parametrize("call", ["cache_append", "cache_decode", "cache_prefill"])
def test_a_call_that_fails_behind_others_leaves_the_lengths(call):
    run, done = _run(), []

    class Calls:
        def __getattr__(self, name):
            def f(*args):
                done.append(name)
                if name == call:
                    raise RuntimeError(name)
            return f
    run.ctx = Calls()
    before = _state(run)
    with pytest.raises(RuntimeError, match=call):
        if call == "cache_prefill":
            run.prefill(*_rows(9), torch.tensor([9, 0, 1, 2, 3, 4], dtype=I32))
        else:
            run.step(*_rows())
    assert done[-1] == call and _state(run) == before


def test_ragged_chunks_go_in_while_there_is_room():
    """Chunks of 80 of which few tokens count: no cache is anywhere near its 208 rows, whatever the chunks' sum."""
    run = _run()
    run.ctx = _Nothing()
    new = torch.tensor([16, 0, 3, 1, 16, 9], dtype=I32)
    for i in range(13):
        run.prefill(*_rows(80), new)
        assert run.len.tolist() == ((i + 1) * new).tolist() and run.longest >= 16 * (i + 1)
    assert run.len.max() == 208 == run.longest
    before = _state(run)
    with pytest.raises(ValueError):
        run.prefill(*_rows(80), new)                       # two caches are full
    with pytest.raises(ValueError):
        run.step(*_rows())
    assert _state(run) == before
    run.prefill(*_rows(80), torch.tensor([0, 80, 80, 80, -5, 91], dtype=I32))
    assert run.len.tolist() == [208, 80, 39 + 80, 13 + 80, 208, 117 + 80] and run.longest == 208


def test_steps_go_on_behind_a_ragged_chunk():
    run = _run()
    run.ctx = _Nothing()
    run.evict_every = 10 ** 9
    for new in (1, 2):
        run.prefill(*_rows(80), torch.full((6,), new, dtype=I32))
    for _ in range(205):
        run.step(*_rows())
    assert run.len.tolist() == [208] * 6 and run.longest == 208
    with pytest.raises(ValueError):
        run.step(*_rows())
    assert run.len.tolist() == [208] * 6
