"""The bookkeeping of PagedRun on the CPU: calls on pages by their definition (page_reference.py), attention that does nothing."""
from types import SimpleNamespace

import pytest
import torch

import paper_2502_04077_amd.runner as runner
from page_reference import Pool
from workloads import CONFIGS

N, B, CAP = 6, 16, 208
I32 = torch.int32


class _Calls:
    """A context whose calls on pages are the definition's; `fail` names one that is refused."""

    def __init__(self, **cfg):
        assert cfg["n_inst"] == N and cfg["block"] == B and cfg["t_cap"] == CAP
        self.fail, self.plans = None, []

    def __getattr__(self, name):
        def f(*args):
            if name == self.fail:
                raise RuntimeError(name)
            return 64 if name.endswith("bytes") else None
        return f

    def pages_state_bytes(self, n_pages):
        return 4 * (n_pages + -(-n_pages // 1024))

    def _do(self, K, V, table, state, info, f):
        pool = Pool(table.tolist(), K.shape[0], B, K, V)
        said = f(pool)
        table.copy_(torch.tensor(pool.table, dtype=I32))
        state[:K.shape[0]] = torch.tensor(pool.refs, dtype=I32)
        K.copy_(pool.K)
        V.copy_(pool.V)
        info.copy_(torch.tensor(said, dtype=I32))

    def pages_count(self, table, n_pages, state):
        assert (table == -1).all()
        state.zero_()

    def pages_resize(self, K, V, table, state, length, n_new, q_cap, info, ws):
        if length.dtype is not I32 or (n_new is not None and n_new.dtype is not I32):
            raise ValueError("n_new")
        self._do(K, V, table, state, info, lambda p: p.resize(length.tolist(), None if n_new is None else n_new.tolist(), q_cap))

    def pages_fork(self, K, V, table, state, parent, length, len_out, info, ws):
        if parent.dtype is not I32:
            raise ValueError("parent")
        out = []

        def f(p):
            lens, said = p.fork(parent.tolist(), length.tolist())
            out.extend(lens)
            return said
        self._do(K, V, table, state, info, f)
        len_out.copy_(torch.tensor(out, dtype=I32))

    def cache_share(self, group, shared, plan):
        if group.dtype is not I32 or shared.dtype is not I32:
            raise ValueError("group")
        self.plans.append((group.tolist(), shared.tolist()))


@pytest.fixture
def run(monkeypatch):
    monkeypatch.setattr(runner, "Context", _Calls)
    w = CONFIGS["cfg1"].with_(kv_heads=2, batch=3, t0=150, steps=58, budget_tokens=96, n_sink=1, n_local=2, g=4)
    assert w.n_inst == N and w.t_cap == CAP
    return runner.PagedRun(w, 24, "cpu", q_cap=80)


def _i(v):
    return torch.tensor(v, dtype=I32)


def _rows(m=None):
    lead = (N,) if m is None else (N, m)
    bf = torch.bfloat16
    return torch.zeros(lead + (4, 128), dtype=bf), torch.zeros(lead + (128,), dtype=bf), torch.zeros(lead + (128,), dtype=bf)


def _state(run):
    return (run.len.tolist(), run.longest, run.table.tolist(), run.state.tolist(), run.group.tolist(), run.shared.tolist(), run.ctx.plans[-1])


def _whole(run):
    """What has to hold at all times."""
    assert run.ctx.plans[-1] == (run.group.tolist(), run.shared.tolist())
    assert run.free <= run.free_pages()
    for i, L in enumerate(run.len.tolist()):
        pages = run.table[i].tolist()
        assert all(p >= 0 for p in pages[:-(-L // B)])
        mates = [j for j in range(N) if run.group[j] == run.group[i] >= 0]
        if mates:
            assert run.group[i] == mates[0] and len(mates) > 1
            common = min(run.shared[j].item() for j in mates)
            assert common <= L and pages[:common // B] == run.table[mates[0], :common // B].tolist()


def test_groups_follow_forks(run):
    run.prefill(*_rows(80), _i([40, 10, 0, 0, 0, 0]))
    _whole(run)
    run.fork(_i([0, 1, 0, 0, 1, -1]))
    _whole(run)
    assert run.len.tolist() == [40, 10, 40, 40, 10, 0] and run.group.tolist() == [0, 1, 0, 0, 1, -1] and run.shared.tolist() == [40, 10, 40, 40, 10, 0]
    run.step(*_rows())
    run.fork(_i([2, 1, 0, 3, 9, 3]))                       # beams of one prompt go on, one ends and the other sample is alone
    _whole(run)
    assert run.len.tolist() == [41, 11, 41, 41, 0, 41] and run.group.tolist() == [0, -1, 0, 0, -1, 0] and run.shared.tolist() == [40, 0, 40, 40, 0, 40]
    run.fork(_i([3, 1, 3, 3, 1, 3]))                       # all from one: all its rows
    _whole(run)
    assert run.group.tolist() == [0, 1, 0, 0, 1, 0] and run.shared.tolist() == [41, 11, 41, 41, 11, 41]
    run.fork(torch.arange(N, dtype=I32))                   # each from itself: nothing changes
    _whole(run)
    assert run.group.tolist() == [0, 1, 0, 0, 1, 0] and run.shared.tolist() == [41, 11, 41, 41, 11, 41]
    run.fork(_i([1, 0, 3, 4, 4, 4]))
    _whole(run)
    assert run.len.tolist() == [11, 41, 41, 11, 11, 11] and run.group.tolist() == [0, 1, 1, 0, 0, 0]
    run.end(torch.tensor([True, True, False, False, False, True]))
    _whole(run)
    assert run.len.tolist() == [0, 0, 41, 11, 11, 0] and run.group.tolist() == [-1, -1, -1, 3, 3, -1]
    run.end(torch.ones(N, dtype=torch.bool))
    _whole(run)
    assert run.free_pages() == 24


# Numbers that groups are given: below the number of instances, up to twice as many, above, and the largest.
NUMBERS = [0, 3, N, N + 3, 2 * N - 1, 2 * N, 1000, 2 ** 31 - 1]


@pytest.mark.parametrize("number", NUMBERS)
def test_groups_of_any_number(run, number):
    """What a group is called does not matter: everything that follows is as for groups that are called by their lowest member."""
    other = (number + 1) % 2 ** 31
    run.prefill(*_rows(80), _i([40] * 6))
    run.share(_i([-1, number, number, other, -2 ** 31, other]), _i([40] * 6))
    assert run.group.tolist() == [-1, 1, 1, 3, -1, 3] and run.shared.tolist()[1:4] == [40] * 3
    run.fork(torch.arange(N, dtype=I32))                   # each from itself: nothing changes
    assert run.group.tolist() == [-1, 1, 1, 3, -1, 3] and run.shared.tolist() == [0, 40, 40, 40, 0, 40]
    run.take_back(_i([0, 0, 3, 0, 0, 0]))
    assert run.group.tolist() == [-1, 1, 1, 3, -1, 3] and run.shared.tolist() == [0, 40, 37, 40, 0, 40]
    run.end(torch.tensor([False, False, False, True, False, False]))
    assert run.group.tolist() == [-1, 1, 1, -1, -1, -1] and run.shared.tolist() == [0, 40, 37, 0, 0, 0]


@pytest.mark.parametrize("number", NUMBERS)
def test_children_of_one_that_stood_alone_are_nobody_elses(run, number):
    """Two instances of a group, and children of one that stands alone."""
    run.prefill(*_rows(80), _i([40] * 6))
    run.share(_i([number, number, -1, -1, -1, -1]), _i([16] * 6))
    run.fork(_i([0, 1, 3, 3, -1, -1]))
    assert run.group.tolist() == [0, 0, 2, 2, -1, -1] and run.shared.tolist() == [16, 16, 40, 40, 0, 0]


def test_a_group_of_one_number_stands_alone(run):
    run.prefill(*_rows(80), _i([40] * 6))
    run.share(_i([7, 8, 9, 10, 11, 12]), _i([16] * 6))
    run.fork(_i([0, 0, 2, 3, 4, 5]))
    assert run.group.tolist() == [0, 0, -1, -1, -1, -1] and run.shared.tolist() == [40, 40, 0, 0, 0, 0]


def test_tokens_are_taken_back(run):
    run.prefill(*_rows(80), _i([33, 0, 0, 0, 0, 20]))
    run.fork(_i([0, 0, 0, -1, -1, 5]))
    run.prefill(*_rows(5), _i([5, 3, 0, 0, 0, 5]))
    run.take_back(_i([2, 3, 4, 9, -7, 25]))
    _whole(run)
    assert run.len.tolist() == [36, 33, 29, 0, 0, 0] and run.shared.tolist()[:3] == [33, 33, 29]
    run.step(*_rows())
    _whole(run)
    assert run.len.tolist() == [37, 34, 30, 1, 1, 1]


def test_pages_that_lack_change_nothing(run):
    run.prefill(*_rows(80), _i([60] * 6))                  # 24 pages: all
    before = _state(run)
    run.free = 0
    with pytest.raises(MemoryError):
        run.prefill(*_rows(5), _i([5, 0, 0, 0, 0, 0]))
    assert _state(run) == before
    run.prefill(*_rows(4))                                 # (they have room)
    before = _state(run)
    for call in (lambda: run.step(*_rows()), lambda: run.prefill(*_rows(1), _i([0, 0, 0, 0, 0, 1]))):
        with pytest.raises(MemoryError):
            call()
        assert _state(run) == before
    run.take_back(_i([1] * 6))
    run.fork(_i([0, 2, 1, 3, 4, 5]))                       # heirs take last pages over
    run.end(torch.tensor([False] * 5 + [True]))
    assert run.free_pages() == 4
    before = _state(run)
    run.free = 0
    with pytest.raises(MemoryError):
        run.step(*_rows())                                 # room for 63 + 1, and instance 5 gets a page
        run.step(*_rows())
    assert run.len.tolist() == [64] * 5 + [1] and run.free_pages() == 3
    run.fork(_i([0, 1, 2, 3, 4, 4]))
    before = _state(run)
    run.free = 0
    with pytest.raises(MemoryError):
        run.step(*_rows())
    assert _state(run) == before and run.free_pages() == 4


@pytest.mark.parametrize("call", ["pages_resize", "cache_append", "cache_decode_shared", "cache_prefill_shared", "pages_fork"])
def test_a_call_that_is_refused_leaves_the_lengths(run, call):
    run.prefill(*_rows(20))
    before = run.len.tolist(), run.longest, run.group.tolist()
    if call in ("pages_resize", "pages_fork"):
        def refuse(*args):
            raise RuntimeError(call)
        setattr(run.ctx, call, refuse)
    run.ctx.fail = call
    with pytest.raises(RuntimeError, match=call):
        if call == "pages_fork":
            run.fork(_i([0] * 6))
        elif call == "cache_prefill_shared":
            run.prefill(*_rows(3), _i([3, 0, 1, 2, 3, 3]))
        else:
            run.step(*_rows())
    if call == "pages_resize":
        for f in (lambda: run.take_back(_i([3] * 6)), lambda: run.end(torch.ones(N, dtype=torch.bool))):
            with pytest.raises(RuntimeError):
                f()
    assert (run.len.tolist(), run.longest, run.group.tolist()) == before


REFUSED = {
    "chunk": lambda r: r.prefill(*_rows(81)),
    "rows": lambda r: r.prefill(_rows(7)[0], *_rows(5)[1:]),
    "counts": lambda r: r.prefill(*_rows(7), torch.full((N,), 7)),
    "taken back, 64 bits": lambda r: r.take_back(torch.ones(N, dtype=torch.int64)),
    "taken back, one": lambda r: r.take_back(torch.ones(1, dtype=I32)),
    "ends, numbers": lambda r: r.end(torch.ones(N, dtype=I32)),
    "parents, 64 bits": lambda r: r.fork(torch.zeros(N, dtype=torch.int64)),
    "groups, 64 bits": lambda r: r.share(torch.zeros(N, dtype=torch.int64), r.shared),
    "nobody aside": lambda r: r.set_aside([]),
    "one aside twice": lambda r: r.set_aside([1, 1]),
    "aside, no instance": lambda r: r.set_aside([-1]),
    "back, not empty": lambda r: r.bring_back({"len": [3]}, [0]),
    "back, too few": lambda r: r.bring_back({"len": [3, 3]}, [5]),
    "full": lambda r: (setattr(r, "longest", CAP), r.len.fill_(CAP), r.step(*_rows())),
}


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_refusals(run, name):
    run.prefill(*_rows(20), _i([20, 3, 1, 20, 20, 0]))
    before = _state(run)
    with pytest.raises((ValueError, RuntimeError)):
        REFUSED[name](run)
    if name != "full":
        assert _state(run) == before


def test_an_empty_cache_waits_and_comes_back(run):
    run.prefill(*_rows(20), _i([20, 3, 1, 20, 20, 0]))
    away = run.set_aside([5])
    run.bring_back(away, [5])
    assert away["len"] == [0] and run.len.tolist() == [20, 3, 1, 20, 20, 0]
    _whole(run)


def _away(lens, block=B, d=128, dtype=torch.bfloat16):
    """What set_aside of a run with such pages returns."""
    pages = sum(-(-x // block) for x in lens)
    return {"len": lens, "K": torch.ones((pages, block, d), dtype=dtype), "V": torch.ones((pages, block, d), dtype=dtype)}


@pytest.mark.parametrize("away,instances", [
    (_away([CAP + 1, 5]), [5, 4]),                         # longer than a cache here
    (_away([5, CAP + 1]), [4, 5]),
    (_away([40], block=8), [5]),
    (_away([40], d=64), [5]),
    (_away([40], dtype=torch.float32), [5]),
    ({**_away([40]), "len": [20]}, [5]),                   # fewer rows than pages
], ids=str)
def test_caches_of_another_kind_do_not_come_back(run, away, instances):
    run.prefill(*_rows(20), _i([20, 3, 1, 20, 0, 0]))
    before = _state(run)
    with pytest.raises(ValueError):
        run.bring_back(away, instances)
    assert _state(run) == before


def test_caches_come_back_alone(run, monkeypatch):
    """Also as an instance that was said to share a beginning while it was empty."""
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: SimpleNamespace(synchronize=lambda: None))
    run.prefill(*_rows(20), _i([20, 3, 0, 0, 0, 0]))
    away = _away([18, 5])
    run.share(_i([-1, -1, 9, 9, 9, 7]), _i([0, 0, 16, 16, 16, 16]))
    run.bring_back(away, [3, 5])
    assert run.len.tolist() == [20, 3, 0, 18, 0, 5]
    assert run.group.tolist() == [-1, -1, 2, -1, 2, -1] and run.shared.tolist() == [0, 0, 16, 0, 16, 0]
    assert run.ctx.plans[-1] == (run.group.tolist(), run.shared.tolist())
