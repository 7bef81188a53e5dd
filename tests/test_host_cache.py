"""Refusals of the calls on caches with lengths of their own: all of them on the host, before anything is launched; no GPU needed."""
import ctypes as C

import pytest
import torch

import paper_2502_04077_amd as ap
from paper_2502_04077_amd.binding import ap_config

OK = 4096          # a fake, aligned, non-null address


@pytest.fixture
def ctx():
    lib = ap.load_library()
    cfg = ap_config(8, 4, 128, 16, 64, 4096, 64, 4, 4, 8, 8, ap.AP_BF16, 0)
    h = C.c_void_p()
    assert lib.ap_create(C.byref(cfg), C.byref(h)) == 0
    yield h
    assert lib.ap_destroy(h) == 0


CALLS = {   # name -> (arguments behind the context, places of pointers that may be null)
    "ap_cache_append": ([OK, OK, OK, 5, OK, OK, OK, None], {2}),
    "ap_cache_decode": ([OK, OK, OK, OK, 0, 0, OK, OK, OK, None], {7}),
    "ap_cache_prefill": ([OK, OK, 5, OK, OK, OK, 0, 0, OK, OK, OK, None], {1, 9}),
    "ap_cache_evict": ([OK, OK, OK, OK, 100, 4, 4, OK, OK, OK, None], set()),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_misaligned_pointers(ctx, name):
    args, optional = CALLS[name]
    call = getattr(ap.load_library(), name)
    assert call(None, *args) == ap.AP_ERR_ARG
    for i, x in enumerate(args[:-1]):
        if x != OK:
            continue
        if i not in optional:
            assert call(ctx, *args[:i], None, *args[i + 1:]) == ap.AP_ERR_ARG, i
        assert call(ctx, *args[:i], OK + 4, *args[i + 1:]) == ap.AP_ERR_ALIGN, i


@pytest.mark.parametrize("name,at,value,code", [
    ("ap_cache_append", 3, 0, ap.AP_ERR_RANGE), ("ap_cache_append", 3, -1, ap.AP_ERR_RANGE), ("ap_cache_append", 3, 1 << 30, ap.AP_ERR_RANGE), ("ap_cache_append", 3, 1 << 25, ap.AP_ERR_RANGE),
    ("ap_cache_decode", 4, -1, ap.AP_ERR_ARG), ("ap_cache_decode", 5, -1, ap.AP_ERR_ARG),
    ("ap_cache_prefill", 2, 0, ap.AP_ERR_RANGE), ("ap_cache_prefill", 2, 1 << 29, ap.AP_ERR_RANGE), ("ap_cache_prefill", 2, 1 << 27, ap.AP_ERR_RANGE),
    ("ap_cache_prefill", 6, -1, ap.AP_ERR_ARG), ("ap_cache_prefill", 7, -1, ap.AP_ERR_ARG),
    ("ap_cache_evict", 4, 0, ap.AP_ERR_ARG), ("ap_cache_evict", 4, 7, ap.AP_ERR_ARG), ("ap_cache_evict", 4, 4097, ap.AP_ERR_RANGE),
    ("ap_cache_evict", 5, -1, ap.AP_ERR_ARG), ("ap_cache_evict", 6, -1, ap.AP_ERR_ARG), ("ap_cache_evict", 6, 97, ap.AP_ERR_ARG),
    ("ap_cache_evict", 5, 2147483647, ap.AP_ERR_ARG), ("ap_cache_evict", 6, 2147483647, ap.AP_ERR_ARG),
])
def test_sizes(ctx, name, at, value, code):
    args = list(CALLS[name][0])
    args[at] = value
    assert getattr(ap.load_library(), name)(ctx, *args) == code


def test_workspace(ctx):
    lib = ap.load_library()
    size = lib.ap_cache_workspace_bytes
    decode, both = size(ctx, 0, 0), size(ctx, 0, 1)
    assert 0 < decode < both and decode % 16 == 0 and both >= decode + 8 * 4 * 4096 * 4
    assert size(ctx, 4096, 0) >= decode and size(ctx, 4096, 1) >= 8 * 4096 * 4 * 8
    assert size(None, 0, 0) == 0 and size(ctx, -1, 0) == 0 and size(ctx, 1 << 30, 0) == 0


def test_binding_checks_types_shapes_and_devices():
    c = ap.Context(n_inst=2, g=4, head_dim=64, block=16, hist_len=1, t_cap=64, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    bf, i32 = torch.bfloat16, torch.int32
    K, V, L = torch.zeros(2, 64, 64, dtype=bf), torch.zeros(2, 64, 64, dtype=bf), torch.zeros(2, dtype=i32)
    q, out, acc = torch.zeros(2, 4, 64, dtype=bf), torch.zeros(2, 4, 64), torch.zeros(2, 64)
    ws = torch.zeros(c.cache_workspace_bytes(8, True), dtype=torch.uint8)

    def refused(f, *args):
        with pytest.raises(ValueError):
            f(*args)

    refused(c.cache_decode, q, K, V, L, 0, 0, out, acc, ws)                       # host tensors
    refused(c.cache_decode, q.float(), K, V, L, 0, 0, out, acc, ws)
    refused(c.cache_decode, q, K.float(), V.float(), L, 0, 0, out, acc, ws)
    refused(c.cache_decode, q, K, V[:1], L, 0, 0, out, acc, ws)
    refused(c.cache_decode, q, K[:1], V[:1], L, 0, 0, out, acc, ws)               # fewer rows than the caches have
    refused(c.cache_decode, q, K, V, L.long(), 0, 0, out, acc, ws)
    refused(c.cache_decode, q, K, V, L[:1], 0, 0, out, acc, ws)
    refused(c.cache_decode, q, K, V, L, 0, 0, out.to(bf), acc, ws)
    refused(c.cache_decode, q, K, V, L, 0, 0, out, acc[:, :32], ws)
    refused(c.cache_decode, q, K, V, L, 0, 0, out, acc, ws[:64])
    new = torch.zeros(2, 3, 64, dtype=bf)
    refused(c.cache_append, new[:, 0], new[:, 0], None, L, K, V)
    refused(c.cache_append, new, new[:, :2], None, L, K, V)
    refused(c.cache_append, new, new, L[:1], L, K, V)
    chunk = torch.zeros(2, 8, 4, 64, dtype=bf)
    refused(c.cache_prefill, q, None, K, V, L, 0, 0, chunk, None, ws)
    refused(c.cache_prefill, chunk, None, K, V, L, 0, 0, chunk.float(), None, ws)
    refused(c.cache_prefill, chunk, L.float(), K, V, L, 0, 0, chunk, None, ws)
    refused(c.cache_evict, K, V, acc, L, 8, 1, 1, acc, L, torch.zeros(2, 7, dtype=i32))
    refused(c.cache_evict, K, V, acc.double(), L, 8, 1, 1, acc, L, torch.zeros(2, 8, dtype=i32))
    c.close()


def test_run_refuses_what_does_not_fit():
    from paper_2502_04077_amd.runner import CacheRun
    run = CacheRun.__new__(CacheRun)
    run.w, run.longest, run.len, run.q_cap = type("W", (), {"t_cap": 10})(), 8, torch.zeros(2, dtype=torch.int32), 4
    run._grow(1, 1)
    assert run.longest == 9 and run.len.tolist() == [1, 1]
    with pytest.raises(ValueError):
        run._grow(2, 2)
    assert run.longest == 9 and run.len.tolist() == [1, 1]
    with pytest.raises(ValueError):
        run.prefill(torch.zeros(2, 5, 1, 64), None, None)
