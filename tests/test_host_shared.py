"""Refusals of the calls on pages and on beginnings in common: all of them on the host, before anything is launched; no GPU needed."""
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
    "ap_pages_count": ([OK, 9, OK, None], set()),
    "ap_pages_resize": ([OK, OK, OK, 9, OK, OK, OK, 5, OK, OK, None], {6}),
    "ap_pages_fork": ([OK, OK, OK, 9, OK, OK, OK, OK, OK, OK, None], set()),
    "ap_pages_compact": ([OK, OK, OK, 9, OK, OK, OK, None], set()),
    "ap_pages_copy": ([OK, OK, 9, OK, OK, OK, 9, OK, 0, None], {3, 7}),
    "ap_cache_share": ([OK, OK, OK, None], set()),
    "ap_cache_decode_shared": ([OK, OK, OK, OK, OK, 0, 0, OK, OK, None], set()),
    "ap_cache_prefill_shared": ([OK, OK, 5, OK, OK, OK, OK, 0, 0, OK, OK, None], {1}),
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


POOLS = [("ap_pages_count", 1), ("ap_pages_resize", 3), ("ap_pages_fork", 3), ("ap_pages_compact", 3), ("ap_pages_copy", 2), ("ap_pages_copy", 6)]


@pytest.mark.parametrize("name,at,value,code", [(n, at, v, ap.AP_ERR_RANGE) for n, at in POOLS for v in (0, -1, (1 << 30) + 1, 2147483647, -2147483648)] + [
    ("ap_pages_resize", 7, -1, ap.AP_ERR_RANGE), ("ap_pages_copy", 8, -1, ap.AP_ERR_RANGE),
    ("ap_cache_decode_shared", 5, -1, ap.AP_ERR_ARG), ("ap_cache_decode_shared", 6, -1, ap.AP_ERR_ARG),
    ("ap_cache_prefill_shared", 7, -1, ap.AP_ERR_ARG), ("ap_cache_prefill_shared", 8, -1, ap.AP_ERR_ARG),
    ("ap_cache_prefill_shared", 2, 0, ap.AP_ERR_RANGE), ("ap_cache_prefill_shared", 2, -3, ap.AP_ERR_RANGE),
    ("ap_cache_prefill_shared", 2, 1 << 29, ap.AP_ERR_RANGE), ("ap_cache_prefill_shared", 2, 1 << 27, ap.AP_ERR_RANGE),
])
def test_sizes(ctx, name, at, value, code):
    args = list(CALLS[name][0])
    args[at] = value
    assert getattr(ap.load_library(), name)(ctx, *args) == code


def test_no_page_to_copy_is_no_call(ctx):
    assert ap.load_library().ap_pages_copy(ctx, *CALLS["ap_pages_copy"][0]) == ap.AP_OK


def test_pageable_memory_is_refused(ctx):
    mem = torch.zeros(9 * 16 * 128, dtype=torch.bfloat16)
    at = mem.data_ptr() + -mem.data_ptr() % 16
    args = list(CALLS["ap_pages_copy"][0])
    args[8] = 1
    for i in (0, 1, 4, 5):
        assert ap.load_library().ap_pages_copy(ctx, *args[:i], at, *args[i + 1:]) == ap.AP_ERR_ARG


def test_sizes_of_buffers(ctx):
    lib = ap.load_library()
    state, pages, plan, ws = lib.ap_pages_state_bytes, lib.ap_pages_workspace_bytes, lib.ap_cache_share_bytes, lib.ap_cache_shared_workspace_bytes
    for n in (1, 1023, 1024, 1025, 1 << 30):
        assert state(ctx, n) == 4 * (n + -(-n // 1024)) and pages(ctx, n) >= 4 * (3 * n + 8 * 256)
    for n in (0, -1, (1 << 30) + 1):
        assert state(ctx, n) == 0 == pages(ctx, n)
    assert plan(ctx) >= 8 * 40 and 0 < ws(ctx, 0) <= ws(ctx, 1) <= ws(ctx, 2) <= ws(ctx, 8) <= ws(ctx, 4096)
    assert ws(ctx, 4096) >= lib.ap_cache_workspace_bytes(ctx, 4096, 0)
    assert ws(ctx, -1) == 0 == ws(ctx, 1 << 30)
    assert state(None, 5) == pages(None, 5) == plan(None) == ws(None, 0) == 0


def test_binding_checks_types_shapes_and_devices():
    c = ap.Context(n_inst=2, g=4, head_dim=64, block=16, hist_len=1, t_cap=64, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    bf, i32 = torch.bfloat16, torch.int32
    K, V, L = torch.zeros(9, 16, 64, dtype=bf), torch.zeros(9, 16, 64, dtype=bf), torch.zeros(2, dtype=i32)
    table, state, info = torch.zeros(2, 4, dtype=i32), torch.zeros(10, dtype=i32), torch.zeros(2, dtype=i32)
    ws = torch.zeros(c.pages_workspace_bytes(9), dtype=torch.uint8)
    plan, shared_ws = torch.zeros(c.cache_share_bytes(), dtype=torch.uint8), torch.zeros(c.cache_shared_workspace_bytes(8), dtype=torch.uint8)
    q, out, chunk = torch.zeros(2, 4, 64, dtype=bf), torch.zeros(2, 4, 64), torch.zeros(2, 8, 4, 64, dtype=bf)

    class Meta:            # calls with tensors of the right shapes, on the host: what is refused is the device alone
        count = (c.pages_count, [table, 9, state])
        resize = (c.pages_resize, [K, V, table, state, L, L, 3, info, ws])
        fork = (c.pages_fork, [K, V, table, state, L, L, L, info, ws])
        compact = (c.pages_compact, [K, V, table, state, info, ws])
        copy = (c.pages_copy, [K, V, L, K.clone(), V.clone(), L])
        share = (c.cache_share, [L, L, plan])
        decode = (c.cache_decode_shared, [q, K, V, L, plan, 0, 0, out, shared_ws])
        prefill = (c.cache_prefill_shared, [chunk, L, K, V, L, plan, 0, 0, chunk, shared_ws])
    for f, args in (v for k, v in vars(Meta).items() if not k.startswith("_")):
        with pytest.raises(ValueError):
            f(*args)
    c.close()
