"""Sizes at the limits of the calls on caches with lengths of their own: what the workspace is sized for is what the calls take.  No GPU."""
import ctypes as C

import pytest
import torch

import paper_2502_04077_amd as ap
from paper_2502_04077_amd.binding import ap_config

OK = 4096          # a fake, aligned, non-null address


@pytest.mark.parametrize("n_inst,g", [(1, 1), (8, 4), (64, 8), (2048, 2), (65535, 1)])
def test_no_workspace_for_chunks_that_are_refused(n_inst, g):
    """The longest chunk that a launch has room for, 2^32 threads and 2^30 rows, has a workspace, and a longer one neither that nor a call.
    (No call is made that is not refused: it would be launched.)"""
    lib = ap.load_library()
    cfg = ap_config(n_inst, g, 128, 16, 64, 4096, 64, 4, 4, 8, 8, ap.AP_BF16, 0)
    ctx = C.c_void_p()
    assert lib.ap_create(C.byref(cfg), C.byref(ctx)) == 0
    tiles = ((1 << 32) - 1) // (256 * n_inst)              # of 128 rows of q
    most = min(tiles * 128 // g, (1 << 30) // g)
    for weights in (0, 1):
        assert lib.ap_cache_workspace_bytes(ctx, most, weights) > 0
        assert lib.ap_cache_workspace_bytes(ctx, most + 1, weights) == 0
    for q_cap in (most + 1, 2 * most, (1 << 30) // g + 1, (1 << 31) - 1):
        assert lib.ap_cache_workspace_bytes(ctx, q_cap, 0) == 0
        assert lib.ap_cache_prefill(ctx, OK, OK, q_cap, OK, OK, OK, 0, 0, OK, OK, OK, None) == ap.AP_ERR_RANGE
    assert lib.ap_destroy(ctx) == 0


@pytest.mark.parametrize("shape,paged,good", [
    ((2, 64, 64), False, True), ((3, 64, 64), False, True), ((2, 4, 16, 64), False, True), ((5, 1, 4, 16, 64), False, True),
    ((128, 64), False, True), ((200, 64), False, True), ((1, 3, 64, 64), False, True), ((8, 16, 64), False, True),
    ((2, 80, 64), False, False), ((2, 96, 64), False, False), ((2, 128, 64), False, False), ((2, 5, 16, 64), False, False), ((9, 16, 64), False, False),
    ((12, 16, 64), True, True), ((20, 16, 64), True, True), ((192, 64), True, True), ((6, 32, 64), True, True), ((5, 64, 16, 64), True, True),
    ((7, 32, 64), True, False), ((24, 8, 64), True, True), ((30, 8, 64), True, False),
])
def test_caches_whose_rows_lie_elsewhere(shape, paged, good):
    """Two caches of 64 rows, or a pool of 12 pages of 16: more memory than that is taken if whole caches (pages) come out of it, not if its
    dimensions say that their rows lie elsewhere.  (Host tensors: the ones whose shape is right are refused for the device.)"""
    c = ap.Context(n_inst=2, g=4, head_dim=64, block=16, hist_len=1, t_cap=64, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    if paged:
        c._kv_numel, c._kv_unit = 12 * 16 * 64, 16 * 64                                # (as set_block_table leaves them)
    K = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one device" if good else "rows"):
        c._cache_kv(K, K.clone())
    c.close()


def test_the_table_says_what_a_page_is(monkeypatch):
    from paper_2502_04077_amd import binding
    monkeypatch.setattr(binding, "_ptr", lambda table: OK)
    c = ap.Context(n_inst=2, g=4, head_dim=64, block=16, hist_len=1, t_cap=64, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4, kv_dtype="bf16")
    assert (c._kv_numel, c._kv_unit) == (2 * 64 * 64, 64 * 64)
    c.set_block_table(torch.zeros(2, 4, dtype=torch.int32), 12)
    assert (c._kv_numel, c._kv_unit) == (12 * 16 * 64, 16 * 64)
    c.set_block_table(None)
    assert (c._kv_numel, c._kv_unit) == (2 * 64 * 64, 64 * 64)
    c.close()
