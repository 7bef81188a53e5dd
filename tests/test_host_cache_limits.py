"""Sizes at the limits of the calls on caches with lengths of their own: what the workspace is sized for is what the calls take.  No GPU."""
import ctypes as C

import pytest

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
