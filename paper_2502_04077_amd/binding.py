"""Thin ctypes binding of libattnpred.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in include/attnpred.h.
Tensors are torch CUDA(ROCm) tensors used purely as device memory; the current torch stream is
passed as the hipStream_t.  There is no CPU fallback: a missing library is an error.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libattnpred.so")

AP_F32, AP_BF16 = 0, 1
AP_PRED_REBASE, AP_PRED_ADVANCE, AP_PRED_HOLD, AP_PRED_SKIP = 0, 1, 2, 3
AP_STEP_REUSE_SELECTION = 16
AP_FLAG_PREDICTOR_FP32 = 1
AP_OK, AP_ERR_ARG, AP_ERR_ALIGN, AP_ERR_RANGE, AP_ERR_HIP, AP_ERR_UNSUPPORTED, AP_ERR_STATE = 0, -1, -2, -3, -4, -5, -6

EXPORTS = [
    "ap_create", "ap_destroy", "ap_workspace_bytes", "ap_hist_slots", "ap_nb_cap", "ap_set_weights", "ap_score_offset", "ap_set_block_table",
    "ap_predict", "ap_predict_incremental", "ap_select_topk", "ap_refresh_selection", "ap_sparse_decode", "ap_sparse_decode_noalloc", "ap_calibrate", "ap_update_history", "ap_step",
    "ap_prefetch_state_bytes", "ap_prefetch_blocks", "ap_append_kv", "ap_offload_begin", "ap_offload_step",
    "ap_cache_workspace_bytes", "ap_cache_append", "ap_cache_decode", "ap_cache_prefill", "ap_cache_evict",
    "ap_pages_state_bytes", "ap_pages_workspace_bytes", "ap_pages_count", "ap_pages_resize", "ap_pages_fork", "ap_pages_compact", "ap_pages_copy",
    "ap_cache_share_bytes", "ap_cache_share", "ap_cache_shared_workspace_bytes", "ap_cache_decode_shared", "ap_cache_prefill_shared", "ap_stream_read", "ap_stream_copy", "ap_strerror",
]


class ap_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_inst", "g", "head_dim", "block", "hist_len", "t_cap", "k_blocks", "n_sink", "n_local",
        "c1", "c2", "kv_dtype", "flags")]


class ApError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"attnpred error {code}: {what}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Loads the HIP library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2502_04077_amd.build` "
            "(or __graft_entry__.build()); this package has no other execution path")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.ap_create.argtypes = [C.POINTER(ap_config), C.POINTER(vp)]
    lib.ap_destroy.argtypes = [vp]
    lib.ap_workspace_bytes.argtypes = [vp]
    lib.ap_workspace_bytes.restype = sz
    lib.ap_hist_slots.argtypes = [vp]
    lib.ap_hist_slots.restype = i32
    lib.ap_nb_cap.argtypes = [vp]
    lib.ap_nb_cap.restype = i32
    lib.ap_set_weights.argtypes = [vp, vp, sz, vp]
    lib.ap_score_offset.argtypes = [vp]
    lib.ap_score_offset.restype = C.c_double
    lib.ap_set_block_table.argtypes = [vp, vp, i32]
    lib.ap_predict.argtypes = [vp, vp, i64, i32, vp, vp, vp]
    lib.ap_predict_incremental.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp, vp, vp]
    lib.ap_select_topk.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.ap_refresh_selection.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.ap_sparse_decode.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.ap_sparse_decode_noalloc.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.ap_calibrate.argtypes = [vp, vp, vp, i32, vp, vp, vp]
    lib.ap_update_history.argtypes = [vp, vp, i64, vp, vp]
    lib.ap_step.argtypes = [vp, vp, i64, vp, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.ap_prefetch_state_bytes.argtypes = [vp]
    lib.ap_prefetch_state_bytes.restype = sz
    lib.ap_prefetch_blocks.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.ap_append_kv.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.ap_offload_begin.argtypes = [vp, vp, i64, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ap_offload_step.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp,
                                    vp, vp, vp, vp]
    lib.ap_cache_workspace_bytes.argtypes = [vp, i32, i32]
    lib.ap_cache_workspace_bytes.restype = sz
    lib.ap_cache_append.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.ap_cache_decode.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.ap_cache_prefill.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.ap_cache_evict.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.ap_pages_state_bytes.argtypes = [vp, i32]
    lib.ap_pages_state_bytes.restype = sz
    lib.ap_pages_workspace_bytes.argtypes = [vp, i32]
    lib.ap_pages_workspace_bytes.restype = sz
    lib.ap_pages_count.argtypes = [vp, vp, i32, vp, vp]
    lib.ap_pages_resize.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp]
    lib.ap_pages_fork.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.ap_pages_compact.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.ap_pages_copy.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, vp, i32, vp]
    lib.ap_cache_share_bytes.argtypes = [vp]
    lib.ap_cache_share_bytes.restype = sz
    lib.ap_cache_share.argtypes = [vp, vp, vp, vp, vp]
    lib.ap_cache_shared_workspace_bytes.argtypes = [vp, i32]
    lib.ap_cache_shared_workspace_bytes.restype = sz
    lib.ap_cache_decode_shared.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.ap_cache_prefill_shared.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.ap_stream_read.argtypes = [vp, sz, vp, i32, vp]
    lib.ap_stream_copy.argtypes = [vp, sz, vp, i32, vp]
    lib.ap_strerror.argtypes = [C.c_int]
    lib.ap_strerror.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("ap_workspace_bytes", "ap_prefetch_state_bytes", "ap_hist_slots", "ap_nb_cap", "ap_strerror",
                        "ap_score_offset", "ap_cache_workspace_bytes", "ap_pages_state_bytes", "ap_pages_workspace_bytes", "ap_cache_share_bytes",
                        "ap_cache_shared_workspace_bytes"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != 0:
        raise ApError(rc, load_library().ap_strerror(rc).decode())


def _ptr(t: torch.Tensor) -> int:
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


def _rptr(t: torch.Tensor) -> int:
    """A tensor a kernel may read: device memory, or pinned (device-mapped) host memory."""
    if not (t.is_cuda or t.is_pinned()) or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor or pinned host tensor")
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# The current stream of a device as a hipStream_t, without the object around it (which costs as much as a launch).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def stream_read(src: torch.Tensor, sink: torch.Tensor, n_workgroups: int) -> None:
    _check(load_library().ap_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), n_workgroups,
                                         _stream()))


def stream_copy(src: torch.Tensor, dst: torch.Tensor, n_workgroups: int) -> None:
    _check(load_library().ap_stream_copy(_ptr(src), src.numel() * src.element_size(), _ptr(dst), n_workgroups,
                                         _stream()))


class Context:
    """Owns one ap_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, *, n_inst, g, head_dim, block, hist_len, t_cap, k_blocks, n_sink, n_local, c1, c2,
                 kv_dtype, flags=0):
        lib = load_library()
        self.cfg = ap_config(n_inst, g, head_dim, block, hist_len, t_cap, k_blocks, n_sink, n_local, c1, c2,
                             AP_BF16 if kv_dtype in ("bf16", AP_BF16) else AP_F32, flags)
        h = C.c_void_p()
        _check(lib.ap_create(C.byref(self.cfg), C.byref(h)))
        self._h = h
        self._lib = lib
        # what the cache_* calls check their tensors against on every call
        self._n, self._g, self._d, self._t_cap, self._b = n_inst, g, head_dim, t_cap, block
        self._dtype = torch.bfloat16 if self.cfg.kv_dtype == AP_BF16 else torch.float32
        self._kv_numel, self._kv_unit = n_inst * t_cap * head_dim, t_cap * head_dim      # of K; of a cache, or a page
        self._decode_ws = [self.cache_workspace_bytes(0, weights) for weights in (False, True)]
        self._shared_ws = (self.cache_share_bytes(), self.cache_shared_workspace_bytes(0))
        self._pages = (0, 0, 0)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.ap_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- sizes ------------------------------------------------------------------------------
    def workspace_bytes(self) -> int:
        return int(self._lib.ap_workspace_bytes(self._h))

    def hist_slots(self) -> int:
        return int(self._lib.ap_hist_slots(self._h))

    def nb_cap(self) -> int:
        return int(self._lib.ap_nb_cap(self._h))

    # -- calls ------------------------------------------------------------------------------
    def set_weights(self, blob: np.ndarray) -> None:
        blob = np.ascontiguousarray(blob, dtype=np.float32)
        _check(self._lib.ap_set_weights(self._h, blob.ctypes.data, blob.size, _stream()))

    def score_offset(self) -> float:
        """P0: pred holds the predictor's output minus this constant (see ap_predict in attnpred.h)."""
        return float(self._lib.ap_score_offset(self._h))

    def set_block_table(self, table, n_phys_blocks: int = 0) -> None:
        """table: device int32 [n_inst][nb_cap] (kept alive by the caller), or None for the contiguous layout."""
        _check(self._lib.ap_set_block_table(self._h, None if table is None else _ptr(table), n_phys_blocks))
        count, rows = (self._n, self._t_cap) if table is None else (n_phys_blocks, self.cfg.block)
        self._kv_numel, self._kv_unit = count * rows * self._d, rows * self._d

    def predict(self, hist, n_pushed, nb_cur, pred, ws) -> None:
        _check(self._lib.ap_predict(self._h, _ptr(hist), n_pushed, nb_cur, _ptr(pred), _ptr(ws), _stream()))

    def predict_incremental(self, hist, n_pushed, nb_cur, nb_prev, mode, pstate, pred, ws) -> None:
        _check(self._lib.ap_predict_incremental(self._h, _ptr(hist), n_pushed, nb_cur, nb_prev, mode, _ptr(pstate),
                                                _ptr(pred), _ptr(ws), _stream()))

    def select_topk(self, pred, nb_cur, idx, cnt, ws) -> None:
        _check(self._lib.ap_select_topk(self._h, _ptr(pred), nb_cur, _ptr(idx), _ptr(cnt), _ptr(ws), _stream()))

    def refresh_selection(self, nb_prev, nb_cur, idx, cnt) -> None:
        _check(self._lib.ap_refresh_selection(self._h, nb_prev, nb_cur, _ptr(idx), _ptr(cnt), _stream()))

    def sparse_decode(self, q, K, V, t_cur, idx, cnt, out, row, ws) -> None:
        _check(self._lib.ap_sparse_decode(self._h, _ptr(q), _ptr(K), _ptr(V), t_cur, _ptr(idx), _ptr(cnt),
                                          _ptr(out), _ptr(row), _ptr(ws), _stream()))

    def sparse_decode_noalloc(self, q, K, V, t_cur, idx, cnt, out, row) -> None:
        _check(self._lib.ap_sparse_decode_noalloc(self._h, _ptr(q), _ptr(K), _ptr(V), t_cur, _ptr(idx), _ptr(cnt),
                                                  _ptr(out), _ptr(row), _stream()))

    def calibrate(self, q, K, t_cur, row, ws) -> None:
        _check(self._lib.ap_calibrate(self._h, _ptr(q), _rptr(K), t_cur, _ptr(row), _ptr(ws), _stream()))

    def prefetch_state_bytes(self) -> int:
        return int(self._lib.ap_prefetch_state_bytes(self._h))

    def prefetch_blocks(self, K_src, V_src, t_avail, nb_cur, idx, cnt, pool_K, pool_V, table, state) -> None:
        _check(self._lib.ap_prefetch_blocks(self._h, _rptr(K_src), _rptr(V_src), t_avail, nb_cur, _ptr(idx), _ptr(cnt),
                                            _ptr(pool_K), _ptr(pool_V), _ptr(table), _ptr(state), _stream()))

    def offload_begin(self, hist, n_pushed, K_src, V_src, t_first, idx, cnt, pred, pstate, pool_K, pool_V, table, state,
                      ws, copy_stream) -> None:
        _check(self._lib.ap_offload_begin(self._h, _ptr(hist), n_pushed, _rptr(K_src), _rptr(V_src), t_first, _ptr(idx),
                                          _ptr(cnt), _ptr(pred), _ptr(pstate), _ptr(pool_K), _ptr(pool_V), _ptr(table),
                                          _ptr(state), _ptr(ws), _stream(), copy_stream.cuda_stream))

    def offload_step(self, hist, n_pushed, q, k_new, v_new, K_src, V_src, t_cur, calibrate, out, idx, cnt, pred, pstate,
                     pred_mode, pool_K, pool_V, table, state, row, ws, copy_stream) -> None:
        _check(self._lib.ap_offload_step(self._h, _ptr(hist), n_pushed, _ptr(q), _ptr(k_new), _ptr(v_new), _rptr(K_src),
                                         _rptr(V_src), t_cur, int(bool(calibrate)), _ptr(out), _ptr(idx), _ptr(cnt),
                                         _ptr(pred), _ptr(pstate), pred_mode, _ptr(pool_K), _ptr(pool_V), _ptr(table),
                                         _ptr(state), _ptr(row), _ptr(ws), _stream(), copy_stream.cuda_stream))

    def append_kv(self, k_new, v_new, t_pos, table, state, pool_K, pool_V) -> None:
        _check(self._lib.ap_append_kv(self._h, _ptr(k_new), _ptr(v_new), t_pos, _ptr(table), _ptr(state), _ptr(pool_K),
                                      _ptr(pool_V), _stream()))

    # -- caches whose instances have lengths of their own ---------------------------------------
    def cache_workspace_bytes(self, q_cap: int = 0, weights: bool = False) -> int:
        """Bytes of `ws` for cache_decode and cache_prefill of up to q_cap tokens; weights: with acc."""
        return int(self._lib.ap_cache_workspace_bytes(self._h, q_cap, int(bool(weights))))

    def _cache_kv(self, K, V) -> int:
        """Checks K and V; the index of the device they lie on."""
        dev = K.get_device()
        if K.shape != V.shape or K.shape[-1:] != (self._d,) or K.dtype is not self._dtype or V.dtype is not self._dtype:
            raise ValueError("K and V: two tensors [..., head_dim] of one shape, in the context's dtype")
        if K.numel() != self._kv_numel:
            self._cache_more(K)
        if dev < 0 or V.get_device() != dev or not (K.is_contiguous() and V.is_contiguous()):
            raise ValueError("K and V: expected contiguous tensors on one device")
        return dev

    def _cache_more(self, K) -> None:
        """Checks caches (pools) of another size than the context's: larger ones are taken by rows, or by whole caches (pages)."""
        if K.numel() < self._kv_numel:
            raise ValueError("K and V: fewer rows than the context's caches, or than the pages of its pool")
        one = 1
        for x in reversed(K.shape):
            one *= x
            if one >= self._kv_unit:
                break
        if one != self._kv_unit and K.dim() > 2:
            raise ValueError(f"K and V: caches (pages) of {self._kv_unit // self._d} rows do not come out of {list(K.shape)}")

    @staticmethod
    def _cache_arg(name, t, dtype, shape, dev) -> int:
        if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous {dtype} {list(shape)} on device {dev}, got {t.dtype} {list(t.shape)} on {t.device}")
        return t.data_ptr()

    @staticmethod
    def _buffer(name, t, need, dev) -> int:
        if t.get_device() != dev or not t.is_contiguous() or t.numel() * t.element_size() < need:
            raise ValueError(f"{name}: expected {need} bytes on device {dev}, contiguous")
        return t.data_ptr()

    @staticmethod
    def _cache_ws(ws, need, dev) -> int:
        return Context._buffer("ws", ws, need, dev)

    @staticmethod
    def _cache_call(dev, call, *args) -> None:
        """The call on the current stream of device `dev`, whichever device is current."""
        if dev == torch.cuda.current_device():
            rc = call(*args, _raw_stream(dev))
        else:
            with torch.cuda.device(dev):
                rc = call(*args, _raw_stream(dev))
        _check(rc)

    def cache_append(self, k_new, v_new, n_new, length, K, V) -> None:
        """k_new, v_new: [n_inst][q_cap][d]; n_new: int32 [n_inst] or None (q_cap each)."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        q_cap = k_new.shape[1] if k_new.dim() == 3 else 0
        new = (self._n, q_cap, self._d)
        self._cache_call(dev, self._lib.ap_cache_append, self._h, arg("k_new", k_new, self._dtype, new, dev),
                         arg("v_new", v_new, self._dtype, new, dev),
                         None if n_new is None else arg("n_new", n_new, torch.int32, (self._n,), dev), q_cap,
                         arg("length", length, torch.int32, (self._n,), dev), K.data_ptr(), V.data_ptr())

    def cache_decode(self, q, K, V, length, window, n_first, out, acc, ws) -> None:
        """q: [n_inst][g][d]; out: float [n_inst][g][d]; acc: float [n_inst][t_cap] or None."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        shape = (self._n, self._g, self._d)
        self._cache_call(dev, self._lib.ap_cache_decode, self._h, arg("q", q, self._dtype, shape, dev), K.data_ptr(), V.data_ptr(),
                         arg("length", length, torch.int32, (self._n,), dev), window, n_first,
                         arg("out", out, torch.float32, shape, dev),
                         None if acc is None else arg("acc", acc, torch.float32, (self._n, self._t_cap), dev),
                         self._cache_ws(ws, self._decode_ws[acc is not None], dev))

    def cache_prefill(self, q, n_q, K, V, length, window, n_first, out, acc, ws) -> None:
        """q: [n_inst][q_cap][g][d]; n_q: int32 [n_inst] or None (q_cap each); out: as q; acc: float [n_inst][t_cap] or None."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        q_cap = q.shape[1] if q.dim() == 4 else 0
        shape = (self._n, q_cap, self._g, self._d)
        self._cache_call(dev, self._lib.ap_cache_prefill, self._h, arg("q", q, self._dtype, shape, dev),
                         None if n_q is None else arg("n_q", n_q, torch.int32, (self._n,), dev), q_cap, K.data_ptr(), V.data_ptr(),
                         arg("length", length, torch.int32, (self._n,), dev), window, n_first,
                         arg("out", out, self._dtype, shape, dev),
                         None if acc is None else arg("acc", acc, torch.float32, (self._n, self._t_cap), dev),
                         self._cache_ws(ws, self.cache_workspace_bytes(q_cap, acc is not None), dev))

    def cache_evict(self, K, V, acc, length, budget, n_first, n_last, acc_out, len_out, kept) -> None:
        """acc_out may be acc, len_out may be length; kept: int32 [n_inst][budget]."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        rows = (self._n, self._t_cap)
        self._cache_call(dev, self._lib.ap_cache_evict, self._h, K.data_ptr(), V.data_ptr(), arg("acc", acc, torch.float32, rows, dev),
                         arg("length", length, torch.int32, (self._n,), dev), budget, n_first, n_last,
                         arg("acc_out", acc_out, torch.float32, rows, dev),
                         arg("len_out", len_out, torch.int32, (self._n,), dev),
                         arg("kept", kept, torch.int32, (self._n, budget), dev))

    # -- pages that instances share --------------------------------------------------------------
    def pages_state_bytes(self, n_pages: int) -> int:
        return int(self._lib.ap_pages_state_bytes(self._h, n_pages))

    def pages_workspace_bytes(self, n_pages: int) -> int:
        return int(self._lib.ap_pages_workspace_bytes(self._h, n_pages))

    def _pool(self, K, V):
        """Checks the pools K and V [n_pages][b][d]; the device they lie on, and their pages."""
        dev, shape = K.get_device(), K.shape
        if len(shape) != 3 or shape[1] != self._b or shape[2] != self._d or V.shape != shape or K.dtype is not self._dtype or V.dtype is not self._dtype:
            raise ValueError(f"K and V: two pools [n_pages][{self._b}][{self._d}] of one shape, in the context's dtype")
        if dev < 0 or V.get_device() != dev or not (K.is_contiguous() and V.is_contiguous()):
            raise ValueError("K and V: expected contiguous tensors on one device")
        return dev, shape[0]

    def _pages_state(self, table, state, n_pages, dev):
        nb = self._t_cap // self._b
        if self._pages[0] != n_pages:                             # (the sizes of a pool, asked once)
            self._pages = (n_pages, self.pages_state_bytes(n_pages) // 4, self.pages_workspace_bytes(n_pages))
        return self._cache_arg("table", table, torch.int32, (self._n, nb), dev), self._cache_arg("state", state, torch.int32, (self._pages[1],), dev)

    def pages_count(self, table, n_pages, state) -> None:
        """table: int32 [n_inst][nb_cap]; state: int32 of pages_state_bytes(n_pages)."""
        dev = table.get_device()
        if dev < 0:
            raise ValueError("table: expected a device tensor")
        table, state = self._pages_state(table, state, n_pages, dev)
        self._cache_call(dev, self._lib.ap_pages_count, self._h, table, n_pages, state)

    def pages_resize(self, K, V, table, state, length, n_new, q_cap, info, ws) -> None:
        """K, V: [n_pages][b][d]; length: int32 [n_inst], the new rows included; n_new: int32 [n_inst] or None (q_cap each); info: int32 [2]."""
        (dev, n_pages), arg = self._pool(K, V), self._cache_arg
        table, state = self._pages_state(table, state, n_pages, dev)
        self._cache_call(dev, self._lib.ap_pages_resize, self._h, K.data_ptr(), V.data_ptr(), table, n_pages, state,
                         arg("length", length, torch.int32, (self._n,), dev),
                         None if n_new is None else arg("n_new", n_new, torch.int32, (self._n,), dev), q_cap,
                         arg("info", info, torch.int32, (2,), dev), self._cache_ws(ws, self._pages[2], dev))

    def pages_fork(self, K, V, table, state, parent, length, len_out, info, ws) -> None:
        """parent: int32 [n_inst]; len_out: int32 [n_inst], may be length."""
        (dev, n_pages), arg = self._pool(K, V), self._cache_arg
        table, state = self._pages_state(table, state, n_pages, dev)
        self._cache_call(dev, self._lib.ap_pages_fork, self._h, K.data_ptr(), V.data_ptr(), table, n_pages, state,
                         arg("parent", parent, torch.int32, (self._n,), dev), arg("length", length, torch.int32, (self._n,), dev),
                         arg("len_out", len_out, torch.int32, (self._n,), dev), arg("info", info, torch.int32, (2,), dev),
                         self._cache_ws(ws, self._pages[2], dev))

    def pages_compact(self, K, V, table, state, info, ws) -> None:
        (dev, n_pages), arg = self._pool(K, V), self._cache_arg
        table, state = self._pages_state(table, state, n_pages, dev)
        self._cache_call(dev, self._lib.ap_pages_compact, self._h, K.data_ptr(), V.data_ptr(), table, n_pages, state,
                         arg("info", info, torch.int32, (2,), dev), self._cache_ws(ws, self._pages[2], dev))

    def pages_copy(self, K_src, V_src, src, K_dst, V_dst, dst, n=None) -> None:
        """Pools [..][b][d], on the device or in pinned host memory; src, dst: int32 [n] or None (0, 1, 2, ...; with both None, n says how many)."""
        dev = K_src.get_device()
        for t in (K_dst, src, dst):                           # (the first of them that lies on a device)
            if dev < 0 and t is not None:
                dev = t.get_device()
        if dev < 0:
            raise ValueError("pools: one of them at least lies on a device")
        n_src, n_dst = self._moved(K_src, V_src, dev), self._moved(K_dst, V_dst, dev)
        for x in (src, dst):
            if x is not None:
                if n is not None and x.numel() != n:
                    raise ValueError("src and dst: as many entries each, n")
                n = x.numel()
        if n is None:
            raise ValueError("n: where src and dst are None")
        if n < 0 or (src is None and n > n_src) or (dst is None and n > n_dst):
            raise ValueError(f"{n} pages are more than a pool has")
        arg = self._cache_arg
        self._cache_call(dev, self._lib.ap_pages_copy, self._h, K_src.data_ptr(), V_src.data_ptr(), n_src,
                         None if src is None else arg("src", src, torch.int32, (n,), dev), K_dst.data_ptr(), V_dst.data_ptr(), n_dst,
                         None if dst is None else arg("dst", dst, torch.int32, (n,), dev), n)

    def _moved(self, K, V, dev) -> int:
        """Checks the pools K and V of pages that are moved; their pages."""
        shape = K.shape
        if len(shape) != 3 or shape[1] != self._b or shape[2] != self._d or V.shape != shape or K.dtype is not self._dtype or V.dtype is not self._dtype:
            raise ValueError(f"K and V: pools [..][{self._b}][{self._d}] in the context's dtype")
        for t in (K, V):
            if not t.is_contiguous() or (t.get_device() != dev and (t.is_cuda or not t.is_pinned())):
                raise ValueError("pools: expected contiguous tensors on one device, or in pinned host memory")
        return shape[0]

    # -- attention of instances whose first rows are the same ------------------------------------
    def cache_share_bytes(self) -> int:
        """Bytes of `plan`."""
        return int(self._lib.ap_cache_share_bytes(self._h))

    def cache_share(self, group, shared, plan) -> None:
        """group, shared: int32 [n_inst]; plan: a device buffer of cache_share_bytes()."""
        dev, arg = group.get_device(), self._cache_arg
        if dev < 0:
            raise ValueError("group: expected a device tensor")
        self._cache_call(dev, self._lib.ap_cache_share, self._h, arg("group", group, torch.int32, (self._n,), dev),
                         arg("shared", shared, torch.int32, (self._n,), dev), self._buffer("plan", plan, self._shared_ws[0], dev))

    def cache_shared_workspace_bytes(self, q_cap: int = 0) -> int:
        """Bytes of `ws` for cache_decode_shared and cache_prefill_shared of up to q_cap tokens."""
        return int(self._lib.ap_cache_shared_workspace_bytes(self._h, q_cap))

    def cache_decode_shared(self, q, K, V, length, plan, window, n_first, out, ws) -> None:
        """As cache_decode; plan: of cache_share."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        shape = (self._n, self._g, self._d)
        self._cache_call(dev, self._lib.ap_cache_decode_shared, self._h, arg("q", q, self._dtype, shape, dev), K.data_ptr(), V.data_ptr(),
                         arg("length", length, torch.int32, (self._n,), dev), self._buffer("plan", plan, self._shared_ws[0], dev), window, n_first,
                         arg("out", out, torch.float32, shape, dev), self._cache_ws(ws, self._shared_ws[1], dev))

    def cache_prefill_shared(self, q, n_q, K, V, length, plan, window, n_first, out, ws) -> None:
        """As cache_prefill; plan: of cache_share."""
        dev, arg = self._cache_kv(K, V), self._cache_arg
        q_cap = q.shape[1] if q.dim() == 4 else 0
        shape = (self._n, q_cap, self._g, self._d)
        self._cache_call(dev, self._lib.ap_cache_prefill_shared, self._h, arg("q", q, self._dtype, shape, dev),
                         None if n_q is None else arg("n_q", n_q, torch.int32, (self._n,), dev), q_cap, K.data_ptr(), V.data_ptr(),
                         arg("length", length, torch.int32, (self._n,), dev), self._buffer("plan", plan, self._shared_ws[0], dev), window, n_first,
                         arg("out", out, self._dtype, shape, dev), self._cache_ws(ws, self.cache_shared_workspace_bytes(q_cap), dev))

    def update_history(self, hist, n_pushed, row) -> None:
        _check(self._lib.ap_update_history(self._h, _ptr(hist), n_pushed, _ptr(row), _stream()))

    def step(self, hist, n_pushed, q, K, V, t_cur, out, idx, cnt, pred, pstate, pred_mode, ws) -> None:
        _check(self._lib.ap_step(self._h, _ptr(hist), n_pushed, _ptr(q), _ptr(K), _ptr(V), t_cur, _ptr(out),
                                 _ptr(idx), _ptr(cnt), _ptr(pred), None if pstate is None else _ptr(pstate),
                                 pred_mode, _ptr(ws), _stream()))
