"""ctypes binding of ``libsam_b200.so``: argument marshalling only.

Function names and argument order follow ``include/sam.h``.  Device arguments are torch
tensors (or raw integer addresses); host arguments are numpy arrays.  Every step of the
path runs in the library's kernels - nothing is computed here.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from pathlib import Path
from typing import Optional

import numpy as np

_PKG = Path(__file__).resolve().parent
_LIB_PATH = _PKG / "libsam_b200.so"
_lib = None

SAM_K_MAX = 32
SAM_MAX_SEPARATORS = 16
SAM_STATIC_MAX_ROWS = 16384
SAM_MAX_BIAS = 512

_vp, _i32, _i64 = C.c_void_p, C.c_int32, C.c_int64

_SIGNATURES = {
    "sam_build": (C.c_int, [_vp, _i64, _vp, _i32, C.POINTER(_vp)]),
    "sam_sizes": (C.c_int, [_vp, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_i64)]),
    "sam_export": (C.c_int, [_vp] * 7),
    "sam_upload": (C.c_int, [_vp, _vp, _i64, _vp]),
    "sam_free": (None, [_vp]),
    "sam_workspace_bytes": (_i64, [_i32, _i32]),
    "sam_workspace_init": (C.c_int, [_vp, _i64, _vp]),
    "sam_draft": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _i32, _i32, _vp, _vp, _vp]),
    "sam_verify": (C.c_int, [_vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "sam_step": (C.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                           _vp, _vp, _i32, _vp, _vp, _vp, _i64, _vp]),
    "sam_verify_ex": (C.c_int, [_vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, C.c_uint32, _vp, _vp, _i64, _vp]),
    "sam_step_ex": (C.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                              _vp, _vp, _i32, _vp, _vp, C.c_uint32, _vp, _vp, _i64, _vp]),
    "sam_adaptive_switch": (C.c_int, [_i64, _i64, _i64, _i64]),
    "sam_speculation_pays": (C.c_int, [_vp, _i32, C.c_double]),
    "sam_set_bytes": (_i64, [_i32]),
    "sam_set_create": (C.c_int, [_vp, _i32, _vp, _i64, _vp, C.POINTER(_vp)]),
    "sam_set_refresh": (C.c_int, [_vp, _vp]),
    "sam_set_free": (None, [_vp]),
    "sam_set_renormalize": (C.c_int, [_vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "sam_multi_workspace_bytes": (_i64, [_i32, _i32, _i32]),
    "sam_multi_step": (C.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp,
                                 _i32, _vp, _vp, _vp, _vp, _i64, _vp]),
    "sam_multi_draft": (C.c_int, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _i32, _vp, _vp, _vp, _vp]),
    "sam_argmax_partial": (C.c_int, [_vp, _i64, _i64, _i32, _i32, _vp, _vp]),
    "sam_step_from_keys": (C.c_int, [_vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp]),
    "sam_verify_static": (C.c_int, [_vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sam_static_status": (C.c_int, [C.POINTER(_i32), _vp]),
    "sam_step_host_staging_bytes": (_i64, [_i64, _i32, _i32, _i32]),
    "sam_step_host": (C.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                _vp, _vp, _i32, _vp, _vp, _vp, _i64, _vp]),
    "sam_step_host_ex": (C.c_int, [_vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
                                   _vp, _vp, _i32, _vp, _vp, C.c_uint32, _vp, _i64, _vp]),
    "sam_workspace_status": (C.c_int, [_vp, _i32, _i32, C.POINTER(_i32), _vp]),
    "sam_set_argmax_variant": (C.c_int, [_i32]),
    "sam_profile_enable": (C.c_int, [_i32]),
    "sam_profile_count": (_i32, []),
    "sam_profile_read": (C.c_int, [_i32, C.POINTER(C.c_float), C.POINTER(C.c_float)]),
    "sam_strerror": (C.c_char_p, [C.c_int]),
    "sam_last_cuda_error": (C.c_int, []),
    "sam_launch_count": (_i64, []),
    "sam_build_growing": (C.c_int, [_vp, _i64, _vp, _i32, _i64, _i32, C.POINTER(_vp)]),
    "sam_extend": (C.c_int, [_vp, _vp, _i64]),
    "sam_extend_async": (C.c_int, [_vp, _vp, _i64]),
    "sam_pending": (C.c_int, [_vp, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_i64)]),
    "sam_sync": (C.c_int, [_vp, _vp, C.POINTER(_i64)]),
    "sam_renormalize": (C.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "sam_sync_renormalize": (C.c_int, [_vp, _i32, _vp, _vp, _vp, C.POINTER(_i64)]),
    "sam_growing_set_relayout_every": (C.c_int, [_vp, _i64]),
    "sam_update_stats": (C.c_int, [_vp, C.POINTER(_i64), C.POINTER(_i64), C.POINTER(_i64)]),
    "sam_cache_page_bytes": (_i64, [_i32, _i32, _i32, _i32]),
    "sam_cache_scratch_bytes": (_i64, [_i32, _i32]),
    "sam_cache_init": (C.c_int, [_vp, _vp]),
    "sam_cache_status": (C.c_int, [_vp, C.POINTER(_i32), C.POINTER(_i32), _vp]),
    "sam_cache_reserve": (C.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "sam_cache_commit": (C.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "sam_cache_fork": (C.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "sam_cache_compact": (C.c_int, [_vp, _vp]),
    "sam_cache_copy_pages": (C.c_int, [_vp, _vp, _i32, _vp, _vp, _vp]),
    "sam_cache_append": (C.c_int, [_vp, _i32, _vp, _vp, _i32, _i64, _i64, _i64, _i32, _i32, _vp, _vp, _vp]),
    "sam_cache_read": (C.c_int, [_vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp]),
    "sam_cache_attend_workspace_bytes": (_i64, [_vp, _i32, _i32, _i32]),
    "sam_cache_attend": (C.c_int, [_vp, _i32, _vp, _i32, _i64, _i64, _i64, _i32, _i32, _i32, _vp, _vp, C.c_float, _i32,
                                   _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp]),
    "sam_rope_turns": (C.c_int, [_vp, _i32, _vp]),
    "sam_cache_append_rotated": (C.c_int, [_vp, _i32, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _vp, _i64, _i64,
                                           _i64, _i32, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp]),
    "sam_cache_bounds_update": (C.c_int, [_vp, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp]),
    "sam_cache_bounds_rebuild": (C.c_int, [_vp, _vp, _vp, _i32, _vp, _vp]),
    "sam_cache_select_workspace_bytes": (_i64, [_vp, _i32, _i32, _i32]),
    "sam_cache_select": (C.c_int, [_vp, _i32, _vp, _vp, _vp, _i32, _i64, _i64, _i64, _i32, _i32, _i32, _vp, _vp, _i32, _i32,
                                   _i32, _vp, _i32, _vp, _i64, _vp]),
    "sam_cache_attend_blocks_workspace_bytes": (_i64, [_vp, _i32, _i32, _i32, _i32]),
    "sam_cache_attend_blocks": (C.c_int, [_vp, _i32, _vp, _i32, _i64, _i64, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _i32,
                                          _i32, C.c_float, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp]),
    "sam_argmax_shaped": (C.c_int, [_vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "sam_verify_from_keys": (C.c_int, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sam_history_add": (C.c_int, [_vp, _vp, _i32, _i32, _i32, _vp, _vp, _i32, _vp, _i32, _vp]),
    "sam_history_copy": (C.c_int, [_vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp]),
}


class SamError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = sam_strerror(status)
        if status == -4:
            msg += f" (cudaError {sam_last_cuda_error()})"
        super().__init__(f"{where}: {msg} [{status}]")


def library_path() -> Path:
    return _LIB_PATH


def use_library(path) -> None:
    """Points the binding at another build of this same library (a tuning run comparing two builds, a test
    of the missing-library error).  Only before the first call has loaded the default one."""
    global _LIB_PATH
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _LIB_PATH = Path(path)


def exported_symbols():
    """Names every build of the library must export (those declared in include/sam.h)."""
    return list(_SIGNATURES)


def _load():
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2512_18337_b200.build` "
                "(there is no CPU fallback)")
        lib = C.CDLL(str(_LIB_PATH))
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _dev(t) -> Optional[int]:
    """Device address of a torch tensor (must be contiguous, on CUDA) or a raw int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _host(a: Optional[np.ndarray], dtype) -> Optional[int]:
    if a is None:
        return None
    if a.dtype != dtype or not a.flags.c_contiguous:
        raise ValueError(f"expected a contiguous {np.dtype(dtype).name} array")
    return a.ctypes.data


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _check(status: int, where: str) -> None:
    if status != 0:
        raise SamError(status, where)


# ------------------------------------------------------------------ setup
def sam_build(corpus: np.ndarray, separators) -> int:
    """Host build; returns the opaque handle (release with sam_free)."""
    corpus = np.ascontiguousarray(corpus, dtype=np.int32)
    seps = np.ascontiguousarray(np.atleast_1d(separators), dtype=np.int32)
    h = _vp()
    _check(_load().sam_build(corpus.ctypes.data, corpus.shape[0], seps.ctypes.data if seps.size else None,
                             seps.shape[0], C.byref(h)), "sam_build")
    return h.value


def sam_build_growing(corpus: np.ndarray, separators, max_tokens: int, max_token_id: int) -> int:
    """Host build of an index that can grow (sam_extend); returns the opaque handle."""
    corpus = np.ascontiguousarray(corpus, dtype=np.int32)
    seps = np.ascontiguousarray(np.atleast_1d(separators), dtype=np.int32)
    h = _vp()
    _check(_load().sam_build_growing(corpus.ctypes.data if corpus.size else None, corpus.shape[0],
                                     seps.ctypes.data if seps.size else None, seps.shape[0],
                                     max_tokens, max_token_id, C.byref(h)), "sam_build_growing")
    return h.value


def sam_extend(handle: int, tokens: np.ndarray, wait: bool = True) -> None:
    """Appends host tokens; wait=False only queues them for the builder thread (sam_extend_async)."""
    t = np.ascontiguousarray(tokens, dtype=np.int32)
    fn = _load().sam_extend if wait else _load().sam_extend_async
    _check(fn(handle, t.ctypes.data if t.size else None, t.shape[0]), "sam_extend" if wait else "sam_extend_async")


def sam_pending(handle: int):
    """(tokens_queued, tokens_built, tokens_on_device)."""
    a, b, c = _i64(), _i64(), _i64()
    _check(_load().sam_pending(handle, C.byref(a), C.byref(b), C.byref(c)), "sam_pending")
    return a.value, b.value, c.value


def sam_sync(handle: int, stream=None) -> int:
    """Applies finished updates to the device copy; returns the tokens visible on the device."""
    n = _i64()
    _check(_load().sam_sync(handle, _stream(stream), C.byref(n)), "sam_sync")
    return int(n.value)


def sam_sync_renormalize(handle: int, B: int, state, matched_len, stream=None) -> int:
    """sam_sync and sam_renormalize in one call (one kernel when the pending update is small); returns the
    tokens visible on the device."""
    n = _i64()
    _check(_load().sam_sync_renormalize(handle, B, _dev(state), _dev(matched_len), _stream(stream), C.byref(n)),
           "sam_sync_renormalize")
    return int(n.value)


def sam_update_stats(handle: int):
    """(incremental updates, whole-image updates, bytes copied) applied by sam_sync so far."""
    a, b, c = _i64(), _i64(), _i64()
    _check(_load().sam_update_stats(handle, C.byref(a), C.byref(b), C.byref(c)), "sam_update_stats")
    return a.value, b.value, c.value


def sam_growing_set_relayout_every(handle: int, every: int) -> None:
    """Every `every`-th update of a growing index is sent as a whole image (0: only when it has to be)."""
    _check(_load().sam_growing_set_relayout_every(handle, every), "sam_growing_set_relayout_every")


def sam_renormalize(handle: int, B: int, state, matched_len, stream=None) -> None:
    _check(_load().sam_renormalize(handle, B, _dev(state), _dev(matched_len), _stream(stream)), "sam_renormalize")


def sam_sizes(handle: int):
    """(n_states, n_edges, device_bytes)."""
    a, b, c = _i64(), _i64(), _i64()
    _check(_load().sam_sizes(handle, C.byref(a), C.byref(b), C.byref(c)), "sam_sizes")
    return a.value, b.value, c.value


def sam_export(handle: int):
    """Flat host arrays of the automaton as a dict of numpy arrays."""
    S, E, _ = sam_sizes(handle)
    out = dict(len=np.empty(S, np.int32), link=np.empty(S, np.int32), firstpos=np.empty(S, np.int32),
               row_ptr=np.empty(S + 1, np.int64), edge_tok=np.empty(E, np.int32), edge_dst=np.empty(E, np.int32))
    _check(_load().sam_export(handle, out["len"].ctypes.data, out["link"].ctypes.data,
                              out["firstpos"].ctypes.data, out["row_ptr"].ctypes.data,
                              out["edge_tok"].ctypes.data, out["edge_dst"].ctypes.data), "sam_export")
    return out


def sam_upload(handle: int, device_buf, nbytes: Optional[int] = None, stream=None) -> None:
    nbytes = device_buf.numel() * device_buf.element_size() if nbytes is None else nbytes
    _check(_load().sam_upload(handle, _dev(device_buf), nbytes, _stream(stream)), "sam_upload")


def sam_free(handle: int) -> None:
    _load().sam_free(handle)


def sam_workspace_bytes(B: int, K: int) -> int:
    n = _load().sam_workspace_bytes(B, K)
    if n < 0:
        raise SamError(int(n), "sam_workspace_bytes")
    return int(n)


def sam_workspace_init(workspace, nbytes: Optional[int] = None, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size() if nbytes is None else nbytes
    _check(_load().sam_workspace_init(_dev(workspace), nbytes, _stream(stream)), "sam_workspace_init")


# ------------------------------------------------------------------ hot path
def sam_draft(handle, B, state, matched_len, new_tokens, ld, n_new, K, min_match, drafts, n_draft, stream=None):
    _check(_load().sam_draft(handle, B, _dev(state), _dev(matched_len), _dev(new_tokens), ld, _dev(n_new),
                             K, min_match, _dev(drafts), _dev(n_draft), _stream(stream)), "sam_draft")


def sam_verify(logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
               workspace, workspace_bytes, stream=None):
    _check(_load().sam_verify(_dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft), _dev(argmax_out),
                              _dev(accepted), _dev(n_accepted), _dev(workspace), workspace_bytes,
                              _stream(stream)), "sam_verify")


def sam_verify_static(logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted, stream=None):
    """sam_verify for callers that cannot allocate device scratch (an engine plugin whose host has
    already claimed all device memory, or code that only holds foreign raw pointers): the scratch is
    a fixed array inside the library, so B*(K+1) <= SAM_STATIC_MAX_ROWS and calls on one GPU must
    not overlap.  Same outputs as sam_verify."""
    _check(_load().sam_verify_static(_dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft),
                                     _dev(argmax_out), _dev(accepted), _dev(n_accepted), _stream(stream)),
           "sam_verify_static")


def sam_static_status(stream=None) -> int:
    """Status word of the last sam_verify_static call on the current device (0 = completed normally)."""
    out = _i32(0)
    _check(_load().sam_static_status(C.byref(out), _stream(stream)), "sam_static_status")
    return int(out.value)


def sam_step(handle, logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
             state, matched_len, min_match, next_drafts, next_n_draft, workspace, workspace_bytes, stream=None):
    _check(_load().sam_step(handle, _dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft),
                            _dev(argmax_out), _dev(accepted), _dev(n_accepted), _dev(state), _dev(matched_len),
                            min_match, _dev(next_drafts), _dev(next_n_draft), _dev(workspace), workspace_bytes,
                            _stream(stream)), "sam_step")


SAM_STEP_NO_SPECULATION = 1
SAM_STEP_SKIP_UNUSED_ROWS = 2
SAM_STEP_ROW_LIST_READY = 4
SAM_N_COUNTERS = 6


def sam_verify_ex(logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
                  flags, counters, workspace, workspace_bytes, stream=None):
    """sam_verify with step options (SAM_STEP_*) and optional device counters (int64[SAM_N_COUNTERS])."""
    _check(_load().sam_verify_ex(_dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft), _dev(argmax_out),
                                 _dev(accepted), _dev(n_accepted), flags, _dev(counters), _dev(workspace),
                                 workspace_bytes, _stream(stream)), "sam_verify_ex")


def sam_step_ex(handle, logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
                state, matched_len, min_match, next_drafts, next_n_draft, flags, counters,
                workspace, workspace_bytes, stream=None):
    """sam_step with step options (SAM_STEP_*) and optional device counters (int64[SAM_N_COUNTERS])."""
    _check(_load().sam_step_ex(handle, _dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft),
                               _dev(argmax_out), _dev(accepted), _dev(n_accepted), _dev(state), _dev(matched_len),
                               min_match, _dev(next_drafts), _dev(next_n_draft), flags, _dev(counters),
                               _dev(workspace), workspace_bytes, _stream(stream)), "sam_step_ex")


def sam_argmax_partial(logits, row_stride, rows, V, v_offset, keys, stream=None):
    """Packed per-row argmax words of a vocabulary shard (columns v_offset.. of the full vocabulary);
    keys: int64[rows + 1] device tensor (last word = status)."""
    _check(_load().sam_argmax_partial(_dev(logits), row_stride, rows, V, v_offset, _dev(keys), _stream(stream)),
           "sam_argmax_partial")


def sam_step_from_keys(handle, keys, B, K, drafts, n_draft, argmax_out, accepted, n_accepted,
                       state, matched_len, min_match, next_drafts, next_n_draft, stream=None):
    _check(_load().sam_step_from_keys(handle, _dev(keys), B, K, _dev(drafts), _dev(n_draft), _dev(argmax_out),
                                      _dev(accepted), _dev(n_accepted), _dev(state), _dev(matched_len), min_match,
                                      _dev(next_drafts), _dev(next_n_draft), _stream(stream)), "sam_step_from_keys")


class SamSet:
    """A table of uploaded indexes for composite drafting (owns the small device table)."""

    def __init__(self, indexes, device="cuda:0", stream=None):
        import torch
        self.indexes = list(indexes)                      # keeps the members alive
        n = len(self.indexes)
        nbytes = _load().sam_set_bytes(n)
        self.table = torch.empty(nbytes, dtype=torch.uint8, device=device)
        arr = (_vp * n)(*[ix.handle for ix in self.indexes])
        h = _vp()
        _check(_load().sam_set_create(arr, n, _dev(self.table), nbytes, _stream(stream), C.byref(h)), "sam_set_create")
        self.handle = h.value

    def refresh(self, stream=None):
        _check(_load().sam_set_refresh(self.handle, _stream(stream)), "sam_set_refresh")

    def renormalize(self, member: int, B: int, M: int, slots, state, matched_len, stream=None):
        """After member `member` has grown and refresh() was called: repair the slots that name it."""
        _check(_load().sam_set_renormalize(self.handle, member, B, M, _dev(slots), _dev(state), _dev(matched_len),
                                           _stream(stream)), "sam_set_renormalize")

    def close(self):
        h, self.handle = self.handle, None
        if h:
            _load().sam_set_free(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sam_multi_draft(set_handle, B, M, slots, weights, state, matched_len, new_tokens, ld, n_new, K, min_match,
                    drafts, n_draft, chosen, stream=None):
    _check(_load().sam_multi_draft(set_handle, B, M, _dev(slots), _dev(weights), _dev(state), _dev(matched_len),
                                   _dev(new_tokens), ld, _dev(n_new), K, min_match, _dev(drafts), _dev(n_draft),
                                   _dev(chosen), _stream(stream)), "sam_multi_draft")


def sam_multi_workspace_bytes(B: int, K: int, M: int) -> int:
    n = _load().sam_multi_workspace_bytes(B, K, M)
    if n < 0:
        raise SamError(int(n), "sam_multi_workspace_bytes")
    return int(n)


def sam_multi_step(set_handle, logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
                   M, slots, weights, state, matched_len, min_match, next_drafts, next_n_draft, chosen,
                   workspace, workspace_bytes, stream=None):
    _check(_load().sam_multi_step(set_handle, _dev(logits), row_stride, B, K, V, _dev(drafts), _dev(n_draft),
                                  _dev(argmax_out), _dev(accepted), _dev(n_accepted), M, _dev(slots), _dev(weights),
                                  _dev(state), _dev(matched_len), min_match, _dev(next_drafts), _dev(next_n_draft),
                                  _dev(chosen), _dev(workspace), workspace_bytes, _stream(stream)), "sam_multi_step")


def sam_adaptive_switch(context_len: int, batch_size: int, max_context_len: int, max_batch_size: int) -> bool:
    return bool(_load().sam_adaptive_switch(context_len, batch_size, max_context_len, max_batch_size))


def sam_speculation_pays(counters, K: int, cost_ratio: float) -> bool:
    """Counter-driven switch; `counters` is a HOST int64[SAM_N_COUNTERS] array (a copy of the device counters)."""
    c = np.ascontiguousarray(counters, dtype=np.int64)
    if c.shape != (SAM_N_COUNTERS,):
        raise ValueError("expected SAM_N_COUNTERS int64 values")
    r = _load().sam_speculation_pays(c.ctypes.data, K, float(cost_ratio))
    if r < 0:
        raise SamError(int(r), "sam_speculation_pays")
    return bool(r)


def _hostptr(a) -> Optional[int]:
    """Host address of a numpy array or a CPU torch tensor (contiguous)."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags.c_contiguous:
            raise ValueError("expected a contiguous array")
        return a.ctypes.data
    if a.is_cuda or not a.is_contiguous():
        raise ValueError("expected a contiguous host tensor")
    return a.data_ptr()


def sam_step_host_staging_bytes(row_stride: int, B: int, K: int, V: int) -> int:
    n = _load().sam_step_host_staging_bytes(row_stride, B, K, V)
    if n < 0:
        raise SamError(int(n), "sam_step_host_staging_bytes")
    return int(n)


def sam_step_host(handle, logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
                  state, matched_len, min_match, next_drafts, next_n_draft, staging, staging_bytes, stream=None):
    """All arrays are HOST memory (numpy or CPU torch tensors) except `staging` (device)."""
    _check(_load().sam_step_host(handle, _hostptr(logits), row_stride, B, K, V, _hostptr(drafts), _hostptr(n_draft),
                                 _hostptr(argmax_out), _hostptr(accepted), _hostptr(n_accepted), _hostptr(state),
                                 _hostptr(matched_len), min_match, _hostptr(next_drafts), _hostptr(next_n_draft),
                                 _dev(staging), staging_bytes, _stream(stream)), "sam_step_host")


def sam_step_host_ex(handle, logits, row_stride, B, K, V, drafts, n_draft, argmax_out, accepted, n_accepted,
                     state, matched_len, min_match, next_drafts, next_n_draft, flags, staging, staging_bytes, stream=None):
    """sam_step_host with step options; with SAM_STEP_SKIP_UNUSED_ROWS only the used rows are copied."""
    _check(_load().sam_step_host_ex(handle, _hostptr(logits), row_stride, B, K, V, _hostptr(drafts), _hostptr(n_draft),
                                    _hostptr(argmax_out), _hostptr(accepted), _hostptr(n_accepted), _hostptr(state),
                                    _hostptr(matched_len), min_match, _hostptr(next_drafts), _hostptr(next_n_draft),
                                    flags, _dev(staging), staging_bytes, _stream(stream)), "sam_step_host_ex")


def sam_workspace_status(workspace, B: int, K: int, stream=None) -> int:
    out = _i32(0)
    _check(_load().sam_workspace_status(_dev(workspace), B, K, C.byref(out), _stream(stream)), "sam_workspace_status")
    return int(out.value)


def sam_set_argmax_variant(variant: int) -> None:
    _check(_load().sam_set_argmax_variant(variant), "sam_set_argmax_variant")


def sam_profile_enable(max_calls: int) -> None:
    _check(_load().sam_profile_enable(max_calls), "sam_profile_enable")


def sam_profile_count() -> int:
    return int(_load().sam_profile_count())


def sam_profile_read(call: int):
    """(argmax_ms, accept_ms) of the call-th profiled sam_verify / sam_step."""
    a, b = C.c_float(), C.c_float()
    _check(_load().sam_profile_read(call, C.byref(a), C.byref(b)), "sam_profile_read")
    return a.value, b.value


def sam_strerror(status: int) -> str:
    return _load().sam_strerror(status).decode()


def sam_last_cuda_error() -> int:
    return int(_load().sam_last_cuda_error())


def sam_launch_count() -> int:
    return int(_load().sam_launch_count())


# ------------------------------------------------------------------ paged 4-bit key/value cache
SAM_CACHE_OUT_OF_PAGES = 1
SAM_CACHE_TABLE_FULL = 2
SAM_CACHE_BAD_FORK = 4
SAM_CACHE_GAVE_UP = 8
SAM_CACHE_BF16 = 0
SAM_CACHE_FP16 = 1
SAM_CACHE_MAX_B = 4096


class _CacheStruct(C.Structure):
    """struct sam_cache of include/sam.h."""
    _fields_ = [(n, _vp) for n in ("pages", "page_table", "seq_len", "ref_count", "free_list", "meta", "scratch")] + \
        [("scratch_bytes", _i64)] + \
        [(n, _i32) for n in ("n_pages", "page_tokens", "n_streams", "max_pages", "n_layers", "n_kv_heads", "head_dim",
                             "k_exp", "v_exp")]


def _size(n: int, where: str) -> int:
    if n < 0:
        raise SamError(int(n), where)
    return int(n)


def sam_cache_page_bytes(page_tokens: int, n_layers: int, n_kv_heads: int, head_dim: int) -> int:
    return _size(_load().sam_cache_page_bytes(page_tokens, n_layers, n_kv_heads, head_dim), "sam_cache_page_bytes")


def sam_cache_scratch_bytes(n_streams: int, n_pages: int) -> int:
    return _size(_load().sam_cache_scratch_bytes(n_streams, n_pages), "sam_cache_scratch_bytes")


def sam_cache_init(handle, stream=None) -> None:
    _check(_load().sam_cache_init(handle, _stream(stream)), "sam_cache_init")


def sam_cache_status(handle, stream=None):
    """(n_free, status bits); synchronises the stream."""
    a, b = _i32(), _i32()
    _check(_load().sam_cache_status(handle, C.byref(a), C.byref(b), _stream(stream)), "sam_cache_status")
    return a.value, b.value


def sam_cache_reserve(handle, B, streams, n_new, stream=None) -> None:
    _check(_load().sam_cache_reserve(handle, B, _dev(streams), _dev(n_new), _stream(stream)), "sam_cache_reserve")


def sam_cache_commit(handle, B, streams, n_keep, stream=None) -> None:
    _check(_load().sam_cache_commit(handle, B, _dev(streams), _dev(n_keep), _stream(stream)), "sam_cache_commit")


def sam_cache_fork(handle, n, src, dst, stream=None) -> None:
    _check(_load().sam_cache_fork(handle, n, _dev(src), _dev(dst), _stream(stream)), "sam_cache_fork")


def sam_cache_compact(handle, stream=None) -> None:
    _check(_load().sam_cache_compact(handle, _stream(stream)), "sam_cache_compact")


def sam_cache_copy_pages(src_handle, dst_handle, n, from_ids, to_ids, stream=None) -> None:
    _check(_load().sam_cache_copy_pages(src_handle, dst_handle, n, _dev(from_ids), _dev(to_ids), _stream(stream)),
           "sam_cache_copy_pages")


def sam_cache_append(handle, layer, k, v, dtype, row_stride, token_stride, head_stride, B, Q, streams, n_new,
                     stream=None) -> None:
    """k, v: raw addresses or contiguous tensors; strides in elements."""
    _check(_load().sam_cache_append(handle, layer, _dev(k), _dev(v), dtype, row_stride, token_stride, head_stride, B, Q,
                                    _dev(streams), _dev(n_new), _stream(stream)), "sam_cache_append")


def sam_cache_read(handle, layer, B, Q, streams, first, n, k_out, v_out, dtype, stream=None) -> None:
    _check(_load().sam_cache_read(handle, layer, B, Q, _dev(streams), _dev(first), _dev(n), _dev(k_out), _dev(v_out),
                                  dtype, _stream(stream)), "sam_cache_read")


def sam_cache_attend_workspace_bytes(handle, B: int, Q: int, H: int) -> int:
    return _size(_load().sam_cache_attend_workspace_bytes(handle, B, Q, H), "sam_cache_attend_workspace_bytes")


def sam_cache_attend(handle, layer, q, dtype, q_strides, B, Q, H, streams, n_new, scale, window, out, out_strides, lse,
                     workspace, workspace_bytes, stream=None) -> None:
    """q, out: raw addresses or contiguous tensors; q_strides, out_strides: (row, token, head) in elements."""
    _check(_load().sam_cache_attend(handle, layer, _dev(q), dtype, *q_strides, B, Q, H, _dev(streams), _dev(n_new),
                                    scale, window, _dev(out), *out_strides, _dev(lse), _dev(workspace), workspace_bytes,
                                    _stream(stream)), "sam_cache_attend")


class _RopeStruct(C.Structure):
    """struct sam_rope of include/sam.h."""
    _fields_ = [("turns", _vp), ("rotary_dim", _i32), ("interleaved", _i32), ("factor", C.c_float)]


def sam_rope_turns(inv_freq) -> np.ndarray:
    """Radians per position -> turns per position in units of 2^-64 (uint64)."""
    f = np.ascontiguousarray(inv_freq, dtype=np.float64)
    turns = np.empty(f.size, np.uint64)
    _check(_load().sam_rope_turns(f.ctypes.data, f.size, turns.ctypes.data), "sam_rope_turns")
    return turns


def sam_cache_append_rotated(handle, layer, q, q_strides, k, v, kv_strides, q_out, out_strides, dtype, rope, B, Q, H, streams,
                             n_new, positions, stream=None) -> None:
    """q, k, v, q_out: raw addresses or contiguous tensors; strides: (row, token, head) in elements; rope: address of a
    sam_rope (SamRope.handle)."""
    _check(_load().sam_cache_append_rotated(handle, layer, _dev(q), *q_strides, _dev(k), _dev(v), *kv_strides, _dev(q_out),
                                            *out_strides, dtype, rope, B, Q, H, _dev(streams), _dev(n_new),
                                            _dev(positions), _stream(stream)), "sam_cache_append_rotated")


def sam_cache_bounds_update(handle, layer, codes, exps, B, Q, streams, n_new, stream=None) -> None:
    _check(_load().sam_cache_bounds_update(handle, layer, _dev(codes), _dev(exps), B, Q, _dev(streams), _dev(n_new),
                                           _stream(stream)), "sam_cache_bounds_update")


def sam_cache_bounds_rebuild(handle, codes, exps, n, pages, stream=None) -> None:
    _check(_load().sam_cache_bounds_rebuild(handle, _dev(codes), _dev(exps), n, _dev(pages), _stream(stream)),
           "sam_cache_bounds_rebuild")


def sam_cache_select_workspace_bytes(handle, B: int, Q: int, share: int) -> int:
    return _size(_load().sam_cache_select_workspace_bytes(handle, B, Q, share), "sam_cache_select_workspace_bytes")


def sam_cache_select(handle, layer, codes, exps, q, dtype, q_strides, B, Q, H, streams, n_new, share, n_sink, n_recent,
                     blocks, n_blocks, workspace, workspace_bytes, stream=None) -> None:
    _check(_load().sam_cache_select(handle, layer, _dev(codes), _dev(exps), _dev(q), dtype, *q_strides, B, Q, H,
                                    _dev(streams), _dev(n_new), share, n_sink, n_recent, _dev(blocks), n_blocks,
                                    _dev(workspace), workspace_bytes, _stream(stream)), "sam_cache_select")


def sam_cache_attend_blocks_workspace_bytes(handle, B: int, Q: int, H: int, share: int) -> int:
    return _size(_load().sam_cache_attend_blocks_workspace_bytes(handle, B, Q, H, share),
                 "sam_cache_attend_blocks_workspace_bytes")


def sam_cache_attend_blocks(handle, layer, q, dtype, q_strides, B, Q, H, streams, n_new, blocks, n_blocks, share, scale, out,
                            out_strides, lse, workspace, workspace_bytes, stream=None) -> None:
    _check(_load().sam_cache_attend_blocks(handle, layer, _dev(q), dtype, *q_strides, B, Q, H, _dev(streams), _dev(n_new),
                                           _dev(blocks), n_blocks, share, scale, _dev(out), *out_strides, _dev(lse),
                                           _dev(workspace), workspace_bytes, _stream(stream)), "sam_cache_attend_blocks")


class SamRope:
    """A rotation: inv_freq (radians per position of each channel pair, in double precision) and how channels pair up."""

    def __init__(self, inv_freq, interleaved: bool = False, factor: float = 1.0, device="cuda:0", stream=None):
        import torch
        turns = torch.from_numpy(sam_rope_turns(inv_freq).view(np.int64))
        self.turns = SamCache._empty(turns.shape, torch.int64, device, stream)
        with SamCache._on(device, stream):
            self.turns.copy_(turns)
        self.rotary_dim = 2 * turns.numel()
        self._struct = _RopeStruct(_dev(self.turns), self.rotary_dim, int(interleaved), factor)
        self.handle = C.addressof(self._struct)


class SamCache:
    """A paged 4-bit key/value cache: owns (or is given) the torch tensors behind a `sam_cache` and marshals its calls.

    tensors: pages, and the books page_table, seq_len, ref_count, free_list, meta, if they exist already.  The books are
    given all together or not at all; then they are allocated, and the cache is emptied.  `handle` serves the
    `sam_cache_*` functions directly; the methods below take strided tensors [B, Q, heads, head_dim]."""

    BOOKS = ("page_table", "seq_len", "ref_count", "free_list", "meta")

    def __init__(self, n_pages: int, page_tokens: int, n_streams: int, max_pages: int, n_layers: int, n_kv_heads: int,
                 head_dim: int, k_exp: int = 0, v_exp: int = 0, device="cuda:0", tensors=None, stream=None):
        import torch
        self.page_bytes = sam_cache_page_bytes(page_tokens, n_layers, n_kv_heads, head_dim)
        shapes = dict(page_table=(n_streams, max_pages), seq_len=(n_streams,), ref_count=(n_pages,),
                      free_list=(n_pages,), meta=(4,))
        given = {n: t for n, t in (tensors or {}).items() if t is not None}
        books = given.keys() - {"pages"}
        if books and books != set(self.BOOKS):
            raise ValueError("tensors: the books " + ", ".join(self.BOOKS) + " are given all together or not at all")
        self.pages = given.get("pages")
        if self.pages is None:
            self.pages = self._empty((n_pages, n_layers, n_kv_heads, page_tokens // 16, 18 * head_dim), torch.uint8, device,
                                     stream)
        if self.pages.numel() * self.pages.element_size() != n_pages * self.page_bytes:
            raise ValueError("pages: n_pages * sam_cache_page_bytes() bytes are wanted")
        for name, shape in shapes.items():
            t = given.get(name)
            if t is None:
                t = self._empty(shape, torch.int32, device, stream)
            if tuple(t.shape) != shape or t.dtype != torch.int32:
                raise ValueError(f"{name}: an int32 tensor of shape {shape} is wanted")
            setattr(self, name, t)
        n_scratch = sam_cache_scratch_bytes(n_streams, n_pages)
        self.scratch = self._empty(n_scratch, torch.uint8, device, stream)
        self.n_streams, self.n_kv_heads, self.head_dim, self.page_tokens = n_streams, n_kv_heads, head_dim, page_tokens
        self._struct = _CacheStruct(*(_dev(getattr(self, n)) for n in ("pages", *self.BOOKS, "scratch")), n_scratch,
                                    n_pages, page_tokens, n_streams, max_pages, n_layers, n_kv_heads, head_dim, k_exp,
                                    v_exp)
        self.handle = C.addressof(self._struct)
        # Of attend, for calls that bring none: enough for few and for many query rows, so that it is never replaced.
        # Recorded graphs keep its address, and other streams may still use it.
        self._ws = self._empty(max(sam_cache_attend_workspace_bytes(self.handle, SAM_CACHE_MAX_B, q, n_kv_heads)
                                   for q in (1, 1 << 20)), torch.uint8, device, stream, zero=True)
        self._codes = {torch.bfloat16: SAM_CACHE_BF16, torch.float16: SAM_CACHE_FP16}
        if not books:
            sam_cache_init(self.handle, stream)

    @staticmethod
    def _on(device, stream):
        """The context of the stream that a call runs on."""
        import torch
        if stream is None:
            return contextlib.nullcontext()
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
        return torch.cuda.stream(stream)

    @staticmethod
    def _empty(shape, dtype, device, stream, zero=False):
        """A tensor that belongs to the stream that the call runs on, so that its memory is not handed on too early."""
        import torch
        make = torch.zeros if zero else torch.empty
        if stream is None:
            return make(shape, dtype=dtype, device=device)
        with SamCache._on(device, stream):
            return make(shape, dtype=dtype, device=device)

    @staticmethod
    def _new(like, shape, dtype, stream):
        """As _empty, on the device of a tensor; shape None: packed, of the tensor's own shape and type."""
        import torch
        if stream is not None:
            return SamCache._empty(like.shape if shape is None else shape, dtype or like.dtype, like.device, stream)
        if shape is None:
            return torch.empty_like(like, memory_format=torch.contiguous_format)
        return like.new_empty(shape, dtype=dtype)

    def _dtype(self, t) -> int:
        code = self._codes.get(t)
        if code is None:
            raise ValueError("bfloat16 or float16 is wanted")
        return code

    def _rows(self, t, heads: Optional[int]):
        """(address, strides of row, token and head)."""
        shape, strides = t.shape, t.stride()
        if len(shape) != 4 or shape[3] != self.head_dim or (heads is not None and shape[2] != heads):
            raise ValueError("a [B, Q, heads, head_dim] tensor is wanted")
        if not t.is_cuda or (strides[3] != 1 and t.numel()):
            raise ValueError("expected a CUDA tensor with contiguous channels")
        return t.data_ptr(), strides[:3]

    def _index(self, t, B: int):
        """Address of an int32 vector with one entry per row (or None)."""
        if t is None:
            return None
        if t.dtype != self.page_table.dtype or t.numel() != B:
            raise ValueError("an int32 tensor with one entry per row is wanted")
        return _dev(t)

    def reserve(self, n_new, streams=None, stream=None) -> None:
        B = n_new.numel()
        sam_cache_reserve(self.handle, B, self._index(streams, B), self._index(n_new, B), stream)

    def commit(self, n_keep, streams=None, stream=None) -> None:
        B = n_keep.numel()
        sam_cache_commit(self.handle, B, self._index(streams, B), self._index(n_keep, B), stream)

    def fork(self, src, dst, stream=None) -> None:
        n = src.numel()
        sam_cache_fork(self.handle, n, self._index(src, n), self._index(dst, n), stream)

    def compact(self, stream=None) -> None:
        sam_cache_compact(self.handle, stream)

    def copy_pages(self, to_cache: "SamCache", from_ids, to_ids, stream=None) -> None:
        n = from_ids.numel()
        sam_cache_copy_pages(self.handle, to_cache.handle, n, self._index(from_ids, n), self._index(to_ids, n), stream)

    def status(self, stream=None):
        return sam_cache_status(self.handle, stream)

    def append(self, layer: int, k, v, n_new=None, streams=None, stream=None) -> None:
        pk, st = self._rows(k, self.n_kv_heads)
        pv, sv = self._rows(v, self.n_kv_heads)
        if k.shape != v.shape or k.dtype != v.dtype or (st != sv and any(x != y and n > 1 for x, y, n in zip(st, sv, k.shape))):
            raise ValueError("keys and values of one shape, type and layout are wanted")
        B, Q = k.shape[:2]
        sam_cache_append(self.handle, layer, pk, pv, self._dtype(k.dtype), *st, B, Q, self._index(streams, B),
                         self._index(n_new, B), stream)

    def read(self, layer: int, first=None, n=None, max_n: Optional[int] = None, dtype=None, streams=None, out=None,
             stream=None):
        """(keys, values) [B, max_n, n_kv_heads, head_dim] of positions first .. first + n - 1."""
        import torch
        B = next((t.numel() for t in (streams, first, n) if t is not None), self.n_streams)
        if out is None:
            shape = (B, max_n, self.n_kv_heads, self.head_dim)
            out = tuple(self._empty(shape, dtype or torch.bfloat16, self.pages.device, stream) for _ in range(2))
        k, v = out
        if k.shape != v.shape or k.dtype != v.dtype or k.shape[0] != B or tuple(k.shape[2:]) != (self.n_kv_heads, self.head_dim):
            raise ValueError("two [B, max_n, n_kv_heads, head_dim] tensors of one type are wanted")
        sam_cache_read(self.handle, layer, B, k.shape[1], self._index(streams, B), self._index(first, B),
                       self._index(n, B), k, v, self._dtype(k.dtype), stream)
        return k, v

    def attend(self, layer: int, q, n_new=None, streams=None, scale: Optional[float] = None, window: int = 0, out=None,
               lse=None, workspace=None, stream=None):
        """(out, lse).  Without a workspace the call uses the cache's, which lives as long as the cache: calls that may
        overlap on the device (several streams) bring their own, zero-filled by sam_workspace_init."""
        import torch
        pq, sq = self._rows(q, None)
        B, Q, H = q.shape[:3]
        if out is None:
            out = self._empty(q.shape, q.dtype, q.device, stream)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out like q is wanted")
        if lse is None:
            lse = self._empty((B, Q, H), torch.float32, q.device, stream)
        elif tuple(lse.shape) != (B, Q, H) or lse.dtype != torch.float32:
            raise ValueError("a float32 lse [B, Q, H] is wanted")
        po, so = self._rows(out, H)
        if workspace is None:
            workspace = self._ws
        sam_cache_attend(self.handle, layer, pq, self._dtype(q.dtype), sq, B, Q, H, self._index(streams, B),
                         self._index(n_new, B), self.head_dim ** -0.5 if scale is None else scale, window, po, so, lse,
                         workspace, workspace.numel() * workspace.element_size(), stream)
        return out, lse


    def append_rotated(self, layer: int, q, k, v, rope: SamRope, n_new=None, streams=None, positions=None, out=None,
                       stream=None):
        """Queries and keys turned to their positions, keys and values appended; returns the turned queries (out may be q)."""
        pq, sq = self._rows(q, None)
        pk, sk = self._rows(k, self.n_kv_heads)
        pv, sv = self._rows(v, self.n_kv_heads)
        if k.shape != v.shape or k.dtype != v.dtype or (sk != sv and any(x != y and n > 1 for x, y, n in zip(sk, sv, k.shape))):
            raise ValueError("keys and values of one shape, type and layout are wanted")
        if q.dtype != k.dtype or q.shape[:2] != k.shape[:2]:
            raise ValueError("queries of the keys' type, rows and tokens are wanted")
        B, Q, H = q.shape[:3]
        if out is None:
            out = self._new(q, None, None, stream)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out like q is wanted")
        po, so = self._rows(out, H)
        if positions is not None and (tuple(positions.shape) != (B, Q) or positions.dtype != self.page_table.dtype):
            raise ValueError("int32 positions [B, Q] are wanted")
        sam_cache_append_rotated(self.handle, layer, pq, sq, pk, pv, sk, po, so, self._dtype(q.dtype), rope.handle, B, Q, H,
                                 self._index(streams, B), self._index(n_new, B), positions, stream)
        return out

    def attend_blocks(self, layer: int, q, blocks, share: int = 1, n_new=None, streams=None, scale: Optional[float] = None,
                      out=None, lse=None, workspace=None, stream=None):
        """(out, lse) over the listed blocks [B, ceil(Q / share), n_kv_heads, n]; otherwise as attend."""
        import torch
        pq, sq = self._rows(q, None)
        B, Q, H = q.shape[:3]
        if out is None:
            out = self._new(q, None, None, stream)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out like q is wanted")
        if lse is None:
            lse = self._new(q, (B, Q, H), torch.float32, stream)
        elif tuple(lse.shape) != (B, Q, H) or lse.dtype != torch.float32:
            raise ValueError("a float32 lse [B, Q, H] is wanted")
        if share < 1 or tuple(blocks.shape[:3]) != (B, -(-Q // share), self.n_kv_heads) or blocks.dim() != 4 or \
                blocks.dtype != torch.int32:
            raise ValueError("int32 blocks [B, ceil(Q / share), n_kv_heads, n] are wanted")
        po, so = self._rows(out, H)
        if workspace is None:
            workspace = self._ws
        sam_cache_attend_blocks(self.handle, layer, pq, self._dtype(q.dtype), sq, B, Q, H, self._index(streams, B),
                                self._index(n_new, B), blocks, blocks.shape[3], share,
                                self.head_dim ** -0.5 if scale is None else scale, po, so, lse, workspace,
                                workspace.numel() * workspace.element_size(), stream)
        return out, lse


class SamBounds:
    """Bounds of the keys of a cache's pages, and the selection of blocks from them.  Owns (or is given) codes int8
    [n_pages, n_layers, n_kv_heads, 2, head_dim] and exps int8 [n_pages, n_layers, n_kv_heads]."""

    def __init__(self, cache: SamCache, codes=None, exps=None, device=None, stream=None):
        import torch
        self.cache = cache
        n_pages, n_layers = cache._struct.n_pages, cache._struct.n_layers
        shape = (n_pages, n_layers, cache.n_kv_heads)
        device = cache.pages.device if device is None else device
        for name, t, want in (("codes", codes, shape + (2, cache.head_dim)), ("exps", exps, shape)):
            if t is None:
                t = SamCache._empty(want, torch.int8, device, stream)
            if tuple(t.shape) != want or t.dtype != torch.int8:
                raise ValueError(f"{name}: an int8 tensor of shape {want} is wanted")
            setattr(self, name, t)

    def update(self, layer: int, max_new: int, n_new=None, streams=None, stream=None) -> None:
        """After an append of up to max_new tokens a row: the bounds of the pages that it filled up."""
        c = self.cache
        B = next((t.numel() for t in (streams, n_new) if t is not None), c.n_streams)
        sam_cache_bounds_update(c.handle, layer, self.codes, self.exps, B, max_new, c._index(streams, B),
                                c._index(n_new, B), stream)

    def rebuild(self, pages=None, stream=None) -> None:
        """The bounds of the listed pages, or of all, in all layers."""
        n = self.cache._struct.n_pages if pages is None else pages.numel()
        sam_cache_bounds_rebuild(self.cache.handle, self.codes, self.exps, n, self.cache._index(pages, n), stream)

    def select(self, layer: int, q, n_blocks: int, n_sink: int = 1, n_recent: int = 2, share: int = 1, n_new=None,
               streams=None, out=None, workspace=None, stream=None):
        """int32 blocks [B, ceil(Q / share), n_kv_heads, n_blocks] for attend_blocks.  Without a workspace the call allocates one
        (sam_cache_select_workspace_bytes: up to 128 MB for most caches)."""
        import torch
        c = self.cache
        pq, sq = c._rows(q, None)
        B, Q, H = q.shape[:3]
        n = sam_cache_select_workspace_bytes(c.handle, B, Q, share)
        shape = (B, -(-Q // share), c.n_kv_heads, n_blocks)
        if out is None:
            out = c._new(q, shape, torch.int32, stream)
        elif tuple(out.shape) != shape or out.dtype != torch.int32:
            raise ValueError(f"an int32 tensor of shape {shape} is wanted")
        if workspace is None:
            workspace = c._new(q, (n,), torch.uint8, stream)
        sam_cache_select(c.handle, layer, self.codes, self.exps, pq, c._dtype(q.dtype), sq, B, Q, H, c._index(streams, B),
                         c._index(n_new, B), share, n_sink, n_recent, out, n_blocks, workspace,
                         workspace.numel() * workspace.element_size(), stream)
        return out


# ------------------------------------------------------------------ penalties, biases and masks
class _ShapeStruct(C.Structure):
    """struct sam_shape of include/sam.h."""
    _fields_ = [(n, _vp) for n in ("counts", "seen", "repetition", "presence", "frequency", "bias_tokens", "bias_values",
                                   "n_bias", "masks", "mask_of")] + \
        [(n, _i32) for n in ("n_streams", "max_bias", "n_masks")]


def sam_argmax_shaped(logits, row_stride, B, K, V, drafts, shape, keys, streams=None, stream=None) -> None:
    """shape: a SamShape (or the address of a sam_shape); keys: int64 [B * (K + 1)]; streams: int32 [B] (or an address)."""
    handle = shape.check(B, K, V) if isinstance(shape, SamShape) else shape
    if streams is not None and not isinstance(streams, int):
        import torch
        if streams.dtype != torch.int32 or streams.numel() != B:
            raise ValueError("int32 streams with one entry per row are wanted")
    _check(_load().sam_argmax_shaped(_dev(logits), row_stride, B, K, V, _dev(drafts), _dev(streams), handle, _dev(keys),
                                     _stream(stream)), "sam_argmax_shaped")


def sam_verify_from_keys(keys, B, K, drafts, n_draft, argmax_out, accepted, n_accepted, values=None, stream=None) -> None:
    _check(_load().sam_verify_from_keys(_dev(keys), B, K, _dev(drafts), _dev(n_draft), _dev(argmax_out), _dev(accepted),
                                        _dev(n_accepted), _dev(values), _stream(stream)), "sam_verify_from_keys")


def sam_history_add(counts, seen, n_streams, V, B, streams, tokens, ld, n, told, stream=None) -> None:
    _check(_load().sam_history_add(_dev(counts), _dev(seen), n_streams, V, B, _dev(streams), _dev(tokens), ld, _dev(n),
                                   int(told), _stream(stream)), "sam_history_add")


def sam_history_copy(counts, seen, n_streams, V, n, src, dst, stream=None) -> None:
    _check(_load().sam_history_copy(_dev(counts), _dev(seen), n_streams, V, n, _dev(src), _dev(dst), _stream(stream)),
           "sam_history_copy")


class SamHistory:
    """What each stream was told and has said: counts int32 [n_streams, V] and seen int32 [n_streams, ceil(V / 32)]."""

    def __init__(self, n_streams: int, V: int, device="cuda:0", stream=None):
        import torch
        self.n_streams, self.V = n_streams, V
        self.counts = SamCache._empty((n_streams, V), torch.int32, device, stream, zero=True)
        self.seen = SamCache._empty((n_streams, -(-V // 32)), torch.int32, device, stream, zero=True)

    def _rows(self, t, B: int):
        if t is not None and (t.dtype != self.counts.dtype or t.numel() != B):
            raise ValueError("an int32 tensor with one entry per row is wanted")
        return t

    def add(self, tokens, n=None, streams=None, told: bool = False, stream=None) -> None:
        """tokens int32 [B, ld], of which the first n[b] count; told: they were in the prompt."""
        if tokens.dim() != 2 or tokens.dtype != self.counts.dtype:
            raise ValueError("int32 tokens [B, ld] are wanted")
        B, ld = tokens.shape
        sam_history_add(self.counts, self.seen, self.n_streams, self.V, B, self._rows(streams, B), tokens, ld,
                        self._rows(n, B), told, stream)

    def fork(self, src, dst, stream=None) -> None:
        n = src.numel()
        sam_history_copy(self.counts, self.seen, self.n_streams, self.V, n, self._rows(src, n), self._rows(dst, n), stream)

    def reset(self, streams, stream=None) -> None:
        n = streams.numel()
        sam_history_copy(self.counts, self.seen, self.n_streams, self.V, n, None, self._rows(streams, n), stream)


class SamShape:
    """What logits are shaped by: keeps the tensors behind a `sam_shape` (all but V may be absent).

    counts, seen: of a SamHistory; repetition, presence, frequency: float32 [B]; bias_tokens int32, bias_values float32
    [B, n], n_bias int32 [B]; masks int32 [n, ceil(V / 32)] (a set bit allows a token) and mask_of int32 [B, K + 1]."""

    def __init__(self, V: int, counts=None, seen=None, repetition=None, presence=None, frequency=None, bias_tokens=None,
                 bias_values=None, n_bias=None, masks=None, mask_of=None):
        import torch
        words = -(-V // 32)
        self.V, self.mask_of, self.tensors = V, mask_of, dict(
            counts=counts, seen=seen, repetition=repetition, presence=presence, frequency=frequency, bias_tokens=bias_tokens,
            bias_values=bias_values, n_bias=n_bias, masks=masks, mask_of=mask_of)
        for name, last in (("counts", V), ("seen", words), ("masks", words), ("bias_tokens", None), ("mask_of", None)):
            t = self.tensors[name]
            if t is not None and (t.dim() != 2 or t.dtype != torch.int32 or (last and t.shape[1] != last)):
                raise ValueError(f"{name}: an int32 matrix{f' with {last} columns' if last else ''} is wanted")
        for pair in (("counts", "seen"), ("bias_tokens", "bias_values"), ("masks", "mask_of")):
            if len({self.tensors[n] is None for n in pair}) > 1:
                raise ValueError(" and ".join(pair) + " are given together or not at all")
        if counts is not None and counts.shape[0] != seen.shape[0]:
            raise ValueError("counts and seen of the same streams are wanted")
        if bias_tokens is not None and (bias_values.shape != bias_tokens.shape or bias_values.dtype != torch.float32):
            raise ValueError("bias_values: a float32 tensor like bias_tokens is wanted")
        for name, kind in (("repetition", torch.float32), ("presence", torch.float32), ("frequency", torch.float32),
                           ("n_bias", torch.int32)):
            t = self.tensors[name]
            if t is not None and (t.dim() != 1 or t.dtype != kind):
                raise ValueError(f"{name}: a {str(kind)[6:]} vector is wanted")
        n_bias_columns = 0 if bias_tokens is None else bias_tokens.shape[1]
        address = {n: None if t is not None and t.numel() == 0 else _dev(t) for n, t in self.tensors.items()}
        self._struct = _ShapeStruct(*address.values(), 0 if counts is None else counts.shape[0], n_bias_columns,
                                    0 if masks is None else masks.shape[0])
        self.handle = C.addressof(self._struct)
        per_row = [self.tensors[n] for n in self._PER_ROW]
        self._most = min((t.shape[0] for t in per_row if t is not None), default=None)   # rows of a call

    _PER_ROW = ("repetition", "presence", "frequency", "bias_tokens", "n_bias", "mask_of")

    def check(self, B: int, K: int, V: int) -> int:
        """The handle, if the tensors fit a call of this shape."""
        if V != self.V:
            raise ValueError("made for another vocabulary")
        if (self._most is None or B <= self._most) and (self.mask_of is None or self.mask_of.shape[1] == K + 1):
            return self.handle
        for name in self._PER_ROW:
            t = self.tensors[name]
            if t is not None and (t.shape[0] < B or (name == "mask_of" and t.shape[1] != K + 1)):
                raise ValueError(f"{name}: too small for {B} rows of {K + 1}")
        return self.handle


# ------------------------------------------------------------------ convenience holder
class SamIndex:
    """Owns a built handle and the torch tensor that holds its device blob (memory plumbing only)."""

    def __init__(self, corpus: np.ndarray, separators, device="cuda:0", upload: bool = True,
                 max_tokens: Optional[int] = None, max_token_id: Optional[int] = None):
        """max_tokens given: an index that can grow up to that many tokens (sam_build_growing)."""
        if max_tokens is None:
            self.handle = sam_build(corpus, separators)
        else:
            self.handle = sam_build_growing(corpus, separators, max_tokens, max_token_id)
        self.n_states, self.n_edges, self.device_bytes = sam_sizes(self.handle)
        self.blob = None
        if upload:
            import torch
            self.blob = torch.empty(self.device_bytes, dtype=torch.uint8, device=device)
            sam_upload(self.handle, self.blob)

    def close(self):
        h, self.handle = self.handle, None
        if h:
            sam_free(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
