"""Thin ctypes binding of the C ABI declared in include/freeze.h.

Argument marshalling only: every step of a look-up runs in the HIP kernels of
libfreeze_hip.so.  PyTorch supplies device memory (tensors) and the stream.
There is no fallback: if the library is not built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Dict, List, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "_lib", "libfreeze_hip.so")

FREEZE_OK, FREEZE_EINVAL, FREEZE_ELAYER, FREEZE_ENOTBUILT, FREEZE_EWORKSPACE, FREEZE_EHIP = 0, -1, -2, -3, -4, -5
FREEZE_ESCRATCH = -6
FREEZE_STATIC_SCRATCH_BYTES = 32 << 20
FREEZE_F32, FREEZE_BF16, FREEZE_E4M3 = 0, 1, 2

_lib = None


class FreezeState(ctypes.Structure):
    """freeze_state of the C ABI."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("outer", ctypes.c_int64), ("outer_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64), ("pieces", ctypes.c_int64), ("piece_stride", ctypes.c_int64),
                ("piece_bytes", ctypes.c_int64)]


class FreezeHeads(ctypes.Structure):
    """freeze_heads of the C ABI."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("src_token_stride", ctypes.c_int64), ("src_head_stride", ctypes.c_int64), ("dst_token_stride", ctypes.c_int64),
                ("dst_head_stride", ctypes.c_int64)]


class FreezePagesPool(ctypes.Structure):
    """freeze_pages of the C ABI."""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("tables", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("num_pages", ctypes.c_int64), ("rows", ctypes.c_int64), ("max_pages", ctypes.c_int64),
                ("layers", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32)]


class FreezeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().freeze_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{where}: {msg} ({code})")


def lib():
    """Load libfreeze_hip.so (built by `python -m paper_2002_02645_amd.build` / __graft_entry__.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build the HIP library first "
                           "(python -m paper_2002_02645_amd.build); there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    p, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    L.freeze_create.restype = i32
    L.freeze_create.argtypes = [ctypes.POINTER(p), i32]
    L.freeze_destroy.restype = i32
    L.freeze_destroy.argtypes = [p]
    L.freeze_cache_storage_bytes.restype = sz
    L.freeze_cache_storage_bytes.argtypes = [i64, i64, i32]
    L.freeze_cache_build.restype = i32
    L.freeze_cache_build.argtypes = [p, i32, p, i32, i64, i64, p, ctypes.c_int32, p, sz, p]
    L.freeze_set_centring.restype = i32
    L.freeze_set_centring.argtypes = [p, i32]
    L.freeze_lookup_workspace_bytes.restype = sz
    L.freeze_lookup_workspace_bytes.argtypes = [p, i32, i64, i32, i32]
    L.freeze_lookup.restype = i32
    L.freeze_lookup.argtypes = [p, i32, p, i64, i32, i32, i32, p, p, p, p, p, p, sz, p]
    L.freeze_lookup_static.restype = i32
    L.freeze_lookup_static.argtypes = [p, i32, p, i64, i32, i32, i32, p, p, p, p, p, p]
    L.freeze_cascade_workspace_bytes.restype = sz
    L.freeze_cascade_workspace_bytes.argtypes = [p, i32, p, i64, i32, i32]
    L.freeze_lookup_cascade.restype = i32
    L.freeze_lookup_cascade.argtypes = [p, i32, p, p, i64, i32, p, i32, p, p, p, p, sz, p]
    L.freeze_compact_misses.restype = i32
    L.freeze_compact_misses.argtypes = [p, p, i64, p, p, p]
    L.freeze_lookup_confidence.restype = i32
    L.freeze_lookup_confidence.argtypes = [p, i32, p, i64, i32, ctypes.c_float, i32, p, p, p, p, p, p, p, sz, p]
    L.freeze_lookup_cascade_confidence.restype = i32
    L.freeze_lookup_cascade_confidence.argtypes = [p, i32, p, p, i64, i32, p, i32, p, p, p, p, sz, p]
    L.freeze_kmeans_storage_bytes.restype = sz
    L.freeze_kmeans_storage_bytes.argtypes = [i64, i64]
    L.freeze_kmeans_workspace_bytes.restype = sz
    L.freeze_kmeans_workspace_bytes.argtypes = [p, i64, i64, i64]
    L.freeze_kmeans_build.restype = i32
    L.freeze_kmeans_build.argtypes = [p, i32, p, i64, i64, p, ctypes.c_int32, p, i64, i32, p, sz, p, sz, p]
    L.freeze_kmeans_read.restype = i32
    L.freeze_kmeans_read.argtypes = [p, i32, p, p, p, p]
    L.freeze_projection_storage_bytes.restype = sz
    L.freeze_projection_storage_bytes.argtypes = [i64, i64, i32]
    L.freeze_projection_build.restype = i32
    L.freeze_projection_build.argtypes = [p, i32, p, i32, i64, i64, p, p, sz, p, sz, p]
    L.freeze_project_workspace_bytes.restype = sz
    L.freeze_project_workspace_bytes.argtypes = [p, i32, i64]
    L.freeze_project.restype = i32
    L.freeze_project.argtypes = [p, i32, p, i64, i32, p, p, sz, p]
    L.freeze_gather_rows.restype = i32
    L.freeze_gather_rows.argtypes = [p, i64, p, p, i64, p, p]
    for name in ("freeze_quantised_code_stride", "freeze_quantised_scale_stride"):
        getattr(L, name).restype = i64
        getattr(L, name).argtypes = [i64]
    L.freeze_quantise_rows.restype = i32
    L.freeze_quantise_rows.argtypes = [p, i32, i64, i64, i64, p, p, p]
    L.freeze_quantised_storage_bytes.restype = sz
    L.freeze_quantised_storage_bytes.argtypes = [i64, i64]
    L.freeze_quantised_build.restype = i32
    L.freeze_quantised_build.argtypes = [p, i32, p, i32, p, i64, i64, p, p, sz, p]
    L.freeze_quantised_workspace_bytes.restype = sz
    L.freeze_quantised_workspace_bytes.argtypes = [p, i32, i64, i32]
    L.freeze_quantised_project.restype = i32
    L.freeze_quantised_project.argtypes = [p, i32, p, i32, p, i64, i64, i32, p, i32, i64, p, sz, p]
    L.freeze_beam_workspace_bytes.restype = sz
    L.freeze_beam_workspace_bytes.argtypes = [i64, i32, i64, i32]
    L.freeze_beam_select.restype = i32
    L.freeze_beam_select.argtypes = [p, i32, i64, i32, i64, i64, p, p, ctypes.c_int32, i32, p, p, p, p, p, sz, p]
    L.freeze_reorder_states.restype = i32
    L.freeze_reorder_states.argtypes = [p, i32, p, i64, i64, p]
    L.freeze_rotate_positions.restype = i32
    L.freeze_rotate_positions.argtypes = [p, i32, i64, i64, p, p, i64, i32, ctypes.c_float, i32, p]
    L.freeze_pages_bytes.restype = sz
    L.freeze_pages_bytes.argtypes = [p]
    L.freeze_pages_workspace_bytes.restype = sz
    L.freeze_pages_workspace_bytes.argtypes = [p]
    L.freeze_pages_reserve.restype = i32
    L.freeze_pages_reserve.argtypes = [p, p, p, p, sz, p]
    L.freeze_pages_fork.restype = i32
    L.freeze_pages_fork.argtypes = [p, p, p]
    L.freeze_pages_truncate.restype = i32
    L.freeze_pages_truncate.argtypes = [p, p, p]
    L.freeze_pages_compact.restype = i32
    L.freeze_pages_compact.argtypes = [p, p, p, sz, p]
    L.freeze_pages_append.restype = i32
    L.freeze_pages_append.argtypes = [p, i32, p, i64, i64, p, i64, i64, i32, i64, p, i64, p, p]
    L.freeze_pages_attend_workspace_bytes.restype = sz
    L.freeze_pages_attend_workspace_bytes.argtypes = [p, i32, i64, i64, i32]
    L.freeze_pages_attend.restype = i32
    L.freeze_pages_attend.argtypes = [p, i32, p, i32, i64, i64, i32, i64, p, i64, ctypes.c_float, i64, p, i32, i64, i64, p, sz, p]
    L.freeze_compute_thresholds.restype = i32
    L.freeze_compute_thresholds.argtypes = [p, i32, p, p, i64, i32, i32, p, p, p, sz, p]
    L.freeze_lookup_stats_attach.restype = i32
    L.freeze_lookup_stats_attach.argtypes = [p, p]
    L.freeze_profile_enable.restype = i32
    L.freeze_profile_enable.argtypes = [p, i32]
    L.freeze_profile_read.restype = i32
    L.freeze_profile_read.argtypes = [p, p, p]
    L.freeze_profile_read_calls.restype = i32
    L.freeze_profile_read_calls.argtypes = [p, p, i32, p]
    L.freeze_calibrate_mfma.restype = i32
    L.freeze_calibrate_mfma.argtypes = [p, sz, p, p]
    L.freeze_calibrate_hbm_read.restype = i32
    L.freeze_calibrate_hbm_read.argtypes = [p, sz, p]
    L.freeze_strerror.restype = ctypes.c_char_p
    L.freeze_strerror.argtypes = [i32]
    _lib = L
    return L


def _ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _check(rc: int, where: str):
    if rc != FREEZE_OK:
        raise FreezeError(rc, where)


# ---- functions with the names of the C entry points ---------------------------------------------

def freeze_strerror(code: int) -> str:
    return lib().freeze_strerror(code).decode()


def freeze_create(num_layers: int) -> ctypes.c_void_p:
    h = ctypes.c_void_p()
    _check(lib().freeze_create(ctypes.byref(h), num_layers), "freeze_create")
    return h


def freeze_destroy(ctx) -> None:
    _check(lib().freeze_destroy(ctx), "freeze_destroy")


def freeze_cache_storage_bytes(n: int, d: int, entries_dtype: int) -> int:
    return int(lib().freeze_cache_storage_bytes(n, d, entries_dtype))


def freeze_cache_build(ctx, layer: int, entries: torch.Tensor, labels: torch.Tensor, num_classes: int,
                       storage: torch.Tensor, stream=None) -> None:
    assert entries.is_cuda and entries.is_contiguous() and entries.dim() == 2
    assert labels.is_cuda and labels.dtype == torch.int32 and labels.is_contiguous()
    dt = {torch.float32: FREEZE_F32, torch.bfloat16: FREEZE_BF16}[entries.dtype]
    n, d = entries.shape
    assert labels.numel() == n
    _check(lib().freeze_cache_build(ctx, layer, _ptr(entries), dt, n, d, _ptr(labels), num_classes, _ptr(storage),
                                    storage.numel() * storage.element_size(), _stream(stream)), "freeze_cache_build")


def freeze_set_centring(ctx, mode: int) -> None:
    """0: caches built from now on are never centred, 1: when their mean dominates their spread (default), 2: always."""
    _check(lib().freeze_set_centring(ctx, mode), "freeze_set_centring")


def freeze_lookup_workspace_bytes(ctx, layer: int, b: int, k: int, rescore_r: int = 0) -> int:
    return int(lib().freeze_lookup_workspace_bytes(ctx, layer, b, k, rescore_r))


def freeze_lookup(ctx, layer: int, queries: torch.Tensor, k: int, vote_threshold: int, rescore_r: int,
                  out_labels: torch.Tensor, out_hit: torch.Tensor, out_votes: torch.Tensor,
                  out_nbr_idx: torch.Tensor, out_nbr_dist: torch.Tensor, workspace: torch.Tensor,
                  stream=None) -> None:
    assert queries.is_cuda and queries.dtype == torch.float32 and queries.is_contiguous() and queries.dim() == 2
    b = queries.shape[0]
    _check(lib().freeze_lookup(ctx, layer, _ptr(queries), b, k, vote_threshold, rescore_r, _ptr(out_labels),
                               _ptr(out_hit), _ptr(out_votes), _ptr(out_nbr_idx), _ptr(out_nbr_dist),
                               _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_lookup")


def freeze_lookup_static(ctx, layer: int, queries: torch.Tensor, k: int, vote_threshold: int, rescore_r: int,
                         out_labels: torch.Tensor, out_hit: torch.Tensor, out_votes: torch.Tensor,
                         out_nbr_idx: torch.Tensor, out_nbr_dist: torch.Tensor, stream=None) -> None:
    assert queries.is_cuda and queries.dtype == torch.float32 and queries.is_contiguous() and queries.dim() == 2
    b = queries.shape[0]
    _check(lib().freeze_lookup_static(ctx, layer, _ptr(queries), b, k, vote_threshold, rescore_r, _ptr(out_labels),
                                      _ptr(out_hit), _ptr(out_votes), _ptr(out_nbr_idx), _ptr(out_nbr_dist),
                                      _stream(stream)), "freeze_lookup_static")


def freeze_cascade_workspace_bytes(ctx, layers: Sequence[int], b: int, k: int, rescore_r: int = 0) -> int:
    arr = (ctypes.c_int * len(layers))(*layers)
    return int(lib().freeze_cascade_workspace_bytes(ctx, len(layers), arr, b, k, rescore_r))


def freeze_lookup_cascade(ctx, layers: Sequence[int], queries_per_layer: Sequence[torch.Tensor], k: int,
                          vote_thresholds: Sequence[int], rescore_r: int, out_labels: torch.Tensor,
                          out_exit_layer: torch.Tensor, out_hits_per_layer: torch.Tensor, workspace: torch.Tensor,
                          stream=None) -> None:
    nl = len(layers)
    assert len(queries_per_layer) == nl and len(vote_thresholds) == nl
    b = queries_per_layer[0].shape[0]
    for q in queries_per_layer:
        assert q.is_cuda and q.dtype == torch.float32 and q.is_contiguous() and q.shape[0] == b
    larr = (ctypes.c_int * nl)(*layers)
    tarr = (ctypes.c_int * nl)(*vote_thresholds)
    qarr = (ctypes.c_void_p * nl)(*[q.data_ptr() for q in queries_per_layer])
    _check(lib().freeze_lookup_cascade(ctx, nl, larr, qarr, b, k, tarr, rescore_r, _ptr(out_labels),
                                       _ptr(out_exit_layer), _ptr(out_hits_per_layer), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_lookup_cascade")


def freeze_lookup_confidence(ctx, layer: int, queries: torch.Tensor, k: int, conf_threshold: float, rescore_r: int,
                             out_labels: torch.Tensor, out_hit: torch.Tensor, out_conf: torch.Tensor,
                             out_votes: torch.Tensor, out_nbr_idx: torch.Tensor, out_nbr_dist: torch.Tensor,
                             workspace: torch.Tensor, stream=None) -> None:
    assert queries.is_cuda and queries.dtype == torch.float32 and queries.is_contiguous() and queries.dim() == 2
    b = queries.shape[0]
    _check(lib().freeze_lookup_confidence(ctx, layer, _ptr(queries), b, k, conf_threshold, rescore_r,
                                          _ptr(out_labels), _ptr(out_hit), _ptr(out_conf), _ptr(out_votes),
                                          _ptr(out_nbr_idx), _ptr(out_nbr_dist), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_lookup_confidence")


def _cascade_arrays(layers, queries_per_layer):
    nl = len(layers)
    assert len(queries_per_layer) == nl
    b = queries_per_layer[0].shape[0]
    for q in queries_per_layer:
        assert q.is_cuda and q.dtype == torch.float32 and q.is_contiguous() and q.shape[0] == b
    larr = (ctypes.c_int * nl)(*layers)
    qarr = (ctypes.c_void_p * nl)(*[q.data_ptr() for q in queries_per_layer])
    return nl, b, larr, qarr


def freeze_lookup_cascade_confidence(ctx, layers: Sequence[int], queries_per_layer: Sequence[torch.Tensor], k: int,
                                     conf_thresholds: Sequence[float], rescore_r: int, out_labels: torch.Tensor,
                                     out_exit_layer: torch.Tensor, out_hits_per_layer: torch.Tensor,
                                     workspace: torch.Tensor, stream=None) -> None:
    nl, b, larr, qarr = _cascade_arrays(layers, queries_per_layer)
    assert len(conf_thresholds) == nl
    tarr = (ctypes.c_float * nl)(*conf_thresholds)
    _check(lib().freeze_lookup_cascade_confidence(ctx, nl, larr, qarr, b, k, tarr, rescore_r, _ptr(out_labels),
                                                  _ptr(out_exit_layer), _ptr(out_hits_per_layer), _ptr(workspace),
                                                  workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_lookup_cascade_confidence")


def freeze_compute_thresholds(ctx, layers: Sequence[int], queries_per_layer: Sequence[torch.Tensor], k: int,
                              rescore_r: int, model_labels: torch.Tensor, out_thresholds: torch.Tensor,
                              workspace: torch.Tensor, stream=None) -> None:
    nl, b, larr, qarr = _cascade_arrays(layers, queries_per_layer)
    assert model_labels.is_cuda and model_labels.dtype == torch.int32 and model_labels.numel() == b
    assert out_thresholds.is_cuda and out_thresholds.dtype == torch.float32 and out_thresholds.numel() == nl
    _check(lib().freeze_compute_thresholds(ctx, nl, larr, qarr, b, k, rescore_r, _ptr(model_labels),
                                           _ptr(out_thresholds), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_compute_thresholds")


def freeze_kmeans_storage_bytes(num_centers: int, d: int) -> int:
    return int(lib().freeze_kmeans_storage_bytes(num_centers, d))


def freeze_kmeans_workspace_bytes(ctx, n: int, d: int, num_centers: int) -> int:
    return int(lib().freeze_kmeans_workspace_bytes(ctx, n, d, num_centers))


def freeze_kmeans_build(ctx, layer: int, points: torch.Tensor, labels: torch.Tensor, num_classes: int,
                        init_centers: torch.Tensor, iters: int, storage: torch.Tensor, workspace: torch.Tensor,
                        stream=None) -> None:
    assert points.is_cuda and points.dtype == torch.float32 and points.is_contiguous() and points.dim() == 2
    assert init_centers.is_cuda and init_centers.dtype == torch.float32 and init_centers.is_contiguous()
    assert init_centers.shape[1] == points.shape[1]
    assert labels.is_cuda and labels.dtype == torch.int32 and labels.numel() == points.shape[0]
    n, d = points.shape
    _check(lib().freeze_kmeans_build(ctx, layer, _ptr(points), n, d, _ptr(labels), num_classes, _ptr(init_centers),
                                     init_centers.shape[0], iters, _ptr(storage),
                                     storage.numel() * storage.element_size(), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_kmeans_build")


def freeze_kmeans_read(ctx, layer: int, out_centers: torch.Tensor, out_majority: torch.Tensor,
                       out_fraction: torch.Tensor, stream=None) -> None:
    _check(lib().freeze_kmeans_read(ctx, layer, _ptr(out_centers), _ptr(out_majority), _ptr(out_fraction),
                                    _stream(stream)), "freeze_kmeans_read")


def freeze_projection_storage_bytes(m: int, d: int, weights_dtype: int) -> int:
    return int(lib().freeze_projection_storage_bytes(m, d, weights_dtype))


def freeze_projection_build(ctx, slot: int, weights: torch.Tensor, bias: torch.Tensor, storage: torch.Tensor,
                            workspace: torch.Tensor, stream=None) -> None:
    assert weights.is_cuda and weights.is_contiguous() and weights.dim() == 2
    assert bias.is_cuda and bias.dtype == torch.float32 and bias.numel() == weights.shape[0]
    dtype = {torch.float32: FREEZE_F32, torch.bfloat16: FREEZE_BF16}[weights.dtype]
    _check(lib().freeze_projection_build(ctx, slot, _ptr(weights), dtype, weights.shape[0], weights.shape[1], _ptr(bias),
                                         _ptr(storage), storage.numel() * storage.element_size(), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)),
           "freeze_projection_build")


def freeze_project_workspace_bytes(ctx, slot: int, b: int) -> int:
    return int(lib().freeze_project_workspace_bytes(ctx, slot, b))


def freeze_project(ctx, slot: int, x: torch.Tensor, relu: bool, out: torch.Tensor, workspace: torch.Tensor,
                   stream=None) -> None:
    assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2
    assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.shape[0] == x.shape[0]
    _check(lib().freeze_project(ctx, slot, _ptr(x), x.shape[0], int(relu), _ptr(out), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)), "freeze_project")


def freeze_gather_rows(x: torch.Tensor, sel: torch.Tensor, count: Optional[torch.Tensor], out: torch.Tensor,
                       stream=None) -> None:
    assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2
    assert sel.dtype == torch.int32 and out.dtype == torch.float32 and out.is_contiguous()
    assert out.shape[0] >= sel.numel() and out.shape[1] == x.shape[1]
    _check(lib().freeze_gather_rows(_ptr(x), x.shape[1], _ptr(sel), _ptr(count), sel.numel(), _ptr(out),
                                    _stream(stream)), "freeze_gather_rows")


def _refused(why: str = "an argument's shape, type or layout is not what the call takes") -> AssertionError:
    """Raised in the place of an assert statement, which an optimised interpreter (-O) takes out: the library sees pointers alone, and would read or
    write past a wrong shape."""
    return AssertionError(why)


def freeze_quantised_code_stride(d: int) -> int:
    return int(lib().freeze_quantised_code_stride(d))


def freeze_quantised_scale_stride(d: int) -> int:
    return int(lib().freeze_quantised_scale_stride(d))


def _here(*tensors: Optional[torch.Tensor], holder: Optional["FreezeCache"] = None) -> int:
    """The library's kernels run on the current device, and a holder's outputs, scratch and weights are on its own.  Returns the device."""
    dev = torch.cuda.current_device()
    if holder is not None and holder._index != dev and holder._index is not None:
        raise _refused("the holder's device is not the current one")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise _refused("tensors of the current device are needed")
    return dev


def _at(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _on(stream) -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _here_and_now() -> tuple:
    """The current device and its current stream."""
    dev = torch.cuda.current_device()
    return dev, torch._C._cuda_getCurrentRawStream(dev)


def _rows_of(t: torch.Tensor) -> int:
    """Elements from row to row of a two-dimensional tensor whose rows are dense."""
    if not (t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise _refused()
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


_DTYPES = {torch.float32: FREEZE_F32, torch.bfloat16: FREEZE_BF16, torch.float8_e4m3fn: FREEZE_E4M3}


def _values_dtype(t: torch.Tensor) -> int:
    return _DTYPES[t.dtype]


def freeze_quantise_rows(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """codes [rows, freeze_quantised_code_stride(d)] float8_e4m3fn, scales [rows, freeze_quantised_scale_stride(d)] uint8."""
    _here(x, codes, scales)
    rows, d = x.shape
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise _refused()
    if not (codes.dtype == torch.float8_e4m3fn and codes.is_contiguous() and codes.shape == (rows, freeze_quantised_code_stride(d))):
        raise _refused()
    if not (scales.dtype == torch.uint8 and scales.is_contiguous() and scales.shape == (rows, freeze_quantised_scale_stride(d))):
        raise _refused()
    _check(lib().freeze_quantise_rows(_at(x), _values_dtype(x), rows, d, _rows_of(x), _at(codes), _at(scales), _on(stream)),
           "freeze_quantise_rows")


def freeze_quantised_storage_bytes(m: int, d: int) -> int:
    return int(lib().freeze_quantised_storage_bytes(m, d))


def freeze_quantised_build(ctx, slot: int, weights: torch.Tensor, scales: Optional[torch.Tensor], d: int, bias: Optional[torch.Tensor],
                           storage: torch.Tensor, stream=None) -> None:
    """weights [m, d] fp32 / bf16 (scales None), or codes [m, freeze_quantised_code_stride(d)] with their scales."""
    _here(weights, scales, bias, storage)
    m = weights.shape[0]
    if not (weights.is_contiguous() and weights.dim() == 2):
        raise _refused()
    if not (bias is None or (bias.dtype == torch.float32 and bias.is_contiguous() and bias.numel() == m)):
        raise _refused()
    if scales is None:
        if weights.shape[1] != d:
            raise _refused()
    else:
        if not (weights.dtype == torch.float8_e4m3fn and weights.shape[1] == freeze_quantised_code_stride(d)):
            raise _refused()
        if not (scales.dtype == torch.uint8 and scales.is_contiguous() and scales.shape == (m, freeze_quantised_scale_stride(d))):
            raise _refused()
    _check(lib().freeze_quantised_build(ctx, slot, _at(weights), _values_dtype(weights), _at(scales), m, d, _at(bias), _at(storage),
                                        storage.nbytes, _on(stream)), "freeze_quantised_build")


def freeze_quantised_workspace_bytes(ctx, slot: int, b: int, out_dtype: int) -> int:
    return int(lib().freeze_quantised_workspace_bytes(ctx, slot, b, out_dtype))


def freeze_quantised_project(ctx, slot: int, x: torch.Tensor, scales: Optional[torch.Tensor], d: int, relu: bool, out: torch.Tensor,
                             workspace: torch.Tensor, stream=None) -> None:
    """x [b, d] fp32 / bf16 (scales None), or codes with their scales; out [b, m] fp32 or bf16.  d, m: the built layer's."""
    _here(x, scales, out, workspace)
    b = x.shape[0]
    if not (out.dtype in (torch.float32, torch.bfloat16) and out.shape[0] == b):
        raise _refused()
    if scales is None:
        if x.shape[1] != d:
            raise _refused()
        stride = _rows_of(x)
    else:
        if not (x.dtype == torch.float8_e4m3fn and x.is_contiguous() and x.shape[1] == freeze_quantised_code_stride(d)):
            raise _refused()
        if not (scales.dtype == torch.uint8 and scales.is_contiguous() and scales.shape == (b, freeze_quantised_scale_stride(d))):
            raise _refused()
        stride = 0
    _check(lib().freeze_quantised_project(ctx, slot, _at(x), _values_dtype(x), _at(scales), b, stride, int(relu), _at(out),
                                          _values_dtype(out), _rows_of(out), _at(workspace),
                                          workspace.nbytes, _on(stream)), "freeze_quantised_project")


def freeze_beam_workspace_bytes(groups: int, beams: int, vocab: int, k: int) -> int:
    return int(lib().freeze_beam_workspace_bytes(groups, beams, vocab, k))


def freeze_beam_select(logits: torch.Tensor, scores: torch.Tensor, finished: Optional[torch.Tensor], beams: int, end_token: int, k: int,
                       out_scores: torch.Tensor, out_tokens: torch.Tensor, out_parents: torch.Tensor,
                       out_finished: Optional[torch.Tensor], workspace: torch.Tensor, stream=None) -> None:
    _here(logits, scores, finished, out_scores, out_tokens, out_parents, out_finished, workspace)
    rows, vocab = logits.shape
    if not (logits.dtype in (torch.float32, torch.bfloat16) and rows % beams == 0):
        raise _refused()
    if not (scores.dtype == torch.float32 and scores.is_contiguous() and scores.numel() == rows):
        raise _refused()
    if not (finished is None or (finished.dtype in (torch.uint8, torch.bool) and finished.is_contiguous() and finished.numel() == rows)):
        raise _refused()
    groups = rows // beams
    n = groups * k
    if not (out_scores.dtype == torch.float32 and out_scores.is_contiguous() and out_scores.numel() == n):
        raise _refused()
    if not (out_tokens.dtype == torch.int32 and out_tokens.is_contiguous() and out_tokens.numel() == n):
        raise _refused()
    if not (out_parents.dtype == torch.int32 and out_parents.is_contiguous() and out_parents.numel() == n):
        raise _refused()
    if not (out_finished is None or (out_finished.dtype == torch.uint8 and out_finished.is_contiguous() and out_finished.numel() == n)):
        raise _refused()
    _check(lib().freeze_beam_select(_at(logits), _values_dtype(logits), groups, beams, vocab, _rows_of(logits), _at(scores),
                                    _at(finished), end_token, k, _at(out_scores), _at(out_tokens), _at(out_parents),
                                    _at(out_finished), _at(workspace), workspace.nbytes,
                                    _on(stream)), "freeze_beam_select")


def state_of(src: torch.Tensor, dst: torch.Tensor, used: Optional[int] = None, row_dim: int = 0) -> FreezeState:
    """The freeze_state of two tensors of one shape, type and layout [outer..., rows, pieces..., places, width] (row_dim: the place of
    the rows; after it at most three dimensions, before it at most one).  used: how many places are taken along; None: all."""
    if not (src.shape == dst.shape and src.dtype == dst.dtype and src.stride() == dst.stride()):
        raise _refused("src and dst of one layout are needed")
    if not (0 <= row_dim <= 1 and src.dim() - row_dim <= 4 and src.dim() > row_dim):
        raise _refused()
    size = src.element_size()
    shape, stride = list(src.shape), list(src.stride())
    outer, outer_stride = (shape[0], stride[0]) if row_dim else (1, 0)
    row_stride = stride[row_dim]
    inner, istr = shape[row_dim + 1:], stride[row_dim + 1:]
    if used is not None:
        if not (len(inner) >= 2 and 0 <= used <= inner[-2]):
            raise _refused()
        inner[-2] = used
    pieces, piece_stride, run = 1, 0, size
    if inner:
        if not (istr[-1] == 1 or inner[-1] <= 1):
            raise _refused("the last dimension has to be dense")
        run *= inner[-1]
    if len(inner) >= 2:
        if istr[-2] * size == run or inner[-2] <= 1:
            run *= inner[-2]
            if len(inner) == 3:
                pieces, piece_stride = inner[0], istr[0]
        else:
            if not (len(inner) == 2 or inner[0] == 1):
                raise _refused("places that do not follow each other, in several pieces")
            pieces, piece_stride = inner[-2], istr[-2]
    return FreezeState(src.data_ptr(), dst.data_ptr(), outer, outer_stride * size, row_stride * size, pieces, piece_stride * size, run)


def freeze_reorder_states(states: Sequence[FreezeState], parents: torch.Tensor, src_rows: int, stream=None) -> None:
    """states as of state_of; row r of every dst becomes row parents[r] of its src."""
    _here(parents)
    if not (parents.dtype == torch.int32 and parents.is_contiguous()):
        raise _refused()
    arr = (FreezeState * len(states))(*states)
    _check(lib().freeze_reorder_states(ctypes.addressof(arr), len(states), _at(parents), parents.numel(), src_rows,
                                       _on(stream)), "freeze_reorder_states")


_HEADS = struct.Struct("QQiiqqqq")   # freeze_heads
_HEAD_TYPES = {torch.float32: FREEZE_F32, torch.bfloat16: FREEZE_BF16}


def _heads_of(t: torch.Tensor, heads: Optional[int] = None, dim: Optional[int] = None) -> tuple:
    """Elements from token to token and from head to head of a tensor [tokens, heads, dim] whose heads are dense."""
    shape = t.shape
    if len(shape) != 3 or t.dtype not in _HEAD_TYPES:
        raise _refused()
    tokens, n, d = shape
    if (heads is not None and n != heads) or (dim is not None and d != dim):
        raise _refused()
    if t.is_contiguous():
        return n * d, d
    token, head, one = t.stride()
    if one != 1 and d > 1:
        raise _refused("the last dimension has to be dense")
    return token if tokens > 1 else 0, head if n > 1 else 0


def _numbers(t: Optional[torch.Tensor], n: int) -> None:
    if t is not None and not (t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n):
        raise _refused("a dense int32 tensor of another size is needed")


def rotary_frequencies(pairs: int, base: float = 10000.0, stretch: float = 1.0, trained: int = 0, low: float = 1.0, high: float = 4.0,
                       device="cuda:0") -> torch.Tensor:
    """Frequencies of freeze_rotate_positions, radians a place, fp64: base ** (-i / pairs) for pair i.  stretch: for a context so many times
    longer than the one that a model was trained on, every frequency is divided by it; where `trained` (the places it was trained on) is given, one that turns
    at least `high` times within them stays as it is, one that turns less than `low` times is divided, those between go over linearly in the turns."""
    if pairs < 0 or not (base > 0 and stretch > 0 and (trained == 0 or high > low)):
        raise _refused()
    f = torch.tensor([base ** (-i / pairs) for i in range(pairs)], dtype=torch.float64)
    if trained:
        keep = ((trained * f / 6.283185307179586 - low) / (high - low)).clamp(0, 1)
        f = f * (keep + (1 - keep) / stretch)
    else:
        f = f / stretch
    return f.to(device)


def freeze_rotate_positions(tensors: Sequence[tuple], positions: torch.Tensor, frequencies: torch.Tensor, interleaved: bool = False, factor: float = 1.0,
                            inverse: bool = False, stream=None) -> None:
    """tensors: pairs (src, dst) of [tokens, heads, head_dim], dst of src's type and shape (or src itself: in place)."""
    if not tensors:
        return
    tokens, _, dim = tensors[0][0].shape
    arr = b""   # freeze_heads, one after another
    for src, dst in tensors:
        _here(src, dst)
        shape = src.shape
        if shape != dst.shape or src.dtype != dst.dtype or shape[0] != tokens or shape[2] != dim:
            raise _refused()
        arr += _HEADS.pack(src.data_ptr(), dst.data_ptr(), _DTYPES[src.dtype], shape[1], *_heads_of(src), *_heads_of(dst))
    _here(positions, frequencies)
    _numbers(positions, tokens)
    pairs = frequencies.numel()
    if not (frequencies.dtype == torch.float64 and frequencies.is_contiguous() and 2 * pairs <= dim):
        raise _refused()
    _check(lib().freeze_rotate_positions(arr, len(tensors), tokens, dim, positions.data_ptr(), frequencies.data_ptr(), pairs, int(interleaved), factor,
                                         int(inverse), _on(stream)), "freeze_rotate_positions")


def freeze_pages_bytes(pool: FreezePagesPool) -> int:
    return int(lib().freeze_pages_bytes(ctypes.addressof(pool)))


def freeze_pages_workspace_bytes(pool: FreezePagesPool) -> int:
    return int(lib().freeze_pages_workspace_bytes(ctypes.addressof(pool)))


def freeze_pages_reserve(pool: FreezePagesPool, add: Optional[torch.Tensor], granted: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _here(add, granted, workspace)
    _numbers(add, pool.rows)
    _numbers(granted, pool.rows)
    _check(lib().freeze_pages_reserve(ctypes.addressof(pool), _at(add), _at(granted), _at(workspace), workspace.nbytes, _on(stream)), "freeze_pages_reserve")


def freeze_pages_fork(pool: FreezePagesPool, parents: torch.Tensor, stream=None) -> None:
    _here(parents)
    _numbers(parents, pool.rows)
    _check(lib().freeze_pages_fork(ctypes.addressof(pool), _at(parents), _on(stream)), "freeze_pages_fork")


def freeze_pages_truncate(pool: FreezePagesPool, keep: torch.Tensor, stream=None) -> None:
    _here(keep)
    _numbers(keep, pool.rows)
    _check(lib().freeze_pages_truncate(ctypes.addressof(pool), _at(keep), _on(stream)), "freeze_pages_truncate")


def freeze_pages_compact(pool: FreezePagesPool, used: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _here(used, workspace)
    _numbers(used, 1)
    _check(lib().freeze_pages_compact(ctypes.addressof(pool), _at(used), _at(workspace), workspace.nbytes, _on(stream)), "freeze_pages_compact")


def freeze_pages_append(pool: FreezePagesPool, layer: int, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None, most: int = 0,
                        granted: Optional[torch.Tensor] = None, stream=None) -> None:
    """k, v [tokens, heads, head_dim] fp32 or bf16; starts [rows + 1] int32, or None for one token a row."""
    _here(k, v, starts, granted)
    if k.shape != v.shape or k.dtype != v.dtype:
        raise _refused()
    ks, vs = _heads_of(k, pool.heads, pool.head_dim), _heads_of(v, pool.heads, pool.head_dim)
    _numbers(starts, pool.rows + 1)
    _numbers(granted, pool.rows)
    _check(lib().freeze_pages_append(ctypes.addressof(pool), layer, k.data_ptr(), *ks, v.data_ptr(), *vs, _DTYPES[k.dtype], k.shape[0], _at(starts), most,
                                     _at(granted), _on(stream)), "freeze_pages_append")


def freeze_pages_attend_workspace_bytes(pool: FreezePagesPool, group: int, tokens: int, most: int = 0, packed: bool = True) -> int:
    return int(lib().freeze_pages_attend_workspace_bytes(ctypes.addressof(pool), group, tokens, most, int(packed)))


def freeze_pages_attend(pool: FreezePagesPool, layer: int, q: torch.Tensor, scale: float, out: torch.Tensor, workspace: torch.Tensor,
                        starts: Optional[torch.Tensor] = None, most: int = 0, window: int = 0, stream=None) -> None:
    """q, out [tokens, heads * group, head_dim] fp32 or bf16 each; starts [rows + 1] int32, or None for one token a row."""
    _here(q, out, workspace, starts)
    qs, os_ = _heads_of(q, None, pool.head_dim), _heads_of(out, None, pool.head_dim)
    if q.shape != out.shape or q.shape[1] == 0 or q.shape[1] % pool.heads != 0:
        raise _refused()
    _numbers(starts, pool.rows + 1)
    _check(lib().freeze_pages_attend(ctypes.addressof(pool), layer, q.data_ptr(), _DTYPES[q.dtype], *qs, q.shape[1] // pool.heads, q.shape[0], _at(starts), most,
                                     scale, window, out.data_ptr(), _DTYPES[out.dtype], *os_, _at(workspace), workspace.nbytes, _on(stream)),
           "freeze_pages_attend")


def freeze_compact_misses(hit: torch.Tensor, sel_in: Optional[torch.Tensor], sel_out: torch.Tensor,
                          out_count: torch.Tensor, stream=None) -> None:
    assert hit.is_cuda and hit.dtype == torch.uint8
    _check(lib().freeze_compact_misses(_ptr(hit), _ptr(sel_in), hit.numel(), _ptr(sel_out), _ptr(out_count),
                                       _stream(stream)), "freeze_compact_misses")


def freeze_lookup_stats_attach(ctx, counters: Optional[torch.Tensor]) -> None:
    """counters: device tensor of three int64 (confirmed at once, after the wider re-scoring, exact scans) or None."""
    if counters is not None:
        assert counters.is_cuda and counters.dtype == torch.int64 and counters.numel() >= 3 and counters.is_contiguous()
    _check(lib().freeze_lookup_stats_attach(ctx, _ptr(counters)), "freeze_lookup_stats_attach")


def freeze_profile_enable(ctx, enable) -> None:
    """enable: 0 / False off, 1 / True events at every stage boundary, 2 events around the distance pass only,
    3 the same for every eighth look-up."""
    _check(lib().freeze_profile_enable(ctx, int(enable)), "freeze_profile_enable")


def freeze_profile_read(ctx):
    """Returns ([prep_ms, dist_ms, finish_ms] summed, number of look-ups covered)."""
    ms = (ctypes.c_float * 3)()
    calls = ctypes.c_int(0)
    _check(lib().freeze_profile_read(ctx, ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(ctypes.byref(calls),
                                                                                     ctypes.c_void_p)),
           "freeze_profile_read")
    return [float(x) for x in ms], int(calls.value)


def freeze_profile_read_calls(ctx, max_calls: int = 256):
    """Returns a list of [prep_ms, dist_ms, finish_ms], one per recorded look-up, in call order."""
    ms = (ctypes.c_float * (3 * max_calls))()
    calls = ctypes.c_int(0)
    _check(lib().freeze_profile_read_calls(ctx, ctypes.cast(ms, ctypes.c_void_p), max_calls,
                                           ctypes.cast(ctypes.byref(calls), ctypes.c_void_p)),
           "freeze_profile_read_calls")
    return [[float(ms[3 * c + i]) for i in range(3)] for c in range(calls.value)]


def freeze_calibrate_mfma(scratch: torch.Tensor):
    """Returns (sustained bf16 MFMA TFLOP/s, shader clock in MHz under that load)."""
    tf, mhz = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib().freeze_calibrate_mfma(_ptr(scratch), scratch.numel() * scratch.element_size(),
                                       ctypes.cast(ctypes.byref(tf), ctypes.c_void_p),
                                       ctypes.cast(ctypes.byref(mhz), ctypes.c_void_p)), "freeze_calibrate_mfma")
    return float(tf.value), float(mhz.value)


def freeze_calibrate_hbm_read(buffer: torch.Tensor) -> float:
    """Returns the sustained read rate over `buffer` in GB/s."""
    gbs = ctypes.c_double(0.0)
    _check(lib().freeze_calibrate_hbm_read(_ptr(buffer), buffer.numel() * buffer.element_size(),
                                           ctypes.cast(ctypes.byref(gbs), ctypes.c_void_p)),
           "freeze_calibrate_hbm_read")
    return float(gbs.value)


# ---- convenience holder: owns the context, the per-layer storage and a reusable workspace ---------

class FreezeCache:
    """A context, the storage of its slots and scratch memory for each stream: calls on several streams may overlap, and calls may be captured into
    graphs (their scratch and outputs are of the graph's memory).  Building a slot and calls that use it on another stream are the caller's to order."""

    def __init__(self, num_layers: int, device="cuda:0"):
        self.device = torch.device(device)
        self._index = self.device.index if self.device.type == "cuda" else -1   # None: whichever device is the current one
        self.ctx = freeze_create(num_layers)
        self.storage: Dict[int, torch.Tensor] = {}
        self.meta: Dict[int, tuple] = {}
        self._scratch: Dict[tuple, torch.Tensor] = {}   # by device and stream

    def close(self):
        if self.ctx is not None:
            freeze_destroy(self.ctx)
            self.ctx = None

    @property
    def _ws(self) -> Optional[torch.Tensor]:
        return self._scratch.get(_here_and_now())

    def _workspace(self, nbytes: int, at: Optional[tuple] = None) -> torch.Tensor:
        # One for each stream: calls on a stream follow one another, those on two may overlap.  (Where a larger one replaces it, the old one's memory
        # goes back to the stream it is used on.)  A captured call keeps none: its replays run beside whatever the stream does then.
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        at = at or _here_and_now()
        ws = self._scratch.get(at)
        if ws is None or ws.numel() < nbytes:
            ws = self._scratch[at] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        return ws

    def build_layer(self, layer: int, entries: torch.Tensor, labels: torch.Tensor, num_classes: int):
        n, d = entries.shape
        dt = FREEZE_F32 if entries.dtype == torch.float32 else FREEZE_BF16
        nbytes = freeze_cache_storage_bytes(n, d, dt)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_cache_storage_bytes")
        st = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        freeze_cache_build(self.ctx, layer, entries, labels, num_classes, st)
        self.storage[layer] = st
        self.meta[layer] = (n, d, num_classes)

    def alloc_outputs(self, b: int, k: int):
        dev = self.device
        return dict(label=torch.empty(b, dtype=torch.int32, device=dev),
                    hit=torch.empty(b, dtype=torch.uint8, device=dev),
                    votes=torch.empty(b, dtype=torch.int32, device=dev),
                    idx=torch.empty((b, k), dtype=torch.int32, device=dev),
                    dist=torch.empty((b, k), dtype=torch.float32, device=dev))

    def lookup(self, layer: int, queries: torch.Tensor, k: int, vote_threshold: int, rescore_r: int = 0,
               out: Optional[dict] = None) -> dict:
        b = queries.shape[0]
        if out is None:
            out = self.alloc_outputs(b, k)
        nbytes = freeze_lookup_workspace_bytes(self.ctx, layer, b, k, rescore_r)
        ws = self._workspace(nbytes)
        freeze_lookup(self.ctx, layer, queries, k, vote_threshold, rescore_r, out["label"], out["hit"], out["votes"],
                      out["idx"], out["dist"], ws)
        return out

    def lookup_cascade(self, layers: Sequence[int], queries_per_layer: List[torch.Tensor], k: int,
                       vote_thresholds: Sequence[int], rescore_r: int = 0, out: Optional[dict] = None) -> dict:
        b = queries_per_layer[0].shape[0]
        if out is None:
            out = dict(label=torch.empty(b, dtype=torch.int32, device=self.device),
                       exit_layer=torch.empty(b, dtype=torch.int32, device=self.device),
                       hits_per_layer=torch.empty(len(layers), dtype=torch.int64, device=self.device))
        nbytes = freeze_cascade_workspace_bytes(self.ctx, layers, b, k, rescore_r)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_cascade_workspace_bytes")
        ws = self._workspace(nbytes)
        freeze_lookup_cascade(self.ctx, layers, queries_per_layer, k, vote_thresholds, rescore_r, out["label"],
                              out["exit_layer"], out["hits_per_layer"], ws)
        return out

    def lookup_confidence(self, layer: int, queries: torch.Tensor, k: int, conf_threshold: float, rescore_r: int = 0,
                          out: Optional[dict] = None) -> dict:
        b = queries.shape[0]
        if out is None:
            out = self.alloc_outputs(b, k)
            out["conf"] = torch.empty(b, dtype=torch.float32, device=self.device)
        nbytes = freeze_lookup_workspace_bytes(self.ctx, layer, b, k, rescore_r)
        ws = self._workspace(nbytes)
        freeze_lookup_confidence(self.ctx, layer, queries, k, conf_threshold, rescore_r, out["label"], out["hit"],
                                 out["conf"], out["votes"], out["idx"], out["dist"], ws)
        return out

    def lookup_cascade_confidence(self, layers: Sequence[int], queries_per_layer: List[torch.Tensor], k: int,
                                  conf_thresholds: Sequence[float], rescore_r: int = 0) -> dict:
        b = queries_per_layer[0].shape[0]
        out = dict(label=torch.empty(b, dtype=torch.int32, device=self.device),
                   exit_layer=torch.empty(b, dtype=torch.int32, device=self.device),
                   hits_per_layer=torch.empty(len(layers), dtype=torch.int64, device=self.device))
        nbytes = freeze_cascade_workspace_bytes(self.ctx, layers, b, k, rescore_r)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_cascade_workspace_bytes")
        ws = self._workspace(nbytes)
        freeze_lookup_cascade_confidence(self.ctx, layers, queries_per_layer, k, conf_thresholds, rescore_r,
                                         out["label"], out["exit_layer"], out["hits_per_layer"], ws)
        return out

    def compute_thresholds(self, layers: Sequence[int], queries_per_layer: List[torch.Tensor], k: int,
                           model_labels: torch.Tensor, rescore_r: int = 0) -> torch.Tensor:
        b = queries_per_layer[0].shape[0]
        thr = torch.empty(len(layers), dtype=torch.float32, device=self.device)
        nbytes = freeze_cascade_workspace_bytes(self.ctx, layers, b, k, rescore_r)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_cascade_workspace_bytes")
        ws = self._workspace(nbytes)
        freeze_compute_thresholds(self.ctx, layers, queries_per_layer, k, rescore_r, model_labels, thr, ws)
        return thr

    def build_kmeans_layer(self, layer: int, points: torch.Tensor, labels: torch.Tensor, num_classes: int,
                           init_centers: torch.Tensor, iters: int) -> dict:
        """k-means cache of `points` (Sec. 4); returns the centres, majority labels and shares."""
        n, d = points.shape
        kc = init_centers.shape[0]
        nbytes = freeze_kmeans_storage_bytes(kc, d)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_kmeans_storage_bytes")
        st = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        wbytes = freeze_kmeans_workspace_bytes(self.ctx, n, d, kc)
        if wbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_kmeans_workspace_bytes")
        ws = self._workspace(wbytes)
        freeze_kmeans_build(self.ctx, layer, points, labels, num_classes, init_centers, iters, st, ws)
        self.storage[layer] = st
        self.meta[layer] = (kc, d, num_classes)
        out = dict(centers=torch.empty((kc, d), dtype=torch.float32, device=self.device),
                   majority=torch.empty(kc, dtype=torch.int32, device=self.device),
                   fraction=torch.empty(kc, dtype=torch.float32, device=self.device))
        freeze_kmeans_read(self.ctx, layer, out["centers"], out["majority"], out["fraction"])
        return out

    def build_projection(self, slot: int, weights: torch.Tensor, bias: torch.Tensor):
        """A dense layer y = W x + bias in front of a look-up (Sec. 3); occupies one slot of the context."""
        m, d = weights.shape
        dtype = FREEZE_BF16 if weights.dtype == torch.bfloat16 else FREEZE_F32
        nbytes = freeze_projection_storage_bytes(m, d, dtype)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_projection_storage_bytes")
        st = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        ws = self._workspace(256 + 4 * m)
        freeze_projection_build(self.ctx, slot, weights, bias, st, ws)
        self.storage[slot] = st
        self.meta[slot] = (m, d, 0)

    def project(self, slot: int, x: torch.Tensor, relu: bool = False) -> torch.Tensor:
        m = self.meta[slot][0]
        out = torch.empty((x.shape[0], m), dtype=torch.float32, device=self.device)
        nbytes = freeze_project_workspace_bytes(self.ctx, slot, x.shape[0])
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_project_workspace_bytes")
        freeze_project(self.ctx, slot, x, relu, out, self._workspace(nbytes))
        return out

    def quantise_rows(self, x: torch.Tensor):
        """Rows in 8 bits: codes [rows, d rounded up to 128] float8_e4m3fn and a scale byte for each block of 128 values."""
        dev = _here(x, holder=self)
        if x.dtype not in (torch.float32, torch.bfloat16):
            raise _refused()
        rows, d = x.shape
        codes = torch.empty((rows, -(-d // 128) * 128), dtype=torch.float8_e4m3fn, device=self.device)
        scales = torch.empty((rows, -(-d // 512) * 4), dtype=torch.uint8, device=self.device)
        _check(lib().freeze_quantise_rows(x.data_ptr(), _values_dtype(x), rows, d, _rows_of(x), codes.data_ptr(), scales.data_ptr(), torch._C._cuda_getCurrentRawStream(dev)),
               "freeze_quantise_rows")
        return codes, scales

    def build_quantised(self, slot: int, weights: torch.Tensor, bias: Optional[torch.Tensor] = None,
                        scales: Optional[torch.Tensor] = None, d: Optional[int] = None):
        """A dense layer y = W x + bias in 8 bits (a model's output layer, or the layer in front of a look-up); occupies one slot.
        weights: fp32 / bf16, quantised here, or codes with their scales (d: the values of a row, where fewer than the codes)."""
        _here(weights, scales, bias, holder=self)
        m = weights.shape[0]
        d = weights.shape[1] if d is None else d
        nbytes = freeze_quantised_storage_bytes(m, d)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_quantised_storage_bytes")
        st = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        freeze_quantised_build(self.ctx, slot, weights, scales, d, bias, st)
        self.storage[slot] = st
        self.meta[slot] = (m, d, 0)

    def quantised_project(self, slot: int, x: torch.Tensor, scales: Optional[torch.Tensor] = None, relu: bool = False,
                          out_dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: fp32 / bf16 rows, or codes with their scales."""
        dev = _here(x, scales, out, holder=self)
        m, d, _ = self.meta[slot]
        b = x.shape[0]
        if out is None:
            out = torch.empty((b, m), dtype=out_dtype, device=self.device)
        if not (out.shape == (b, m) and out.dtype in (torch.float32, torch.bfloat16)):
            raise _refused()
        if scales is None:
            if not (x.shape[1] == d and x.dtype in (torch.float32, torch.bfloat16)):
                raise _refused()
            stride = _rows_of(x)
        else:
            if not (x.dtype == torch.float8_e4m3fn and x.is_contiguous() and x.shape == (b, -(-d // 128) * 128)):
                raise _refused()
            if not (scales.dtype == torch.uint8 and scales.is_contiguous() and scales.shape == (b, -(-d // 512) * 4)):
                raise _refused()
            stride = 0
        out_type = _values_dtype(out)
        nbytes = lib().freeze_quantised_workspace_bytes(self.ctx, slot, b, out_type)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_quantised_workspace_bytes")
        stream = torch._C._cuda_getCurrentRawStream(dev)
        ws = self._workspace(nbytes, (dev, stream))
        _check(lib().freeze_quantised_project(self.ctx, slot, x.data_ptr(), _values_dtype(x), _at(scales), b, stride, int(relu), out.data_ptr(),
                                              out_type, _rows_of(out), ws.data_ptr(), ws.numel(), stream), "freeze_quantised_project")
        return out

    def beam_select(self, logits: torch.Tensor, scores: torch.Tensor, beams: int, k: int, finished: Optional[torch.Tensor] = None,
                    end_token: int = -1) -> dict:
        """The k best continuations of every group of `beams` rows: score, token, parent (row), finished; each [groups, k]."""
        rows, vocab = logits.shape
        dev = _here(logits, scores, finished, holder=self)
        if not (rows % beams == 0 and scores.dtype == torch.float32 and scores.is_contiguous() and scores.numel() == rows):
            raise _refused()
        if not (finished is None or (finished.dtype in (torch.uint8, torch.bool) and finished.is_contiguous() and finished.numel() == rows)):
            raise _refused()
        if logits.dtype not in (torch.float32, torch.bfloat16):
            raise _refused()
        groups = rows // beams
        nbytes = lib().freeze_beam_workspace_bytes(groups, beams, vocab, k)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_beam_workspace_bytes")
        stream = torch._C._cuda_getCurrentRawStream(dev)
        ws = self._workspace(nbytes, (dev, stream))
        words = torch.empty((3, groups, k), dtype=torch.int32, device=self.device)
        ended = torch.empty((groups, k), dtype=torch.uint8, device=self.device)
        at, size = words.data_ptr(), 4 * groups * k
        _check(lib().freeze_beam_select(logits.data_ptr(), _values_dtype(logits), groups, beams, vocab, _rows_of(logits), scores.data_ptr(),
                                        _at(finished), end_token, k, at, at + size, at + 2 * size, ended.data_ptr(), ws.data_ptr(), ws.numel(),
                                        stream), "freeze_beam_select")
        score, token, parent = words.unbind(0)
        return dict(score=score.view(torch.float32), token=token, parent=parent, finished=ended)

    def reorder_states(self, src, dst, parents: torch.Tensor, used: Optional[int] = None, row_dim: int = 0) -> None:
        """Row r of every dst becomes row parents[r] of its src (tensors or lists of tensors; see state_of)."""
        if isinstance(src, torch.Tensor):
            src, dst = (src,), (dst,)
        if len(src) != len(dst):
            raise _refused()
        if not src:
            return
        _here(*src, *dst)
        rows = src[0].shape[row_dim]
        if not (parents.numel() <= rows and all(t.shape[row_dim] == rows for t in src)):   # (state_of: a dst is like its src)
            raise _refused()
        freeze_reorder_states([state_of(s, d, used, row_dim) for s, d in zip(src, dst)], parents, rows)

    def rotate_positions(self, x, positions: torch.Tensor, frequencies: torch.Tensor, interleaved: bool = False, factor: float = 1.0,
                         inverse: bool = False, out=None):
        """Heads turned by their tokens' places (a tensor [tokens, heads, head_dim], or several that share positions; see rotary_frequencies).
        out: where they go, x itself for in place; None: new tensors."""
        one = isinstance(x, torch.Tensor)
        xs = (x,) if one else x
        outs = list(map(torch.empty_like, xs)) if out is None else [out] if one else list(out)
        if len(outs) != len(xs):
            raise _refused()
        dev = _here(*xs, *outs, positions, frequencies, holder=self)
        if not outs:
            return outs
        tokens, _, dim = xs[0].shape
        pairs, arr = frequencies.numel(), b""
        for src, dst in zip(xs, outs):
            strides, shape, dtype = _heads_of(src, None, dim), src.shape, src.dtype
            if shape[0] != tokens:
                raise _refused()
            if out is None and src.is_contiguous():
                to = strides
            else:
                if dst.shape != shape or dst.dtype != dtype:
                    raise _refused()
                to = _heads_of(dst)
            arr += _HEADS.pack(src.data_ptr(), dst.data_ptr(), _HEAD_TYPES[dtype], shape[1], *strides, *to)
        _numbers(positions, tokens)
        if not (frequencies.dtype == torch.float64 and frequencies.is_contiguous() and 2 * pairs <= dim):
            raise _refused()
        _check(lib().freeze_rotate_positions(arr, len(outs), tokens, dim, positions.data_ptr(), frequencies.data_ptr(), pairs, interleaved, factor, inverse,
                                             torch._C._cuda_getCurrentRawStream(dev)), "freeze_rotate_positions")
        return outs[0] if one else outs


class FreezePages:
    """A generating model's keys and values in pages of 8 bits: the pool, the rows' tables and scratch memory for each stream.  Rows start empty.  What changes the
    pool (reserve, fork, truncate, compact, append) and calls that read it on another stream are the caller's to order."""

    def __init__(self, layers: int, num_pages: int, rows: int, max_pages: int, heads: int, head_dim: int, page_tokens: int = 64, device="cuda:0"):
        self.device = torch.device(device)
        self._index = self.device.index if self.device.type == "cuda" else -1
        self.pool = FreezePagesPool(None, None, None, None, None, num_pages, rows, max_pages, layers, heads, head_dim, page_tokens)
        nbytes = freeze_pages_bytes(self.pool)
        if nbytes == 0:
            raise FreezeError(FREEZE_EINVAL, "freeze_pages_bytes")
        width = (head_dim + 31) // 32 * 32
        lead = (layers, num_pages, heads, page_tokens // 32, 2)
        self.codes = torch.zeros((*lead, 32 * width), dtype=torch.uint8, device=self.device).view(torch.float8_e4m3fn)
        self.scales = torch.full(lead, 1, dtype=torch.uint8, device=self.device)
        # the bookkeeping in one run of memory: tables, lengths, references
        self.book = torch.zeros(rows * max_pages + rows + num_pages, dtype=torch.int32, device=self.device)
        tables, self.lengths, self.refs = self.book.split([rows * max_pages, rows, num_pages])
        self.tables = tables.view(rows, max_pages)
        self.tables.fill_(-1)
        self.pool.codes, self.pool.scales = self.codes.data_ptr(), self.scales.data_ptr()
        self.pool.refs, self.pool.tables, self.pool.lengths = self.refs.data_ptr(), self.tables.data_ptr(), self.lengths.data_ptr()
        self._scratch: Dict[tuple, torch.Tensor] = {}   # by device and stream
        self._at = ctypes.addressof(self.pool)
        self._book_bytes = freeze_pages_workspace_bytes(self.pool)
        self._attend_bytes: Dict[tuple, int] = {}       # by what the size goes by

    _workspace = FreezeCache._workspace

    def reserve(self, add: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Room for add[row] more tokens of every row (None: one each), whose lengths grow; returns what each row was granted, [rows]."""
        dev, pool = _here(add, holder=self), self.pool
        _numbers(add, pool.rows)
        granted = torch.empty(pool.rows, dtype=torch.int32, device=self.device)
        stream = torch._C._cuda_getCurrentRawStream(dev)
        ws = self._workspace(self._book_bytes, (dev, stream))
        _check(lib().freeze_pages_reserve(self._at, _at(add), granted.data_ptr(), ws.data_ptr(), ws.numel(), stream), "freeze_pages_reserve")
        return granted

    def fork(self, parents: torch.Tensor) -> None:
        """Row r becomes what row parents[r] was, on the same pages (outside the rows: it stays)."""
        _here(parents, holder=self)
        freeze_pages_fork(self.pool, parents)

    def truncate(self, keep: torch.Tensor) -> None:
        """Row r keeps its first keep[r] tokens (below 0: all); 0 frees it."""
        _here(keep, holder=self)
        freeze_pages_truncate(self.pool, keep)

    def compact(self) -> torch.Tensor:
        """The pages in use move together at the front; returns how many they are, [1]."""
        _here(holder=self)
        used = torch.empty(1, dtype=torch.int32, device=self.device)
        freeze_pages_compact(self.pool, used, self._workspace(self._book_bytes))
        return used

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None, most: int = 0,
               granted: Optional[torch.Tensor] = None) -> None:
        """The rows' newest tokens' keys and values [tokens, heads, head_dim] into a layer's pages: row r's are tokens starts[r] .. starts[r + 1] - 1
        (None: one token a row).  granted: as reserve returned it, rows that got another number of tokens are not written."""
        dev, pool = _here(k, v, starts, granted, holder=self), self.pool
        if k.shape != v.shape or k.dtype != v.dtype:
            raise _refused()
        ks, vs = _heads_of(k, pool.heads, pool.head_dim), _heads_of(v, pool.heads, pool.head_dim)
        _numbers(starts, pool.rows + 1)
        _numbers(granted, pool.rows)
        _check(lib().freeze_pages_append(self._at, layer, k.data_ptr(), *ks, v.data_ptr(), *vs, _DTYPES[k.dtype], k.shape[0], _at(starts), most, _at(granted),
                                         torch._C._cuda_getCurrentRawStream(dev)), "freeze_pages_append")

    def attend(self, layer: int, q: torch.Tensor, starts: Optional[torch.Tensor] = None, most: int = 0, scale: Optional[float] = None, window: int = 0,
               out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the rows' newest tokens, q [tokens, heads * group, head_dim], over a layer's pages; scale: head_dim ** -0.5 by default.  Outputs of
        tokens of no row are left as they are (in a new tensor: whatever they were).  A row that reserve granted nothing attends from its last old places: its
        outputs are no answer to a new token."""
        dev, pool = _here(q, starts, out, holder=self), self.pool
        dim = pool.head_dim
        qs = _heads_of(q, None, dim)
        tokens, heads, _ = shape = q.shape
        if out is None:
            out = torch.empty_like(q, dtype=out_dtype) if out_dtype else torch.empty_like(q)
        os_ = _heads_of(out, None, dim)
        if shape != out.shape or heads == 0 or heads % pool.heads != 0:
            raise _refused()
        _numbers(starts, pool.rows + 1)
        L, group = lib(), heads // pool.heads
        sizes = (group, tokens, most, starts is not None)
        nbytes = self._attend_bytes.get(sizes)
        if nbytes is None:
            nbytes = L.freeze_pages_attend_workspace_bytes(self._at, *sizes)
            if nbytes == 0:
                raise FreezeError(FREEZE_EINVAL, "freeze_pages_attend_workspace_bytes")
            if len(self._attend_bytes) >= 256:
                self._attend_bytes.clear()
            self._attend_bytes[sizes] = nbytes
        stream = torch._C._cuda_getCurrentRawStream(dev)
        ws = self._workspace(nbytes, (dev, stream))
        _check(L.freeze_pages_attend(self._at, layer, q.data_ptr(), _DTYPES[q.dtype], *qs, group, tokens, _at(starts), most, dim ** -0.5 if scale is None else scale,
                                     window, out.data_ptr(), _DTYPES[out.dtype], *os_, ws.data_ptr(), ws.numel(), stream), "freeze_pages_attend")
        return out
