"""Thin binding of libsepattn.so: argument marshalling only.

Each function has the name and the semantics of the C entry point declared in include/sepattn.h and
takes torch tensors that already live on the GPU (torch is used for device memory and streams,
nothing else).  Workspaces are allocated with torch and handed to the library, which never
allocates.  Every step of the computation runs in the library's HIP kernels; if the library is
missing this module raises at load time: there is no fallback.

The calls that enqueue work go through the extension module `_native` (csrc/native_binding.cpp), which
checks the tensors, allocates what the caller did not pass and calls the library: in Python those steps
took longer than a small kernel.  `load()` gives the library itself through ctypes, for the queries, the
measurement hooks and callers of the C interface.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# SEPATTN_LIB names another build of the same library (the host-sanitizer build that a CPU test runs the
# argument-validation tests against); every build runs the same kernels
LIB_PATH = os.environ.get("SEPATTN_LIB") or os.path.join(_HERE, "libsepattn.so")

SEPATTN_BF16 = 0
SEPATTN_FP32 = 1

EXPORTS = (
    "sepattn_status_string",
    "sepattn_mark_separators",
    "sepattn_mark_interval",
    "sepattn_compact_workspace_bytes",
    "sepattn_compact_indices",
    "sepattn_compact_indices_filled",
    "sepattn_mark_compact",
    "sepattn_mark_compact_filled",
    "sepattn_forward_workspace_bytes",
    "sepattn_forward",
    "sepattn_forward_headwise",
    "sepattn_backward_headwise_workspace_bytes",
    "sepattn_backward_headwise",
    "sepattn_doc_bounds",
    "sepattn_forward_packed",
    "sepattn_backward_packed",
    "sepattn_backward_workspace_bytes",
    "sepattn_backward",
    "sepattn_decode_workspace_bytes",
    "sepattn_decode",
    "sepattn_decode_noalloc_scratch_bytes",
    "sepattn_decode_noalloc",
    "sepkv_evict_workspace_bytes",
    "sepkv_evict_window",
    "sepkv_fill_from_prefill",
    "sepkv_fill_from_prefill_zeroed",
    "sepkv_rope_table",
    "sepattn_decode_rope",
    "sepkv_append",
    "sepattn_rope_frequencies",
    "sepattn_rope",
    "sepattn_rope_backward",
    "sepkv_rope_table_frequencies",
    "sepkv_append_rope",
    "sepkv_group_sequences",
    "sepkv_rope_cache",
    "sepattn_decode_shared_workspace_bytes",
    "sepattn_decode_shared",
    "sepattn_decode_shared_rope",
    "sepattn_norm_rope",
    "sepattn_norm_rope_backward_workspace_bytes",
    "sepattn_norm_rope_backward",
    "sepkv_append_norm_rope",
    "sepkv_fill_from_prefill_mx",
    "sepkv_fill_from_prefill_mx_zeroed",
    "sepkv_append_mx",
    "sepkv_append_rope_mx",
    "sepkv_append_norm_rope_mx",
    "sepkv_evict_window_mx",
    "sepkv_expand_mx",
    "sepattn_decode_mx_workspace_bytes",
    "sepattn_decode_mx",
    "sepattn_decode_rope_mx",
    "sepattn_kernel_name",
    "sepattn_profile_create",
    "sepattn_profile_attach",
    "sepattn_profile_detach",
    "sepattn_profile_read",
    "sepattn_profile_destroy",
)


class SepattnParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int), ("L", ctypes.c_int),
                ("d", ctypes.c_int), ("a", ctypes.c_int), ("n", ctypes.c_int), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("cap", ctypes.c_int)]


class SepkvParams(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int), ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int), ("d", ctypes.c_int),
                ("a", ctypes.c_int), ("s", ctypes.c_int), ("w", ctypes.c_int), ("c", ctypes.c_int),
                ("scale", ctypes.c_float), ("dtype", ctypes.c_int)]


class SepattnRopeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("B", "Hq", "Hkv", "L", "d", "rotary_dim", "interleaved", "dtype")]


class SepattnNormRopeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("B", "Hq", "Hkv", "L", "d", "rotary_dim", "interleaved", "dtype", "weight_dtype")] + [("eps", ctypes.c_float)]


class SepattnStrides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("b", "h", "l")]


class SepattnError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: status {status} ({status_string(status)})")


_lib = None
_calls = None  # the extension module, once its calls are bound to _lib


def load(path: Optional[str] = None):
    """Load the shared library (once).  Raises if it has not been built."""
    global _lib, _calls
    if _lib is not None and path is None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2412_12094_amd.build` (hipcc, gfx950)")
    lib = ctypes.CDLL(path)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.sepattn_status_string.restype = ctypes.c_char_p
    lib.sepattn_status_string.argtypes = [ci]
    lib.sepattn_mark_separators.restype = ci
    lib.sepattn_mark_separators.argtypes = [vp, ci, ci, vp, ci, vp, vp]
    lib.sepattn_mark_interval.restype = ci
    lib.sepattn_mark_interval.argtypes = [ci, ci, ci, ci, vp, vp]
    lib.sepattn_compact_workspace_bytes.restype = sz
    lib.sepattn_compact_workspace_bytes.argtypes = [ci, ci]
    lib.sepattn_compact_indices.restype = ci
    lib.sepattn_compact_indices.argtypes = [vp, ci, ci, vp, ci, vp, vp, vp, sz, vp]
    lib.sepattn_compact_indices_filled.restype = ci
    lib.sepattn_compact_indices_filled.argtypes = [vp, ci, ci, vp, ci, vp, vp, ctypes.c_int32, vp, sz, vp]
    lib.sepattn_mark_compact.restype = ci
    lib.sepattn_mark_compact.argtypes = [vp, ci, ci, vp, ci, vp, vp, ci, vp, vp, vp, sz, vp]
    lib.sepattn_mark_compact_filled.restype = ci
    lib.sepattn_mark_compact_filled.argtypes = [vp, ci, ci, vp, ci, vp, vp, ci, vp, vp, ctypes.c_int32, vp, sz, vp]
    pp = ctypes.POINTER(SepattnParams)
    lib.sepattn_forward_workspace_bytes.restype = sz
    lib.sepattn_forward_workspace_bytes.argtypes = [pp]
    lib.sepattn_forward.restype = ci
    lib.sepattn_forward.argtypes = [pp] + [vp] * 9 + [sz, vp]
    lib.sepattn_forward_headwise.restype = ci
    lib.sepattn_forward_headwise.argtypes = [pp] + [vp] * 10 + [sz, vp]
    lib.sepattn_backward_headwise_workspace_bytes.restype = sz
    lib.sepattn_backward_headwise_workspace_bytes.argtypes = [pp, vp]
    lib.sepattn_backward_headwise.restype = ci
    lib.sepattn_backward_headwise.argtypes = [pp] + [vp] * 14 + [sz, vp]
    lib.sepattn_doc_bounds.restype = ci
    lib.sepattn_doc_bounds.argtypes = [vp, ci, ci, ci, vp, vp, vp, vp]
    lib.sepattn_forward_packed.restype = ci
    lib.sepattn_forward_packed.argtypes = [pp] + [vp] * 11 + [sz, vp]
    lib.sepattn_backward_packed.restype = ci
    lib.sepattn_backward_packed.argtypes = [pp] + [vp] * 15 + [sz, vp]
    lib.sepattn_backward_workspace_bytes.restype = sz
    lib.sepattn_backward_workspace_bytes.argtypes = [pp]
    lib.sepattn_backward.restype = ci
    lib.sepattn_backward.argtypes = [pp] + [vp] * 13 + [sz, vp]
    kp = ctypes.POINTER(SepkvParams)
    lib.sepattn_decode_workspace_bytes.restype = sz
    lib.sepattn_decode_workspace_bytes.argtypes = [kp]
    lib.sepattn_decode.restype = ci
    lib.sepattn_decode.argtypes = [kp] + [vp] * 7 + [sz, vp]
    lib.sepattn_decode_noalloc_scratch_bytes.restype = sz
    lib.sepattn_decode_noalloc_scratch_bytes.argtypes = [kp]
    lib.sepattn_decode_noalloc.restype = ci
    lib.sepattn_decode_noalloc.argtypes = [kp] + [vp] * 7
    lib.sepkv_evict_workspace_bytes.restype = sz
    lib.sepkv_evict_workspace_bytes.argtypes = [kp]
    lib.sepkv_evict_window.restype = ci
    lib.sepkv_evict_window.argtypes = [kp] + [vp] * 5 + [sz, vp]
    lib.sepkv_fill_from_prefill.restype = ci
    lib.sepkv_fill_from_prefill.argtypes = [kp, ci, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp]
    lib.sepkv_fill_from_prefill_zeroed.restype = ci
    lib.sepkv_fill_from_prefill_zeroed.argtypes = [kp, ci, ci, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp]
    lib.sepkv_rope_table.restype = ci
    lib.sepkv_rope_table.argtypes = [ci, ci, ctypes.c_double, vp, vp]
    lib.sepattn_decode_rope.restype = ci
    lib.sepattn_decode_rope.argtypes = [kp, vp, vp, vp, vp, vp, ci, vp, vp, vp, sz, vp]
    lib.sepkv_append.restype = ci
    lib.sepkv_append.argtypes = [kp] + [vp] * 8
    cd, rp = ctypes.c_double, ctypes.POINTER(SepattnRopeParams)
    lib.sepattn_rope_frequencies.restype = ci
    lib.sepattn_rope_frequencies.argtypes = [ci, cd, cd, cd, cd, ci, vp]
    for name in ("sepattn_rope", "sepattn_rope_backward"):
        getattr(lib, name).restype = ci
        getattr(lib, name).argtypes = [rp, vp, vp, vp] + [vp, ctypes.POINTER(SepattnStrides)] * 6 + [vp]
    lib.sepkv_rope_table_frequencies.restype = ci
    lib.sepkv_rope_table_frequencies.argtypes = [ci, ci, vp, vp, vp]
    lib.sepkv_append_rope.restype = ci
    lib.sepkv_append_rope.argtypes = [kp, ci, ci] + [vp] * 12
    lib.sepkv_group_sequences.restype = ci
    lib.sepkv_group_sequences.argtypes = [vp, ci, ci, vp, vp, vp]
    lib.sepkv_rope_cache.restype = ci
    lib.sepkv_rope_cache.argtypes = [kp, vp, vp, ci, vp, vp, vp]
    lib.sepattn_decode_shared_workspace_bytes.restype = sz
    lib.sepattn_decode_shared_workspace_bytes.argtypes = [kp, kp]
    lib.sepattn_decode_shared.restype = ci
    lib.sepattn_decode_shared.argtypes = [kp, kp] + [vp] * 13 + [sz, vp]
    lib.sepattn_decode_shared_rope.restype = ci
    lib.sepattn_decode_shared_rope.argtypes = [kp, kp] + [vp] * 11 + [ci, vp, vp, vp, sz, vp]
    np_, strided = ctypes.POINTER(SepattnNormRopeParams), [vp, ctypes.POINTER(SepattnStrides)]
    lib.sepattn_norm_rope.restype = ci
    lib.sepattn_norm_rope.argtypes = [np_] + [vp] * 5 + strided * 6 + [vp]
    lib.sepattn_norm_rope_backward_workspace_bytes.restype = sz
    lib.sepattn_norm_rope_backward_workspace_bytes.argtypes = [np_]
    lib.sepattn_norm_rope_backward.restype = ci
    lib.sepattn_norm_rope_backward.argtypes = [np_] + [vp] * 5 + strided * 8 + [vp, vp, vp, sz, vp]
    norm = [kp, ci, ci, ctypes.c_float, ci, vp, vp]  # params, rotary_dim, interleaved, eps, weight_dtype, weights
    lib.sepkv_append_norm_rope.restype = ci
    lib.sepkv_append_norm_rope.argtypes = norm + [vp] * 12
    lib.sepkv_append_mx.restype = ci
    lib.sepkv_append_mx.argtypes = [kp] + [vp] * 10
    lib.sepkv_append_rope_mx.restype = ci
    lib.sepkv_append_rope_mx.argtypes = [kp, ci, ci] + [vp] * 14
    lib.sepkv_append_norm_rope_mx.restype = ci
    lib.sepkv_append_norm_rope_mx.argtypes = norm + [vp] * 14
    for name in ("sepkv_fill_from_prefill_mx", "sepkv_fill_from_prefill_mx_zeroed"):
        getattr(lib, name).restype = ci
        getattr(lib, name).argtypes = [kp, ci, ci, vp, vp, vp, vp, ci] + [vp] * 8
    lib.sepkv_evict_window_mx.restype = ci
    lib.sepkv_evict_window_mx.argtypes = [kp] + [vp] * 7
    lib.sepkv_expand_mx.restype = ci
    lib.sepkv_expand_mx.argtypes = [kp] + [vp] * 8
    lib.sepattn_decode_mx_workspace_bytes.restype = sz
    lib.sepattn_decode_mx_workspace_bytes.argtypes = [kp]
    lib.sepattn_decode_mx.restype = ci
    lib.sepattn_decode_mx.argtypes = [kp] + [vp] * 9 + [sz, vp]
    lib.sepattn_decode_rope_mx.restype = ci
    lib.sepattn_decode_rope_mx.argtypes = [kp] + [vp] * 7 + [ci, vp, vp, vp, sz, vp]
    lib.sepattn_kernel_name.restype = ctypes.c_char_p
    lib.sepattn_kernel_name.argtypes = [ci]
    lib.sepattn_profile_create.restype = ci
    lib.sepattn_profile_create.argtypes = [ci, ci, ctypes.POINTER(vp)]
    lib.sepattn_profile_attach.restype = ci
    lib.sepattn_profile_attach.argtypes = [vp]
    lib.sepattn_profile_detach.restype = ci
    lib.sepattn_profile_detach.argtypes = [vp]
    lib.sepattn_profile_read.restype = ci
    lib.sepattn_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ci, ctypes.POINTER(ctypes.c_int)]
    lib.sepattn_profile_destroy.restype = None
    lib.sepattn_profile_destroy.argtypes = [vp]
    if path == LIB_PATH or _lib is None:
        _lib = lib
        _calls = None
    return lib


def _native():
    """The extension module, its calls bound to the library that load() gives (once)."""
    global _calls
    calls = _calls
    if calls is None:
        lib = load()
        from . import _native as calls

        calls.bind(lib._name, _raise_status)
        _calls = calls
    return calls


def status_string(status: int) -> str:
    return load().sepattn_status_string(int(status)).decode()


KERNEL_IDS = {"mark": 0, "compact_count": 1, "compact_write": 2, "forward": 3, "bwd_dq": 4, "bwd_dkv": 5,
              "bwd_combine": 6, "decode_split": 7, "decode_merge": 8, "evict_sizes": 9, "evict_move": 10,
              "cache_fill": 11, "rope_table": 12, "cache_append": 13,
              "mark_interval": 14, "doc_bounds": 15, "mark_compact": 16}


def sepattn_kernel_name(kernel: int) -> str:
    return load().sepattn_kernel_name(int(kernel)).decode()


def sepattn_profile_begin(kernel: int, max_records: int):
    """Create a measurement handle for one kernel and attach it to this thread: the thread's next launches
    of that kernel are bracketed with HIP events on the launch stream.  Returns the handle."""
    lib = load()
    h = ctypes.c_void_p()
    _check("sepattn_profile_create", lib.sepattn_profile_create(int(kernel), int(max_records), ctypes.byref(h)))
    rc = lib.sepattn_profile_attach(h)
    if rc != 0:
        lib.sepattn_profile_destroy(h)
        raise SepattnError("sepattn_profile_attach", rc)
    return (h, int(max_records))


def sepattn_profile_end(handle):
    """Detach the handle, wait for the recorded events, free it; returns the per-launch durations in
    milliseconds."""
    lib = load()
    h, max_records = handle
    ms = (ctypes.c_float * max_records)()
    n = ctypes.c_int(0)
    rc = lib.sepattn_profile_detach(h)
    rc = rc or lib.sepattn_profile_read(h, ms, max_records, ctypes.byref(n))
    lib.sepattn_profile_destroy(h)
    _check("sepattn_profile_end", rc)
    return [float(ms[i]) for i in range(n.value)]


def _check(fn: str, rc: int) -> None:
    if rc != 0:
        raise SepattnError(fn, rc)


def _raise_status(fn: str, rc: int) -> None:
    raise SepattnError(fn, rc)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(t: torch.Tensor):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return SEPATTN_BF16
    if t.dtype == torch.float32:
        return SEPATTN_FP32
    raise TypeError(f"unsupported dtype {t.dtype}: bf16 or fp32 expected")


def _dev(*ts: torch.Tensor) -> None:
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("libsepattn works on GPU tensors only")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


# ------------------------------------------------------------------------------------------------
def sepattn_mark_separators(token_ids: torch.Tensor, sep_ids, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """token_ids int32 [B,L] (GPU), sep_ids: host sequence of ints -> is_sep uint8 [B,L]."""
    return _native().mark_separators(token_ids, sep_ids, out)


def sepattn_mark_interval(B: int, L: int, delta: int, phase: int, device, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> is_sep uint8 [B,L] with is_sep[b, j] = (j % delta == phase): the fixed-interval variant's markers."""
    if out is None:
        out = torch.empty((int(B), int(L)), dtype=torch.uint8, device=device)
    _dev(out)
    _check("sepattn_mark_interval",
           load().sepattn_mark_interval(int(B), int(L), int(delta), int(phase), _ptr(out), _stream(out)))
    return out


def sepattn_compact_indices(is_sep: torch.Tensor, cap: Optional[int] = None, want_prefix: bool = True,
                            fill: int = -1, out=None, ws: Optional[torch.Tensor] = None
                            ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """is_sep uint8 [B,L] -> (sep_idx int32 [B,cap], sep_count int32 [B], sep_prefix int32 [B,L+1]).

    Unless `out` = (sep_idx, sep_count, sep_prefix) is given, sep_idx is allocated and pre-filled
    with `fill` by torch; the library leaves entries beyond the count untouched.
    """
    return _native().compact_indices(is_sep, cap, want_prefix, fill, out, ws)


def sepattn_mark_compact(token_ids: torch.Tensor, sep_ids, cap: Optional[int] = None, want_prefix: bool = True,
                         fill: int = -1, out=None, ws: Optional[torch.Tensor] = None):
    """token_ids int32 [B,L] (GPU), sep_ids: host sequence of ints -> (is_sep uint8 [B,L], sep_idx int32 [B,cap],
    sep_count int32 [B], sep_prefix int32 [B,L+1]): marking and compaction in one call.

    Unless `out` = (is_sep, sep_idx, sep_count, sep_prefix) is given, the outputs are allocated and sep_idx is
    pre-filled with `fill` by torch; the library leaves entries beyond the count untouched.
    """
    return _native().mark_compact(token_ids, sep_ids, cap, want_prefix, fill, out, ws)


def _attn_params(Q, K, a, n, scale, cap) -> SepattnParams:
    B, Hq, L, d = Q.shape
    Hkv = K.shape[1]
    return SepattnParams(B, Hq, Hkv, L, d, int(a), int(n), float(scale), _dtype_code(Q), int(cap))


def sepattn_forward(Q, K, V, sep_idx, sep_count, sep_prefix, a: int, n: int, scale: float,
                    out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """Q [B,Hq,L,d], K,V [B,Hkv,L,d] -> (O like Q, LSE fp32 [B,Hq,L])."""
    return _native().forward(Q, K, V, sep_idx, sep_count, sep_prefix, a, n, scale, out, ws)


def sepattn_forward_headwise(Q, K, V, sep_idx, sep_count, sep_prefix, a: int, n_per_head, scale: float,
                             out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """sepattn_forward with a neighbour window of its own for every query head (n_per_head: Hq ints, host)."""
    return _native().forward_headwise(Q, K, V, sep_idx, sep_count, sep_prefix, a, n_per_head, scale, out, ws)


def sepattn_backward_headwise(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, a: int, n_per_head, scale: float,
                              out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                              ws: Optional[torch.Tensor] = None):
    """sepattn_backward with per-head neighbour windows -> (dQ, dK, dV)."""
    return _native().backward_headwise(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, a, n_per_head, scale, out, ws)


def sepattn_doc_bounds(cu_seqlens: torch.Tensor, L: int, a: int = 0, is_sep_row: Optional[torch.Tensor] = None,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
    """One packed row: cu_seqlens int32 [n_docs+1] (GPU; cu[0] = 0, cu[-1] = L) -> (doc_start, doc_end) int32 [L].
    If is_sep_row (uint8 [L], one row of the marker bitmap) is given, the first a tokens of every
    document are marked in it, in place."""
    return _native().doc_bounds(cu_seqlens, L, a, is_sep_row, out)


def sepattn_forward_packed(Q, K, V, doc_start, doc_end, sep_idx, sep_count, sep_prefix, n: int, scale: float,
                           out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """Forward over rows of packed documents: doc_start, doc_end int32 [B,L] per-position bounds;
    the index arrays come from a bitmap in which every document's initial tokens are marked (a = 0 here)."""
    return _native().forward_packed(Q, K, V, sep_idx, sep_count, sep_prefix, 0, n, scale, out, ws, doc_start, doc_end)


def sepattn_backward_workspace_bytes(Q, K, a: int, n: int, scale: float, cap: int) -> int:
    p = _attn_params(Q, K, a, n, scale, cap)
    return int(load().sepattn_backward_workspace_bytes(ctypes.byref(p)))


def sepattn_backward(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, a: int, n: int, scale: float,
                     out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                     ws: Optional[torch.Tensor] = None):
    """-> (dQ like Q, dK like K, dV like V)."""
    return _native().backward(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, a, n, scale, out, ws)


def sepattn_backward_packed(Q, K, V, O, LSE, dO, doc_start, doc_end, sep_idx, sep_count, sep_prefix, n: int,
                            scale: float, out=None, ws: Optional[torch.Tensor] = None):
    """Backward over rows of packed documents -> (dQ, dK, dV); arguments as sepattn_forward_packed."""
    return _native().backward_packed(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, 0, n, scale, out, ws, doc_start, doc_end)


def _kv_params(q, Kc, a, s, w, scale) -> SepkvParams:
    S, Hq, d = q.shape
    _, Hkv, c, _ = Kc.shape
    return SepkvParams(S, Hq, Hkv, d, int(a), int(s), int(w), c, float(scale), _dtype_code(Kc))


def sepattn_decode(q, Kc, Vc, sizes, a: int, s: int, w: int, scale: float,
                   out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """q [S,Hq,d], Kc,Vc [S,Hkv,c,d], sizes int32 [S,6] -> (out [S,Hq,d], lse fp32 [S,Hq])."""
    return _native().decode(q, Kc, Vc, sizes, None, a, s, w, scale, out, ws)


def sepattn_decode_noalloc(q, Kc, Vc, sizes, a: int, s: int, w: int, scale: float,
                           out: Tuple[torch.Tensor, torch.Tensor]):
    """sepattn_decode without a workspace (the library's fixed scratch array is used); the caller passes
    the outputs (out [S,Hq,d], lse fp32 [S,Hq]), so nothing at all is allocated by the call."""
    return _native().decode_noalloc(q, Kc, Vc, sizes, None, a, s, w, scale, out, None)


def sepkv_rope_table(n_pos: int, d: int, base: float, device, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> fp32 [n_pos, 2, d/2]: cos, then sin, of position * base^(-2i/d)."""
    if out is None:
        out = torch.empty((int(n_pos), 2, int(d) // 2), dtype=torch.float32, device=device)
    _dev(out)
    _check("sepkv_rope_table", load().sepkv_rope_table(int(n_pos), int(d), float(base), _ptr(out), _stream(out)))
    return out


def sepattn_decode_rope(q, Kc, Vc, sizes, rope_table, a: int, s: int, w: int, scale: float,
                        out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, ws: Optional[torch.Tensor] = None):
    """As sepattn_decode, with q and the cached keys stored without position encoding and turned by
    their positions within the cache inside the kernel; rope_table from sepkv_rope_table."""
    return _native().decode_rope(q, Kc, Vc, sizes, rope_table, a, s, w, scale, out, ws)


def sepkv_append(k_new, v_new, is_sep_new, Kc, Vc, win_is_sep, sizes, Hq: int, a: int, s: int, w: int) -> None:
    """In place: k_new, v_new [S,Hkv,d] and is_sep_new uint8 [S] enter Kc, Vc [S,Hkv,c,d], win_is_sep, sizes."""
    _native().append(k_new, v_new, is_sep_new, Kc, Vc, win_is_sep, sizes, Hq, a, s, w)


def sepkv_evict_window(Kc, Vc, win_is_sep, sizes, Hq: int, a: int, s: int, w: int,
                       ws: Optional[torch.Tensor] = None) -> None:
    """In place on Kc, Vc [S,Hkv,c,d], win_is_sep uint8 [S,c-a-s], sizes int32 [S,6]."""
    _native().evict_window(Kc, Vc, win_is_sep, sizes, Hq, a, s, w, ws)


def sepkv_fill_from_prefill(K, V, is_sep, sep_idx, sep_prefix, Hq: int, a: int, s: int, w: int, c: int, nw: int,
                            out=None):
    """Prefill K, V [S,Hkv,L,d] -> (Kc, Vc [S,Hkv,c,d], win_is_sep uint8 [S,c-a-s], sizes int32 [S,6]).
    Freshly allocated outputs are zero-filled (the call leaves slots beyond the sizes untouched)."""
    return _native().fill_from_prefill(K, V, is_sep, sep_idx, sep_prefix, Hq, a, s, w, c, nw, out)


# ---- rotary positions in front of the attention --------------------------------------------------
def sepattn_rope_frequencies(rotary_dim: int, base: float, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                             original_length: int = 0, device="cpu") -> torch.Tensor:
    """-> float64 [rotary_dim/2], radians per position: base^(-2p/rotary_dim), for contexts longer than the trained one
    divided by `factor` (all, or with original_length > 0 the pairs that make fewer than `low` turns in it, blended up to `high`).
    The calls take it on the GPU."""
    rotary_dim, original_length = int(rotary_dim), int(original_length)
    if not all(-2 ** 31 <= x < 2 ** 31 for x in (rotary_dim, original_length)):
        raise OverflowError("argument does not fit 32 bits")
    f = torch.empty(max(1, rotary_dim // 2), dtype=torch.float64)
    _check("sepattn_rope_frequencies", load().sepattn_rope_frequencies(
        rotary_dim, float(base), float(factor), float(low), float(high), original_length, _ptr(f)))
    return f.to(device)


def sepattn_rope(q, k, v, freqs, positions: Optional[torch.Tensor] = None, doc_start: Optional[torch.Tensor] = None,
                 interleaved: bool = False, out=None):
    """q [B,Hq,L,d], k, v [B,Hkv,L,d] with any strides (views of what the projections put out) -> (Q, K, V) dense, Q and K turned
    by the tokens' positions: `positions` int32 [B,L], else the index in the row, minus doc_start int32 [B,L] if given.  freqs float64
    [rotary_dim/2] (GPU).  v may be None, then V is.  `out`: three tensors of the same shapes, any strides."""
    return _native().rope(q, k, v, freqs, positions, doc_start, interleaved, out)


def sepattn_rope_backward(dQ, dK, dV, freqs, positions: Optional[torch.Tensor] = None, doc_start: Optional[torch.Tensor] = None,
                          interleaved: bool = False, out=None):
    """Gradient of sepattn_rope: dQ [B,Hq,L,d], dK, dV [B,Hkv,L,d] -> (dq, dk, dv) of the same shapes.  Unless `out` is given (views
    of a projection's gradient), they are views of one buffer [B, L, Hq + 2 Hkv, d]."""
    return _native().rope_backward(dQ, dK, dV, freqs, positions, doc_start, interleaved, out)


def sepkv_rope_table_frequencies(n_pos: int, freqs: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sepkv_rope_table for frequencies of the caller's: freqs float64 [d/2] (GPU) -> fp32 [n_pos, 2, d/2]."""
    _dev(freqs)
    if freqs.dtype != torch.float64 or freqs.dim() != 1:
        raise TypeError("freqs: float64 [d/2]")
    d = 2 * freqs.numel()
    if out is None:
        out = torch.empty((int(n_pos), 2, d // 2), dtype=torch.float32, device=freqs.device)
    _dev(out)
    if out.dtype != torch.float32 or tuple(out.shape) != (int(n_pos), 2, d // 2) or out.device != freqs.device:
        raise ValueError("out: fp32 [n_pos, 2, d/2] on the device of freqs")
    with torch.cuda.device(out.device):
        _check("sepkv_rope_table_frequencies",
               load().sepkv_rope_table_frequencies(int(n_pos), d, _ptr(freqs), _ptr(out), _stream(out)))
    return out


def sepkv_append_rope(q, k_new, v_new, is_sep_new, positions, freqs, Kc, Vc, win_is_sep, sizes, a: int, s: int, w: int,
                      interleaved: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sepkv_append for a token that is not turned yet: q [S,Hq,d] turned by positions int32 [S] is returned, k_new, v_new [S,Hkv,d]
    enter Kc, Vc, win_is_sep, sizes in place, the key turned.  `out` may be q."""
    return _native().append_rope(q, k_new, v_new, is_sep_new, positions, freqs, Kc, Vc, win_is_sep, sizes, a, s, w, interleaved, out)


# ---- shared prompts ----------------------------------------------------------------------------------
def sepkv_group_sequences(prefix_of: torch.Tensor, n_prefixes: int, out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """prefix_of int32 [S] (anything outside 0 .. n_prefixes-1: none) -> (group_start int32 [n_prefixes+1], group_seq int32 [S])."""
    return _native().group_sequences(prefix_of, n_prefixes, out)


def sepkv_rope_cache(Kc, sizes, rope_table, a: int, s: int, w: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The keys of Kc [S,Hkv,c,d] turned by their positions within the cache, in place or into `out` (other slots as they are)."""
    return _native().rope_cache(Kc, sizes, rope_table, a, s, w, out)


def sepattn_decode_shared_workspace_bytes(q, Kc, a: int, s: int, w: int, Kp, prefix_a: int, prefix_s: int, prefix_w: int) -> int:
    return _native().decode_shared_workspace_bytes(q, Kc, a, s, w, Kp, prefix_a, prefix_s, prefix_w)


def sepattn_decode_shared(q, Kc, Vc, sizes, a: int, s: int, w: int, Kp, Vp, prefix_sizes, prefix_a: int, prefix_s: int, prefix_w: int,
                          prefix_of, group_start, group_seq, scale: float, out=None, ws: Optional[torch.Tensor] = None):
    """sepattn_decode behind shared prompts: Kp, Vp [G,Hkv,prefix_c,d] and prefix_sizes int32 [G,6] are the prefix caches, prefix_of
    int32 [S] says which one a sequence shares, group_start, group_seq come from sepkv_group_sequences
    -> (out [S,Hq,d], lse fp32 [S,Hq])."""
    return _native().decode_shared(q, Kc, Vc, sizes, a, s, w, Kp, Vp, prefix_sizes, prefix_a, prefix_s, prefix_w, prefix_of, group_start,
                                   group_seq, None, scale, out, ws)


def sepattn_decode_shared_rope(q, Kc, Vc, sizes, a: int, s: int, w: int, Kp, Vp, prefix_sizes, prefix_a: int, prefix_s: int,
                               prefix_w: int, prefix_of, group_start, group_seq, rope_table, scale: float, out=None,
                               ws: Optional[torch.Tensor] = None):
    """The same with positions within the caches, the prefix's first: Kp holds keys turned by sepkv_rope_cache, Kc and q are
    stored without encoding; rope_table with prefix_c + c rows or more."""
    return _native().decode_shared_rope(q, Kc, Vc, sizes, a, s, w, Kp, Vp, prefix_sizes, prefix_a, prefix_s, prefix_w, prefix_of,
                                        group_start, group_seq, rope_table, scale, out, ws)


# ---- norms of queries and keys in front of the rotary positions ------------------------------------
def sepattn_norm_rope(q, k, v, q_weight, k_weight, freqs, eps: float, positions: Optional[torch.Tensor] = None,
                      doc_start: Optional[torch.Tensor] = None, interleaved: bool = False, out=None):
    """sepattn_rope with the rows of q and k divided by their root mean square (eps added to the mean square) and multiplied by
    q_weight, k_weight [d] (bf16 or fp32, None: ones) first.  freqs None: normed only."""
    return _native().norm_rope(q, k, v, q_weight, k_weight, freqs, eps, positions, doc_start, interleaved, out)


def sepattn_norm_rope_backward_workspace_bytes(q, k, eps: float = 0.0, rotary_dim: int = 0) -> int:
    """Of a call with q [B,Hq,L,d], k [B,Hkv,L,d]; the largest over all positions and weights."""
    B, Hq, L, d = q.shape
    p = SepattnNormRopeParams(B, Hq, k.shape[1], L, d, int(rotary_dim), 0, _dtype_code(q), SEPATTN_FP32, float(eps))
    with torch.cuda.device(q.device):
        return int(load().sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(p)))


def sepattn_norm_rope_backward(q, k, dQ, dK, dV, q_weight, k_weight, freqs, eps: float, positions: Optional[torch.Tensor] = None,
                               doc_start: Optional[torch.Tensor] = None, interleaved: bool = False, out=None, out_weights=None,
                               ws: Optional[torch.Tensor] = None):
    """Gradient of sepattn_norm_rope, whose inputs q, k were: dQ [B,Hq,L,d], dK, dV [B,Hkv,L,d] (dV may be None)
    -> (dq, dk, dv, dq_weight, dk_weight), the last two fp32 [d].  Unless `out` = (dq, dk, dv) is given, these are views of one buffer
    [B, L, Hq + 2 Hkv, d].  out_weights: two tensors fp32 [d], None in the place of one that is not wanted."""
    return _native().norm_rope_backward(q, k, dQ, dK, dV, q_weight, k_weight, freqs, eps, positions, doc_start, interleaved, out, out_weights, ws)


def sepkv_append_norm_rope(q, k_new, v_new, is_sep_new, positions, q_weight, k_weight, freqs, eps: float, Kc, Vc, win_is_sep, sizes, a: int,
                           s: int, w: int, interleaved: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sepkv_append_rope for a token whose query and key are normed first (sepattn_norm_rope; freqs and positions may be None)."""
    return _native().append_norm_rope(q, k_new, v_new, is_sep_new, positions, q_weight, k_weight, freqs, eps, Kc, Vc, win_is_sep, sizes, a, s, w,
                                      interleaved, out)


# ---- the cache in 4 bits -----------------------------------------------------------------------------
# Kc, Vc uint8 [S,Hkv,c,d/2]: codes; Ks, Vs uint8 [S,Hkv,c,d/32]: scales
def sepkv_fill_from_prefill_mx(K, V, is_sep, sep_idx, sep_prefix, Hq: int, a: int, s: int, w: int, c: int, nw: int, out=None):
    """sepkv_fill_from_prefill with the rows rounded to 4 bits -> (Kc, Ks, Vc, Vs, win_is_sep, sizes).  Freshly allocated outputs hold
    zeros beyond the sizes (`out`: left untouched there)."""
    return _native().fill_from_prefill_fp4(K, V, is_sep, sep_idx, sep_prefix, Hq, a, s, w, c, nw, out)


def sepkv_append_mx(k_new, v_new, is_sep_new, Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq: int, a: int, s: int, w: int) -> None:
    """In place: k_new, v_new [S,Hkv,d], rounded to 4 bits, and is_sep_new uint8 [S] enter the cache."""
    _native().append_fp4(k_new, v_new, is_sep_new, Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq, a, s, w)


def sepkv_append_rope_mx(q, k_new, v_new, is_sep_new, positions, freqs, Kc, Ks, Vc, Vs, win_is_sep, sizes, a: int, s: int, w: int,
                          interleaved: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sepkv_append_rope into a cache in 4 bits."""
    return _native().append_rope_fp4(q, k_new, v_new, is_sep_new, positions, freqs, Kc, Ks, Vc, Vs, win_is_sep, sizes, a, s, w, interleaved, out)


def sepkv_append_norm_rope_mx(q, k_new, v_new, is_sep_new, positions, q_weight, k_weight, freqs, eps: float, Kc, Ks, Vc, Vs, win_is_sep,
                               sizes, a: int, s: int, w: int, interleaved: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """sepkv_append_norm_rope into a cache in 4 bits."""
    return _native().append_norm_rope_fp4(q, k_new, v_new, is_sep_new, positions, q_weight, k_weight, freqs, eps, Kc, Ks, Vc, Vs, win_is_sep, sizes,
                                          a, s, w, interleaved, out)


def sepkv_evict_window_mx(Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq: int, a: int, s: int, w: int) -> None:
    """sepkv_evict_window on a cache in 4 bits."""
    _native().evict_window_fp4(Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq, a, s, w)


def sepkv_expand_mx(Kc, Ks, Vc, Vs, sizes, a: int, s: int, w: int, dtype: torch.dtype = torch.bfloat16, out=None):
    """-> (K, V) [S,Hkv,c,d]: the values of the cache's valid entries, exact in bf16 and fp32, 0 in all other slots."""
    if out is None and dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("unsupported dtype: bf16 or fp32 expected")
    return _native().expand_fp4(Kc, Ks, Vc, Vs, sizes, a, s, w, dtype == torch.float32, out)


def sepattn_decode_mx_workspace_bytes(q, Kc, a: int, s: int, w: int) -> int:
    S, Hq, d = q.shape
    p = SepkvParams(S, Hq, Kc.shape[1], d, int(a), int(s), int(w), Kc.shape[2], 1.0, _dtype_code(q))
    with torch.cuda.device(q.device):
        return int(load().sepattn_decode_mx_workspace_bytes(ctypes.byref(p)))


def sepattn_decode_mx(q, Kc, Ks, Vc, Vs, sizes, a: int, s: int, w: int, scale: float, out=None, ws: Optional[torch.Tensor] = None):
    """sepattn_decode over the values of a cache in 4 bits: q [S,Hq,d] -> (out [S,Hq,d], lse fp32 [S,Hq])."""
    return _native().decode_fp4(q, Kc, Ks, Vc, Vs, sizes, None, a, s, w, scale, out, ws)


def sepattn_decode_rope_mx(q, Kc, Ks, Vc, Vs, sizes, rope_table, a: int, s: int, w: int, scale: float, out=None,
                            ws: Optional[torch.Tensor] = None):
    """The same with positions within the cache (sepattn_decode_rope): q and the cached keys are stored without encoding."""
    return _native().decode_rope_fp4(q, Kc, Ks, Vc, Vs, sizes, rope_table, a, s, w, scale, out, ws)
