"""Binding of libsuffixspec.so: argument marshalling only (ctypes; the calls that a serving loop
makes every step go through the native module _call, see csrc/call.cpp).

Tensors are torch CUDA tensors used as plain device buffers; the stream is
torch's current stream.  The module-level functions sd_build / sd_append /
sd_speculate / sd_free mirror the C entry points one to one; `SuffixStore`
wraps them with output allocation.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import math
import os
import subprocess
import warnings
from typing import Dict, Optional

import torch

from . import build as _build

FLAG_GLOBAL_ONLY, FLAG_REQUEST_ONLY, FLAG_LINEAR = 1, 2, 4
STATUS_BAD_SLOT, STATUS_POOL_FULL, STATUS_GLOBAL_FULL, STATUS_BAD_TOKEN = 1, 2, 4, 8
STATUS_BAD_ROWS, STATUS_BAD_PAGE, STATUS_FAILED = 16, 32, 64

EXPORTS = ["sd_build", "sd_build_requests", "sd_append", "sd_speculate", "sd_step", "sd_speculate_noalloc", "sd_query_counts",
           "sd_enumerate", "sd_slot_info", "sd_entropy", "sd_stats", "sd_free", "sd_trim", "sd_strerror", "sd_debug_fail_alloc",
           "sd_debug_small_clusters", "sd_debug_attend_limit", "sd_rotate", "sd_attend", "sd_attend_workspace", "sd_accept", "sd_commit"]


class SuffixSpecError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {library().sd_strerror(code).decode()} ({code})")


class _BuildParams(C.Structure):
    _fields_ = [("vocab", C.c_int32), ("depth_cap", C.c_int32), ("max_requests", C.c_int32),
                ("max_req_tokens", C.c_int32), ("max_spec_cap", C.c_int32), ("global_extra_nodes", C.c_int64),
                ("slot_pool_nodes", C.c_int64)]


class _SpecParams(C.Structure):
    _fields_ = [("P", C.c_int32), ("alpha", C.c_double), ("max_spec", C.c_int32), ("flags", C.c_uint32),
                ("tau", C.c_double)]


class _Stats(C.Structure):
    _fields_ = [("global_nodes", C.c_int64), ("global_pool_used", C.c_int64), ("global_pool_cap", C.c_int64),
                ("global_tokens", C.c_int64), ("slot_pool_nodes", C.c_int64), ("device_bytes", C.c_int64),
                ("global_status", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("dtype", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("k_stride", C.c_int64 * 4),
                ("v_stride", C.c_int64 * 4)]


class _Rows(C.Structure):
    _fields_ = [("n", C.c_int32), ("rows", C.c_int32), ("max_draft", C.c_int32), ("table_stride", C.c_int32), ("d_offsets", C.c_void_p),
                ("d_cached", C.c_void_p), ("d_table", C.c_void_p), ("d_mask", C.c_void_p), ("d_status", C.c_void_p)]


class _RotateParams(C.Structure):
    _fields_ = [("q_heads", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float), ("eps", C.c_float),
                ("q_stride", C.c_int64 * 2), ("k_stride", C.c_int64 * 2), ("v_stride", C.c_int64 * 2), ("out_stride", C.c_int64 * 2)]


class _AttendParams(C.Structure):
    _fields_ = [("q_heads", C.c_int32), ("scale", C.c_float), ("window", C.c_int32), ("sinks", C.c_int32), ("shared", C.c_int32),
                ("q_stride", C.c_int64 * 2), ("out_stride", C.c_int64 * 2)]


MAX_DRAFT = 64
_DTYPES = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}

_lib = None
_call = None               # the module of the per-step calls; loaded with the library


def library() -> C.CDLL:
    """Load libsuffixspec.so (building it with nvcc if the sources are newer).
    Raises if it cannot be had: there is no fallback path."""
    global _lib, _call
    if _lib is None:
        path = _build.LIB
        if not os.path.exists(path) or os.environ.get("SUFFIXSPEC_REBUILD"):
            path = _build.build()
        lib = C.CDLL(path)
        vp = C.c_void_p
        lib.sd_build.restype = C.c_int
        lib.sd_build.argtypes = [C.POINTER(_BuildParams), vp, vp, C.c_int32, vp, C.POINTER(vp)]
        lib.sd_build_requests.restype = C.c_int
        lib.sd_build_requests.argtypes = [vp, C.c_int32, vp, vp, vp, vp]
        lib.sd_append.restype = C.c_int
        lib.sd_append.argtypes = [vp, C.c_int32, vp, vp, vp, vp, vp]
        lib.sd_speculate.restype = C.c_int
        lib.sd_speculate.argtypes = [vp, C.c_int32, vp, C.POINTER(_SpecParams)] + [vp] * 11
        lib.sd_step.restype = C.c_int
        lib.sd_step.argtypes = [vp, C.c_int32, vp, vp, vp, C.POINTER(_SpecParams)] + [vp] * 11
        lib.sd_speculate_noalloc.restype = C.c_int
        lib.sd_speculate_noalloc.argtypes = lib.sd_speculate.argtypes
        lib.sd_query_counts.restype = C.c_int
        lib.sd_query_counts.argtypes = [vp, C.c_int32, vp, vp, vp, vp, vp]
        lib.sd_enumerate.restype = C.c_int
        lib.sd_enumerate.argtypes = [vp, C.c_int32, C.c_int64, vp, vp, vp, vp, C.POINTER(C.c_int64), vp]
        lib.sd_slot_info.restype = C.c_int
        lib.sd_slot_info.argtypes = [vp, C.c_int32, vp, vp, vp, vp, vp]
        lib.sd_entropy.restype = C.c_int
        lib.sd_entropy.argtypes = [vp, C.c_int32, C.POINTER(C.c_double), vp]
        lib.sd_stats.restype = C.c_int
        lib.sd_stats.argtypes = [vp, C.POINTER(_Stats), vp]
        lib.sd_free.restype = None
        lib.sd_free.argtypes = [vp]
        lib.sd_trim.restype = None
        lib.sd_trim.argtypes = []
        lib.sd_debug_fail_alloc.restype = None
        lib.sd_debug_fail_alloc.argtypes = [C.c_int64]
        lib.sd_debug_small_clusters.restype = None
        lib.sd_debug_small_clusters.argtypes = [C.c_int32]
        lib.sd_debug_attend_limit.restype = None
        lib.sd_debug_attend_limit.argtypes = [C.c_int64]
        cache, rows = C.POINTER(_Cache), C.POINTER(_Rows)
        lib.sd_rotate.restype = C.c_int
        lib.sd_rotate.argtypes = [cache, rows, C.POINTER(_RotateParams)] + [vp] * 9
        lib.sd_attend.restype = C.c_int
        lib.sd_attend.argtypes = [cache, rows, C.POINTER(_AttendParams), vp, vp, vp, vp, C.c_int64, vp]
        lib.sd_attend_workspace.restype = C.c_int64
        lib.sd_attend_workspace.argtypes = [cache, rows, C.POINTER(_AttendParams)]
        lib.sd_accept.restype = C.c_int
        lib.sd_accept.argtypes = [C.c_int32] * 5 + [C.c_int64] + [vp] * 10
        lib.sd_commit.restype = C.c_int
        lib.sd_commit.argtypes = [cache, rows, vp, vp, vp]
        lib.sd_strerror.restype = C.c_char_p
        lib.sd_strerror.argtypes = [C.c_int]
        _lib, _call = lib, _load_call(lib)
    return _lib


def _load_call(lib):
    """The native module of the per-step calls, built if this torch has none yet; if it cannot be had (no compiler), the
    same calls with their arguments converted here."""
    try:
        path = _build.call_path()
        if not os.path.exists(path):
            path = _build.build_call()
        spec = importlib.util.spec_from_file_location(__package__ + "._call", path)
        call = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(call)
        call.setup(*(C.cast(f, C.c_void_p).value for f in (lib.sd_speculate, lib.sd_step, lib.sd_append)), _ptr)
        call.setup_verifier(*(C.cast(f, C.c_void_p).value for f in (lib.sd_rotate, lib.sd_attend, lib.sd_attend_workspace,
                                                                    lib.sd_accept, lib.sd_commit)))
        return call
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"the native module of the per-step calls could not be had ({e}): each call takes the host some 6 us longer",
                      RuntimeWarning)
        return _PlainCall(lib)


class _PlainCall:
    """The calls of the module _call through ctypes."""

    def __init__(self, lib):
        self._lib = lib

    def speculate(self, store, slots, P, alpha, max_spec, flags, tau, budget_cap, out) -> int:
        return self._lib.sd_speculate(
            store, int(slots.numel()), _ptr(slots, torch.int32, "slots"), C.byref(_SpecParams(P, alpha, max_spec, flags, tau)),
            _ptr(budget_cap, torch.int32, "budget_cap"), *_out_ptrs(out), _stream())

    def step(self, store, slots, offsets, new_tokens, P, alpha, max_spec, flags, tau, budget_cap, out) -> int:
        return self._lib.sd_step(
            store, int(slots.numel()), _ptr(slots, torch.int32, "slots"), _ptr(offsets, torch.int64, "offsets"),
            _ptr(new_tokens, torch.int32, "new_tokens"), C.byref(_SpecParams(P, alpha, max_spec, flags, tau)),
            _ptr(budget_cap, torch.int32, "budget_cap"), *_out_ptrs(out), _stream())

    def append(self, store, slots, offsets, tokens, reset) -> int:
        return self._lib.sd_append(
            store, int(slots.numel()), _ptr(slots, torch.int32, "slots"), _ptr(offsets, torch.int64, "offsets"),
            _ptr(tokens, torch.int32, "tokens"), _ptr(reset, torch.uint8, "reset"), _stream())


    def rotate(self, q, k, v, k_cache, v_cache, table, offsets, cached, freq, mask, positions, q_weight, k_weight, eps, interleaved,
               scale, out, status):
        cache, dt = _cache_of(k_cache, v_cache, (4,)), k_cache.dtype
        rows = _length(q, "q")
        b = _rows_of(rows, table, offsets, cached, mask, status)
        heads, D = _q_heads(q), k_cache.shape[-1]
        if heads > 65536 or freq.numel() > 64:
            raise TypeError("rotate: at most 65,536 heads and 64 frequencies")
        out = torch.empty(q.shape, dtype=q.dtype, device=_device()) if out is None else out
        strides = [_heads(t, dt, (rows, h, D), name) for t, h, name in ((q, heads, "q"), (k, cache.kv_heads, "k"), (v, cache.kv_heads, "v"), (out, heads, "out"))]
        p = _RotateParams(heads, 2 * freq.numel(), int(interleaved), scale, eps, *strides)
        return self._lib.sd_rotate(
            C.byref(cache), C.byref(b), C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), _array(freq, torch.float64, (freq.numel(),), "freq"),
            _array(positions, torch.int32, (rows,), "positions"), _array(q_weight, dt, (D,), "q_weight"),
            _array(k_weight, dt, (D,), "k_weight"), out.data_ptr(), _stream()) or out

    def attend(self, q, k_cache, v_cache, table, offsets, cached, mask, scale, window, sinks, shared, out, lse, status):
        cache, dt = _cache_of(k_cache, v_cache, (4,)), k_cache.dtype
        rows = _length(q, "q")
        b = _rows_of(rows, table, offsets, cached, mask, status)
        heads, D = _q_heads(q), k_cache.shape[-1]
        for name, x in (("q_heads", heads), ("window", window), ("sinks", sinks), ("shared", shared)):
            if not 0 <= x <= (65536 if name == "q_heads" else 0x7FFFFFFF):
                raise SuffixSpecError(-1, f"sd_attend: {name} {x}")
        out = torch.empty(q.shape, dtype=q.dtype, device=_device()) if out is None else out
        scale = max(D, 1) ** -0.5 if scale is None else scale
        p = _AttendParams(heads, scale, window, sinks, shared, _heads(q, dt, (rows, heads, D), "q"), _heads(out, dt, (rows, heads, D), "out"))
        lse = _array(lse, torch.float32, (rows, heads), "lse")
        size = self._lib.sd_attend_workspace(C.byref(cache), C.byref(b), C.byref(p))
        if size < 0:
            return size
        work = torch.empty(size, dtype=torch.uint8, device=_device())
        return self._lib.sd_attend(C.byref(cache), C.byref(b), C.byref(p), q.data_ptr(), out.data_ptr(), lse, work.data_ptr(), size, _stream()) or out

    def accept(self, logits, offsets, tokens, parents, out, status):
        if logits.dim() != 2 or tokens.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise TypeError("accept: expected logits [rows, vocab] with adjacent entries and tokens [n, max_draft]")
        (rows, vocab), (n, M) = logits.shape, tokens.shape
        if logits.dtype not in _DTYPES or M > MAX_DRAFT or max(rows, vocab, n) > 0x7FFFFFFE:
            raise TypeError(f"accept: logits of {logits.dtype}, drafts of {M}")
        _here(logits, "logits")
        if out is None:
            i32 = dict(dtype=torch.int32, device=_device())
            out = {"targets": torch.empty(rows, **i32), "path": torch.empty(n, M + 1, **i32),
                   "offsets": torch.empty(n + 1, dtype=torch.int64, device=_device()), "tokens": torch.empty(rows, **i32)}
        targets, path, new_offsets, new_tokens = (out[k] for k in ("targets", "path", "offsets", "tokens"))
        args = [_array(t, dt, shape, name) for t, dt, shape, name in (
            (offsets, torch.int64, (n + 1,), "offsets"), (tokens, torch.int32, (n, M), "tokens"), (parents, torch.int32, (n, M), "parents"),
            (targets, torch.int32, (rows,), "targets"), (path, torch.int32, (n, M + 1), "path"), (new_offsets, torch.int64, (n + 1,), "new_offsets"),
            (new_tokens, torch.int32, (rows,), "new_tokens"), (status, torch.int32, (n,), "status"))]
        return self._lib.sd_accept(n, rows, M, vocab, _DTYPES[logits.dtype], logits.stride(0) if rows > 1 else vocab, logits.data_ptr(), *args, _stream()) or out

    def commit(self, k_cache, v_cache, table, cached, path, out, status):
        cache = _cache_of(k_cache, v_cache, (4, 5))
        if path.dim() != 2 or not 1 <= path.shape[1] <= MAX_DRAFT + 1 or table.dim() != 2:
            raise TypeError("commit: expected a path [n, max_draft + 1] and a table [n, pages]")
        n, M1 = path.shape
        _counts("path, table", n, table.shape[1])
        b = _Rows(n, 0, M1 - 1, table.shape[1], None, _array(cached, torch.int32, (n,), "cached"),
                  _array(table, torch.int32, (n, table.shape[1]), "table"), None, _array(status, torch.int32, (n,), "status"))
        out = torch.empty(cached.shape, dtype=cached.dtype, device=_device()) if out is None else out
        return self._lib.sd_commit(C.byref(cache), C.byref(b), _array(path, torch.int32, (n, M1), "path"),
                                   _array(out, torch.int32, (n,), "out"), _stream()) or out


def _device() -> torch.device:
    """Where results and workspaces are made: the arguments may be in pinned host memory."""
    return torch.device("cuda", _current_device())


def _here(t: torch.Tensor, name: str) -> None:
    if not (t.is_cuda and t.device.index == _current_device()) and not t.is_pinned():
        raise TypeError(f"{name}: expected a tensor on the current CUDA device (or in pinned host memory), got one on {t.device}")


def _array(t: Optional[torch.Tensor], dtype: torch.dtype, shape: tuple, name: str) -> Optional[int]:
    if t is not None and tuple(t.shape) != shape:
        raise TypeError(f"{name}: expected the shape {shape}, got {tuple(t.shape)}")
    p = _ptr(t, dtype, name)
    if t is not None:
        _here(t, name)
    return p


def _counts(name: str, *sizes: int) -> None:
    """Sizes that the structures hold in 31 bits (a larger one would go over as what is left of it)."""
    if max(sizes) > 0x7FFFFFFE:
        raise TypeError(f"{name}: a size of {max(sizes)} is beyond 31 bits")


def _length(t: torch.Tensor, name: str) -> int:
    if t.dim() < 1:
        raise TypeError(f"{name}: expected rows")
    return t.shape[0]


def _q_heads(q: torch.Tensor) -> int:
    if q.dim() != 3:
        raise TypeError(f"q: expected [rows, q_heads, head_dim], got {tuple(q.shape)}")
    return q.shape[1]


def _heads(t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str):
    """Strides of rows of heads whose elements are adjacent."""
    if t.dtype != dtype or tuple(t.shape) != shape or t.stride(2) != 1:
        raise TypeError(f"{name}: expected {dtype} of the shape {shape} with adjacent elements, got {t.dtype} {tuple(t.shape)}, strides {t.stride()}")
    _here(t, name)
    return (C.c_int64 * 2)(t.stride(0), t.stride(1))


def _cache_of(k: torch.Tensor, v: torch.Tensor, dims: tuple) -> _Cache:
    if k.dtype != v.dtype or k.dtype not in _DTYPES or k.shape != v.shape or k.dim() not in dims or k.stride(-1) != 1 or v.stride(-1) != 1:
        raise TypeError("k_cache, v_cache: expected two alike tensors [pages, page_size, kv_heads, head_dim] (sd_commit: or one per layer before "
                        f"that) with adjacent elements, got {k.dtype} {tuple(k.shape)} and {v.dtype} {tuple(v.shape)}")
    _here(k, "k_cache")
    _here(v, "v_cache")
    _counts("k_cache, v_cache", *k.shape)
    layers = k.dim() == 5
    st = [(C.c_int64 * 4)(t.stride(0) if layers else 0, t.stride(-4), t.stride(-3), t.stride(-2)) for t in (k, v)]
    return _Cache(k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], k.shape[-2], k.shape[-1], k.shape[0] if layers else 1, k.shape[-4], k.shape[-3], *st)


def _rows_of(rows: int, table, offsets, cached, mask, status) -> _Rows:
    n = _length(offsets, "offsets") - 1
    if n < 0 or table.dim() != 2:
        raise TypeError("offsets: expected one more than requests; table: expected [n, pages]")
    _counts("rows, offsets, table", rows, n, table.shape[1])
    M = MAX_DRAFT
    if mask is not None:
        if mask.dim() != 3 or mask.shape[1] > MAX_DRAFT:
            raise TypeError(f"mask: expected [n, max_draft <= {MAX_DRAFT}, words], got {tuple(mask.shape)}")
        M = mask.shape[1]
    return _Rows(n, rows, M, table.shape[1], _array(offsets, torch.int64, (n + 1,), "offsets"), _array(cached, torch.int32, (n,), "cached"),
                 _array(table, torch.int32, (n, table.shape[1]), "table"),
                 _array(mask, torch.int32, (n, M, (M + 31) // 32), "mask"), _array(status, torch.int32, (n,), "status"))


def _ptr(t: Optional[torch.Tensor], dtype: torch.dtype, name: str) -> Optional[int]:
    if t is None:
        return None
    # pinned host memory has a device address of its own (unified addressing): the kernels then
    # read or write it across the bus, with no copy before or after the call
    if not (t.is_cuda or t.is_pinned()) or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous CUDA (or pinned host) tensor of {dtype}, "
                        f"got {t.dtype} on {t.device}")
    return t.data_ptr()


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


_OUT_FIELDS = (("n_draft", torch.int32), ("tokens", torch.int32), ("parents", torch.int32), ("positions", torch.int32),
               ("mask", torch.int32), ("chosen_tree", torch.int32), ("chosen_p", torch.int32), ("score", torch.float64),
               ("status", torch.int32))


def _out_ptrs(out: Dict[str, torch.Tensor]) -> list:
    return [_ptr(out[name], dtype, name) for name, dtype in _OUT_FIELDS]


def _loaded():
    """The module of the per-step calls."""
    library()
    return _call


# ---- the C entry points, one to one ------------------------------------------------------
def sd_build(corpus: Optional[torch.Tensor], seq_offsets: Optional[torch.Tensor], *, vocab: int, depth_cap: int,
             max_requests: int, max_req_tokens: int, max_spec_cap: int, global_extra_nodes: int = -1,
             slot_pool_nodes: int = 0) -> int:
    """Returns the store handle (an integer address)."""
    p = _BuildParams(vocab, depth_cap, max_requests, max_req_tokens, max_spec_cap, global_extra_nodes,
                     slot_pool_nodes)
    n_seqs = 0 if seq_offsets is None else int(seq_offsets.numel()) - 1
    out = C.c_void_p()
    rc = library().sd_build(C.byref(p), _ptr(corpus, torch.int32, "corpus"),
                            _ptr(seq_offsets, torch.int64, "seq_offsets"), n_seqs, _stream(), C.byref(out))
    if rc != 0:
        raise SuffixSpecError(rc, "sd_build")
    return out.value


def sd_append(store: int, slots: torch.Tensor, offsets: torch.Tensor, tokens: torch.Tensor,
              reset: Optional[torch.Tensor] = None) -> None:
    rc = (_call or _loaded()).append(store, slots, offsets, tokens, reset)
    if rc != 0:
        raise SuffixSpecError(rc, "sd_append")


def sd_speculate(store: int, slots: torch.Tensor, P: int, alpha: float, max_spec: int, flags: int,
                 budget_cap: Optional[torch.Tensor], out: Dict[str, torch.Tensor], tau: float = 0.0) -> None:
    rc = (_call or _loaded()).speculate(store, slots, P, alpha, max_spec, flags, tau, budget_cap, out)
    if rc != 0:
        raise SuffixSpecError(rc, "sd_speculate")


def sd_speculate_noalloc(store: int, slots: torch.Tensor, P: int, alpha: float, max_spec: int, flags: int,
                         budget_cap: Optional[torch.Tensor], out: Dict[str, torch.Tensor], tau: float = 0.0) -> None:
    """sd_speculate for callers that may not allocate device memory: the scratch
    records live in a fixed array inside the library, so the batch is limited
    (n * 2 * depth_cap <= 4096 jobs) and calls on one device must not overlap.
    `out` must be preallocated by the caller; nothing is allocated here."""
    rc = library().sd_speculate_noalloc(
        store, slots.numel(), _ptr(slots, torch.int32, "slots"),
        C.byref(_SpecParams(P, alpha, max_spec, flags, tau)), _ptr(budget_cap, torch.int32, "budget_cap"), *_out_ptrs(out), _stream())
    if rc != 0:
        raise SuffixSpecError(rc, "sd_speculate_noalloc")


def _made(name: str, result, args: tuple):
    """What the native call gave; where one of its tensors was not usual (None), what the same call in Python gives.  Raises what a status says."""
    if result is None:
        result = getattr(_PlainCall(library()), name)(*args)
    if type(result) is int:
        raise SuffixSpecError(result, "sd_" + name)
    return result


def sd_rotate(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
              offsets: torch.Tensor, cached: torch.Tensor, freq: torch.Tensor, *, mask: Optional[torch.Tensor] = None,
              positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
              eps: float = 1e-6, interleaved: bool = False, scale: float = 1.0, out: Optional[torch.Tensor] = None,
              status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Queries q [rows, q_heads, head_dim], normed (where they have a weight) and turned to the rows' positions; keys likewise and values go to the
    rows' places in the cache [pages, page_size, kv_heads, head_dim].  freq: float64, radians per position of each pair (see
    rotary_frequencies); the first 2 * len(freq) elements of a head are turned.  offsets, cached, table, mask: the batch (see suffixspec.h).  out may be q."""
    args = (q, k, v, k_cache, v_cache, table, offsets, cached, freq, mask, positions, q_weight, k_weight, eps, interleaved, scale, out, status)
    got = (_call or _loaded()).rotate(*args)
    return got if type(got) is torch.Tensor else _made("rotate", got, args)


def sd_attend(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, offsets: torch.Tensor, cached: torch.Tensor,
              *, mask: Optional[torch.Tensor] = None, scale: Optional[float] = None, window: int = 0, sinks: int = 0, shared: int = 0,
              out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the rows q [rows, q_heads, head_dim] of draft trees over their requests' caches under the mask of sd_speculate (None: each row
    sees those before it).  scale: 1 / sqrt(head_dim) unless given.  window, sinks: a row sees the last `window` positions and the first `sinks` (0: all).
    shared: so many first places of all requests are in the same pages and are read once for the batch."""
    args = (q, k_cache, v_cache, table, offsets, cached, mask, scale, window, sinks, shared, out, lse, status)
    got = (_call or _loaded()).attend(*args)
    return got if type(got) is torch.Tensor else _made("attend", got, args)


def sd_accept(logits: torch.Tensor, offsets: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor, *,
              out: Optional[Dict[str, torch.Tensor]] = None, status: Optional[torch.Tensor] = None) -> Dict[str, torch.Tensor]:
    """Greedy verification of the drafts (tokens, parents: of sd_speculate) against logits [rows, vocab].  Returns targets [rows], path [n, max_draft + 1],
    and offsets [n + 1] and tokens [rows], which sd_step takes as they are."""
    args = (logits, offsets, tokens, parents, out, status)
    got = (_call or _loaded()).accept(*args)
    return got if type(got) is dict else _made("accept", got, args)


def sd_commit(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, cached: torch.Tensor, path: torch.Tensor, *,
              out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Keys and values of the accepted rows (path: of sd_accept) to where their sequences continue, in a cache
    [pages, page_size, kv_heads, head_dim] or, for all layers at once, [layers, pages, ...].  Returns the requests' lengths from now on; out may be cached."""
    args = (k_cache, v_cache, table, cached, path, out, status)
    got = (_call or _loaded()).commit(*args)
    return got if type(got) is torch.Tensor else _made("commit", got, args)


def rotary_frequencies(rot_dim: int, base: float = 10000.0, *, device=None, factor: float = 1.0, original: int = 0, fast: float = 32.0,
                       slow: float = 1.0) -> tuple:
    """(freq, scale) for sd_rotate: base ** (-2 j / rot_dim) radians per position for pair j.  For contexts longer than a model was trained with,
    `factor` times as long: all frequencies divided by `factor` (original = 0), or, with `original` the length it was trained with, only
    those that turn less than `slow` times within it, none of those that turn more than `fast` times, the others in between in proportion
    (linear in j), and the turned elements times 1 + 0.1 ln(factor): the method "YaRN" of Peng et al. (arXiv 2309.00071), with its constants."""
    j = torch.arange(rot_dim // 2, dtype=torch.float64)
    freq = base ** (-2.0 * j / rot_dim)
    scale = 1.0
    if factor != 1.0 and original:
        def pair(turns):                                         # the pair that turns so many times within `original`
            return rot_dim * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot_dim - 1)
        part = ((j - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        freq = freq * (1 - part) + freq / factor * part
        scale = 1.0 + 0.1 * math.log(factor)
    else:
        freq = freq / factor
    return freq.to(device or torch.device("cuda", torch.cuda.current_device())), scale


def sd_free(store: int) -> None:
    library().sd_free(store)


def sd_trim() -> None:
    """Give back the memory that is kept of freed stores (by itself that takes up to 30 seconds)."""
    library().sd_trim()


# ---- convenience wrapper ---------------------------------------------------------------------
class BoundStep:
    """One sd_step call with all of its arguments already converted (see SuffixStore.bind_step).
    Calling the object launches the step; `out` holds the output tensors it writes."""

    def __init__(self, store, slots, offsets, new_tokens, P, alpha, max_spec, flags, budget_cap, out, stream, tau=0.0):
        self.out = out
        self._keep = (store, slots, offsets, new_tokens, budget_cap)       # the buffers must outlive the calls
        self._prm = _SpecParams(P, alpha, max_spec, flags, tau)
        self._fn = library().sd_step
        self._args = (
            store._h, int(slots.numel()), _ptr(slots, torch.int32, "slots"), _ptr(offsets, torch.int64, "offsets"),
            _ptr(new_tokens, torch.int32, "new_tokens"), C.byref(self._prm), _ptr(budget_cap, torch.int32, "budget_cap"),
            *_out_ptrs(out), stream)

    def __call__(self) -> Dict[str, torch.Tensor]:
        rc = self._fn(*self._args)
        if rc != 0:
            raise SuffixSpecError(rc, "sd_step")
        return self.out


class SuffixStore:
    """Global suffix tree + per-request trees on one GPU."""

    def __init__(self, corpus: Optional[torch.Tensor], seq_offsets: Optional[torch.Tensor], *, vocab: int,
                 depth_cap: int, max_requests: int, max_req_tokens: int, max_spec_cap: int,
                 global_extra_nodes: int = -1, slot_pool_nodes: int = 0):
        self.vocab, self.depth_cap, self.max_requests = vocab, depth_cap, max_requests
        self.max_req_tokens, self.max_spec_cap = max_req_tokens, max_spec_cap
        self.device = corpus.device if corpus is not None else torch.device("cuda", torch.cuda.current_device())
        self._h = sd_build(corpus, seq_offsets, vocab=vocab, depth_cap=depth_cap, max_requests=max_requests,
                           max_req_tokens=max_req_tokens, max_spec_cap=max_spec_cap,
                           global_extra_nodes=global_extra_nodes, slot_pool_nodes=slot_pool_nodes)

    @property
    def handle(self) -> int:
        return self._h

    def free(self) -> None:
        if self._h:
            sd_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def append(self, slots: torch.Tensor, offsets: torch.Tensor, tokens: torch.Tensor,
               reset: Optional[torch.Tensor] = None) -> None:
        sd_append(self._h, slots, offsets, tokens, reset)

    def build_requests(self, slots, offsets, tokens: torch.Tensor) -> None:
        """Start new requests: `slots` and `offsets` are HOST sequences, `tokens` a CUDA tensor."""
        import numpy as np
        hs = np.ascontiguousarray(slots, dtype=np.int32)
        ho = np.ascontiguousarray(offsets, dtype=np.int64)
        rc = library().sd_build_requests(self._h, int(hs.size), hs.ctypes.data, ho.ctypes.data,
                                         _ptr(tokens, torch.int32, "tokens"), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_build_requests")

    def alloc_outputs(self, n: int) -> Dict[str, torch.Tensor]:
        """Output tensors of sd_speculate for n requests.  They are views into ONE device
        buffer (returned under the key "packed"), so a caller that wants the drafts on the host
        needs a single device-to-host copy; `unpack_outputs` makes the same views on a host copy."""
        packed = torch.empty(self.packed_output_bytes(n), dtype=torch.uint8, device=self.device)
        return self.unpack_outputs(packed, n)

    def _output_layout(self, n: int):
        M = self.max_spec_cap
        words = (M + 31) // 32
        fields = [("score", torch.float64, (n,)), ("tokens", torch.int32, (n, M)), ("parents", torch.int32, (n, M)),
                  ("positions", torch.int32, (n, M)), ("mask", torch.int32, (n, M, words)),
                  ("n_draft", torch.int32, (n,)), ("chosen_tree", torch.int32, (n,)), ("chosen_p", torch.int32, (n,)),
                  ("status", torch.int32, (n,))]
        off, lay = 0, []
        for name, dt, shape in fields:
            size = torch.empty(0, dtype=dt).element_size()
            cnt = 1
            for d in shape:
                cnt *= d
            lay.append((name, dt, shape, off, cnt * size))
            off += (cnt * size + 15) // 16 * 16
        return lay, off

    def packed_output_bytes(self, n: int) -> int:
        return max(16, self._output_layout(n)[1])

    def unpack_outputs(self, packed: torch.Tensor, n: int) -> Dict[str, torch.Tensor]:
        lay, _ = self._output_layout(n)
        out = {"packed": packed}
        for name, dt, shape, off, nbytes in lay:
            out[name] = packed[off:off + nbytes].view(dt).view(shape)
        return out

    def speculate(self, slots: torch.Tensor, P: int, alpha: float, max_spec: int, flags: int = 0,
                  budget_cap: Optional[torch.Tensor] = None,
                  out: Optional[Dict[str, torch.Tensor]] = None, tau: float = 0.0) -> Dict[str, torch.Tensor]:
        """mask is returned as int32 words (same bits as the uint32 of the C ABI)."""
        if out is None:
            out = self.alloc_outputs(int(slots.numel()))
        sd_speculate(self._h, slots, P, alpha, max_spec, flags, budget_cap, out, tau)
        return out

    def step(self, slots: torch.Tensor, offsets: torch.Tensor, new_tokens: torch.Tensor, P: int, alpha: float,
             max_spec: int, flags: int = 0, budget_cap: Optional[torch.Tensor] = None,
             out: Optional[Dict[str, torch.Tensor]] = None, tau: float = 0.0) -> Dict[str, torch.Tensor]:
        """One decode step in one launch: append `new_tokens` (ragged by `offsets`) to the slots,
        then speculate.  Same result as append() followed by speculate()."""
        if out is None:
            out = self.alloc_outputs(int(slots.numel()))
        rc = (_call or _loaded()).step(self._h, slots, offsets, new_tokens, P, alpha, max_spec, flags, tau, budget_cap,
                                       out)
        if rc != 0:
            raise SuffixSpecError(rc, "sd_step")
        return out

    def bind_step(self, slots: torch.Tensor, offsets: torch.Tensor, new_tokens: torch.Tensor, P: int, alpha: float,
                  max_spec: int, flags: int = 0, budget_cap: Optional[torch.Tensor] = None,
                  out: Optional[Dict[str, torch.Tensor]] = None, stream: Optional[int] = None,
                  tau: float = 0.0) -> "BoundStep":
        """step() with the argument marshalling done once.  A serving loop calls sd_step with the
        same buffers every step (it refills them in place: `new_tokens` is the whole token buffer,
        `offsets` says how much of it a step uses), so the returned object keeps the converted
        pointers and each call of it is just the C call.  `stream`: a cudaStream_t as an integer;
        default: the stream that is current now."""
        if out is None:
            out = self.alloc_outputs(int(slots.numel()))
        return BoundStep(self, slots, offsets, new_tokens, P, alpha, max_spec, flags, budget_cap, out,
                         _stream() if stream is None else stream, tau)

    def query_counts(self, tree: torch.Tensor, offsets: torch.Tensor, paths: torch.Tensor) -> torch.Tensor:
        n = int(tree.numel())
        counts = torch.empty(n, dtype=torch.int32, device=self.device)
        rc = library().sd_query_counts(self._h, n, _ptr(tree, torch.int32, "tree"),
                                       _ptr(offsets, torch.int64, "offsets"), _ptr(paths, torch.int32, "paths"),
                                       _ptr(counts, torch.int32, "counts"), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_query_counts")
        return counts

    def enumerate(self, tree: int, max_nodes: int) -> Dict[str, torch.Tensor]:
        """All nodes of `tree` (-1: global) as records parent / token / count / depth (see sd_enumerate)."""
        o = {k: torch.empty(max(max_nodes, 1), dtype=torch.int32, device=self.device) for k in ("parent", "token", "count", "depth")}
        n = C.c_int64(0)
        rc = library().sd_enumerate(self._h, tree, max_nodes, o["parent"].data_ptr(), o["token"].data_ptr(),
                                    o["count"].data_ptr(), o["depth"].data_ptr(), C.byref(n), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_enumerate")
        return {k: v[:n.value] for k, v in o.items()}

    def slot_info(self, slots: torch.Tensor):
        n = int(slots.numel())
        o = [torch.empty(n, dtype=torch.int32, device=self.device) for _ in range(3)]
        rc = library().sd_slot_info(self._h, n, _ptr(slots, torch.int32, "slots"), o[0].data_ptr(), o[1].data_ptr(),
                                    o[2].data_ptr(), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_slot_info")
        return {"len": o[0], "nodes": o[1], "status": o[2]}

    def entropy(self, tree: int = -1) -> float:
        """Count-weighted mean entropy (bits) of the children distributions of `tree`."""
        h = C.c_double(0.0)
        rc = library().sd_entropy(self._h, tree, C.byref(h), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_entropy")
        return h.value

    def stats(self) -> dict:
        st = _Stats()
        rc = library().sd_stats(self._h, C.byref(st), _stream())
        if rc != 0:
            raise SuffixSpecError(rc, "sd_stats")
        return {k: getattr(st, k) for k, _ in _Stats._fields_}
