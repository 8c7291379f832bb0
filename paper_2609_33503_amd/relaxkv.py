"""Thin ctypes binding of ``librelaxkv.so`` (the C ABI in include/relaxkv.h).

Argument marshalling only: every step of the hot path runs in the library's
HIP kernels.  PyTorch supplies device memory (tensors) and streams.  There is
no fallback: if the library is missing or a call fails, an exception is raised.
"""

from __future__ import annotations

import ctypes
import math
import os
from ctypes import (POINTER, Structure, c_char_p, c_double, c_float, c_int32, c_int64,
                    c_size_t, c_void_p)

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librelaxkv.so")

OK, EINVAL, ENOSPACE, EUNSUPPORTED, EDEVICE = 0, -1, -2, -3, -4
ERR_NAN_SCORE, ERR_BAD_TARGETS, ERR_ROWS = 1, 2, 4      # bits of the device error word
DTYPE_F32, DTYPE_BF16 = 0, 1
CONTEXT_UNION, CONTEXT_FULL = 0, 1
CONTEXT_SETS_UNION, CONTEXT_SETS_GLOBAL, CONTEXT_SETS_LAYERWISE = 0, 1, 2
BATCH_ERR_LENGTHS = 1                                   # bit of a batch's error word
MAX_SELECTED_BLOCKS = 2048

EXPORTS = ("relaxkv_status_string", "relaxkv_anchor_count", "relaxkv_validate",
           "relaxkv_score_workspace_bytes", "relaxkv_sets_bytes", "relaxkv_sets_bind",
           "relaxkv_score", "relaxkv_select", "relaxkv_build_sets", "relaxkv_build_sets_context",
           "relaxkv_select_global",
           "relaxkv_build_sets_global", "relaxkv_sparse_attn", "relaxkv_update_cache",
           "relaxkv_query_attn_workspace_bytes", "relaxkv_query_attn",
           "relaxkv_query_attn_noalloc", "relaxkv_counts_to_host",
           "relaxkv_batch_bytes", "relaxkv_batch_bind", "relaxkv_batch_plan",
           "relaxkv_batch_to_host", "relaxkv_fresh_rows", "relaxkv_batch_rows",
           "relaxkv_shared_attn_workspace_bytes", "relaxkv_shared_attn", "relaxkv_block_means",
           "relaxkv_block_select_workspace_bytes", "relaxkv_block_select",
           "relaxkv_block_attn_workspace_bytes", "relaxkv_block_attn")
QUERY_ATTN_NOALLOC_MAX_BYTES = 32 << 20


class RelaxKVError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {_status_text(status)} ({status})")


class Problem(Structure):
    _fields_ = [("L", c_int32), ("T_c", c_int32), ("n_query", c_int32), ("H", c_int32),
                ("H_kv", c_int32), ("d", c_int32), ("dtype", c_int32),
                ("softmax_scale", c_float), ("anchor_ratio", c_double),
                ("q", c_void_p), ("k_cache", c_void_p), ("v_cache", c_void_p),
                ("q_lse", c_void_p), ("kv_stride_layer", c_int64), ("kv_stride_head", c_int64),
                ("kv_stride_token", c_int64)]


class Sets(Structure):
    _fields_ = [("L", c_int32), ("T_c", c_int32), ("k", c_int32),
                ("anchors", c_void_p), ("h", c_void_p), ("U", c_void_p), ("cidx", c_void_p),
                ("R_off", c_void_p), ("R_idx", c_void_p), ("R_u", c_void_p),
                ("src", c_void_p), ("rank", c_void_p), ("counts", c_void_p),
                ("edges", c_void_p), ("ctx", c_void_p), ("g", c_void_p), ("tiles", c_void_p),
                ("global_targets", c_int32), ("context_sets", c_int32)]


class CBatch(Structure):
    _fields_ = [("n_seq", c_int32), ("n_rows", c_int32), ("max_suffix", c_int32),
                ("tile_cap", c_int32), ("T_c", c_int32), ("H", c_int32), ("H_kv", c_int32),
                ("d", c_int32), ("dtype", c_int32), ("row_off", c_void_p), ("row_seq", c_void_p),
                ("row_pos", c_void_p), ("tiles", c_void_p), ("counts", c_void_p)]


class CSuffix(Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("stride_seq", c_int64),
                ("stride_head", c_int64), ("stride_token", c_int64)]


class CRope(Structure):
    _fields_ = [("inv_freq", c_void_p), ("q_weight", c_void_p), ("k_weight", c_void_p),
                ("eps", c_float), ("rot", c_int32), ("interleaved", c_int32)]


class CRows(Structure):
    _fields_ = [("q", c_void_p), ("k", c_void_p), ("v", c_void_p), ("q_stride", c_int64),
                ("k_stride", c_int64), ("v_stride", c_int64), ("n_rows", c_int32)]


_lib = None


def load(path=None):
    """Load the library (once).  Raises if it has not been built, or if the
    in-tree library was not built from the sources in the tree (its build
    record, written by ``build.py``, must match them)."""
    global _lib
    if _lib is not None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2609_33503_amd.build`")
    if path is None:
        from . import build
        build.verify(p)
    lib = ctypes.CDLL(p)
    lib.relaxkv_status_string.restype = c_char_p
    lib.relaxkv_status_string.argtypes = [c_int32]
    lib.relaxkv_anchor_count.restype = c_int32
    lib.relaxkv_anchor_count.argtypes = [c_double, c_int32]
    lib.relaxkv_validate.restype = c_int32
    lib.relaxkv_validate.argtypes = [POINTER(Problem)]
    lib.relaxkv_score_workspace_bytes.restype = c_size_t
    lib.relaxkv_score_workspace_bytes.argtypes = [POINTER(Problem)]
    lib.relaxkv_sets_bytes.restype = c_size_t
    lib.relaxkv_sets_bytes.argtypes = [POINTER(Problem)]
    lib.relaxkv_sets_bind.restype = c_int32
    lib.relaxkv_sets_bind.argtypes = [POINTER(Problem), c_void_p, c_size_t, POINTER(Sets)]
    lib.relaxkv_score.restype = c_int32
    lib.relaxkv_score.argtypes = [POINTER(Problem), c_void_p, c_size_t, c_void_p, c_void_p]
    lib.relaxkv_select.restype = c_int32
    lib.relaxkv_select.argtypes = [POINTER(Problem), c_void_p, POINTER(Sets), c_void_p]
    lib.relaxkv_build_sets.restype = c_int32
    lib.relaxkv_build_sets.argtypes = [POINTER(Problem), POINTER(Sets), c_void_p]
    lib.relaxkv_build_sets_context.restype = c_int32
    lib.relaxkv_build_sets_context.argtypes = [POINTER(Problem), c_void_p, c_int32, POINTER(Sets),
                                               c_void_p]
    lib.relaxkv_select_global.restype = c_int32
    lib.relaxkv_select_global.argtypes = [POINTER(Problem), c_void_p, c_double, POINTER(Sets),
                                          c_void_p, c_void_p, c_void_p, c_void_p]
    lib.relaxkv_build_sets_global.restype = c_int32
    lib.relaxkv_build_sets_global.argtypes = [POINTER(Problem), POINTER(Sets), c_void_p, c_void_p,
                                              c_void_p]
    lib.relaxkv_sparse_attn.restype = c_int32
    lib.relaxkv_sparse_attn.argtypes = [POINTER(Problem), POINTER(Sets), c_int32, c_void_p,
                                        c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                        c_int32, c_void_p]
    lib.relaxkv_update_cache.restype = c_int32
    lib.relaxkv_update_cache.argtypes = [POINTER(Problem), POINTER(Sets), c_int32, c_void_p,
                                         c_void_p, c_int32, c_void_p, c_void_p, c_void_p]
    lib.relaxkv_query_attn_workspace_bytes.restype = c_size_t
    lib.relaxkv_query_attn_workspace_bytes.argtypes = [POINTER(Problem)]
    lib.relaxkv_query_attn.restype = c_int32
    lib.relaxkv_query_attn.argtypes = [POINTER(Problem), c_int32, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.relaxkv_query_attn_noalloc.restype = c_int32
    lib.relaxkv_query_attn_noalloc.argtypes = [POINTER(Problem), c_int32, c_void_p, c_void_p,
                                               c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.relaxkv_counts_to_host.restype = c_int32
    lib.relaxkv_counts_to_host.argtypes = [POINTER(Sets), POINTER(c_int32), POINTER(c_int64),
                                           c_void_p]
    lib.relaxkv_batch_bytes.restype = c_size_t
    lib.relaxkv_batch_bytes.argtypes = [POINTER(Problem), c_int32, c_int32, c_int32]
    lib.relaxkv_batch_bind.restype = c_int32
    lib.relaxkv_batch_bind.argtypes = [POINTER(Problem), c_int32, c_int32, c_int32, c_void_p,
                                       c_size_t, POINTER(CBatch)]
    lib.relaxkv_batch_plan.restype = c_int32
    lib.relaxkv_batch_plan.argtypes = [POINTER(Problem), POINTER(CBatch), c_void_p, c_void_p,
                                       c_void_p]
    lib.relaxkv_batch_to_host.restype = c_int32
    lib.relaxkv_batch_to_host.argtypes = [POINTER(CBatch), POINTER(c_int32), c_void_p]
    lib.relaxkv_fresh_rows.restype = c_int32
    lib.relaxkv_fresh_rows.argtypes = [POINTER(Problem), POINTER(CRope), POINTER(CRows), c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_void_p]
    lib.relaxkv_batch_rows.restype = c_int32
    lib.relaxkv_batch_rows.argtypes = [POINTER(Problem), POINTER(CRope), POINTER(CBatch),
                                       POINTER(CRows), c_void_p, POINTER(CSuffix), c_void_p]
    lib.relaxkv_shared_attn_workspace_bytes.restype = c_size_t
    lib.relaxkv_shared_attn_workspace_bytes.argtypes = [POINTER(Problem), POINTER(CBatch)]
    lib.relaxkv_shared_attn.restype = c_int32
    lib.relaxkv_shared_attn.argtypes = [POINTER(Problem), POINTER(CBatch), c_int32, c_void_p,
                                        c_void_p, c_void_p, POINTER(CSuffix), c_void_p, c_void_p,
                                        c_void_p, c_size_t, c_void_p]
    lib.relaxkv_block_means.restype = c_int32
    lib.relaxkv_block_means.argtypes = [POINTER(Problem), c_int32, c_void_p, c_int32, c_void_p,
                                        c_void_p]
    lib.relaxkv_block_select_workspace_bytes.restype = c_size_t
    lib.relaxkv_block_select_workspace_bytes.argtypes = [POINTER(Problem), POINTER(CBatch), c_int32]
    lib.relaxkv_block_select.restype = c_int32
    lib.relaxkv_block_select.argtypes = [POINTER(Problem), POINTER(CBatch), c_int32, c_void_p,
                                         c_void_p, c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.relaxkv_block_attn_workspace_bytes.restype = c_size_t
    lib.relaxkv_block_attn_workspace_bytes.argtypes = [POINTER(Problem), POINTER(CBatch), c_int32,
                                                       c_int32]
    lib.relaxkv_block_attn.restype = c_int32
    lib.relaxkv_block_attn.argtypes = [POINTER(Problem), POINTER(CBatch), c_int32, c_void_p,
                                       c_void_p, c_int32, c_void_p, c_int32, c_void_p,
                                       POINTER(CSuffix), c_void_p, c_void_p, c_void_p, c_size_t,
                                       c_void_p]
    _lib = lib
    return lib


def _status_text(s):
    try:
        return load().relaxkv_status_string(s).decode()
    except Exception:  # pragma: no cover - only when the library itself is missing
        return "status"


def _check(status, what):
    if status != OK:
        raise RelaxKVError(status, what)


# Host cost matters here: the small calls are as short on the GPU as the
# marshalling of one call (6 tensors) is on the host.  So addresses go to ctypes
# as plain integers, and each tensor passes one combined test of the usual case;
# whatever fails it is checked again in full (_need, _need_cache), which accepts it
# or says what is wrong.  Per call with its launches: query_attn 19.2 -> 11.9 us,
# update_cache 15.4 -> 9.0 us, sparse_attn 12.5 -> 7.6 us.
_Tensor = torch.Tensor
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


def _dense(t, dtype, shape, index):
    """A plain contiguous tensor of this dtype and shape on GPU `index` (get_device() is -1 for
    a host tensor)."""
    return (type(t) is _Tensor and t.dtype is dtype and t.shape == shape
            and t.get_device() == index and t.is_contiguous())


def _need(t, name, dtype, shape, device):
    """Raise ValueError unless t is a contiguous tensor on `device` with this dtype
    and shape (None in `shape` matches any size).  Every pointer the library
    gets passes through here, so a host tensor, a tensor on another device or
    one too small never reaches a kernel."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the problem's tensors are on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    _need_shape(t, name, shape)


def _need_shape(t, name, shape):
    if t.dim() != len(shape) or any(want is not None and got != want
                                    for got, want in zip(t.shape, shape)):
        want = tuple("*" if x is None else x for x in shape)
        raise ValueError(f"{name} must have shape {want}, got {tuple(t.shape)}")


def _need_cache(t, name, dtype, shape, device, strides=None):
    """A [L][H_kv][T_c][d] cache tensor: like _need, but any strides of the first
    three dimensions are passed on (the library checks them); d must be
    contiguous, and with `strides` given the tensor must have exactly those."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the problem's tensors are on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    _need_shape(t, name, shape)
    if t.stride(3) != 1:
        raise ValueError(f"{name} must have contiguous rows (stride 1 in d)")
    if strides is not None and _cache_strides(t) != tuple(strides):
        raise ValueError(f"{name} must have the strides {tuple(strides)} of the request's "
                         f"cache, got {_cache_strides(t)}")


def _cache_strides(t):
    """The layer, KV-head and token strides of a cache tensor for the descriptor
    (0, the dense value, for a dimension of size 1, whose stride torch leaves
    arbitrary and the library never uses)."""
    if any(st == 0 and n > 1 for st, n in zip(t.stride()[:3], t.shape[:3])):
        raise ValueError("an expanded tensor (stride 0) is no cache")
    return tuple(st if n > 1 else 0 for st, n in zip(t.stride()[:3], t.shape[:3]))


def _nbytes(t):
    return t.numel() * t.element_size()


def anchor_count(ratio, T_c):
    k = load().relaxkv_anchor_count(float(ratio), int(T_c))
    _check(OK if k > 0 else k, "relaxkv_anchor_count")
    return k


class Request:
    """One problem: the descriptor plus the tensors it points at (kept alive).

    q        [L][n_query][H][d]   bf16 or f32, CUDA, contiguous
    k_cache  [L][H_kv][T_c][d]    any strides with contiguous rows (e.g. a slice of a
                                  cache allocated for more tokens); the library checks them
    v_cache  [L][H_kv][T_c][d]    the same strides as k_cache
    q_lse    optional [L][n_query][H] f32 (natural log)
    """

    def __init__(self, q, k_cache, v_cache, anchor_ratio, softmax_scale=0.0, q_lse=None):
        lib = load()
        if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 4:
            raise ValueError("q must be a [L][n_query][H][d] device tensor")
        dt = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}.get(q.dtype)
        if dt is None:
            raise ValueError("dtype must be bfloat16 or float32")
        L, Qn, H, d = q.shape
        if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
            raise ValueError("k_cache must be a [L][H_kv][T_c][d] tensor")
        H_kv, T_c = k_cache.shape[1], k_cache.shape[2]
        self.device = q.device
        self._index = q.get_device()
        _need(q, "q", q.dtype, (L, Qn, H, d), self.device)
        _need_cache(k_cache, "k_cache", q.dtype, (L, H_kv, T_c, d), self.device)
        self.kv_strides = _cache_strides(k_cache)
        _need_cache(v_cache, "v_cache", q.dtype, (L, H_kv, T_c, d), self.device, self.kv_strides)
        if q_lse is not None:
            _need(q_lse, "q_lse", torch.float32, (L, Qn, H), self.device)
        self.dtype = q.dtype
        self.tensors = (q, k_cache, v_cache, q_lse)
        self.p = Problem(L, T_c, Qn, H, H_kv, d, dt, float(softmax_scale), float(anchor_ratio),
                         _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(q_lse), *self.kv_strides)
        _check(lib.relaxkv_validate(ctypes.byref(self.p)), "relaxkv_validate")
        self.L, self.T_c, self.n_query, self.H, self.H_kv, self.d = L, T_c, Qn, H, H_kv, d
        self.k = anchor_count(anchor_ratio, T_c)
        self._lib = lib
        self._cache_shape, self._cache_stride = (L, H_kv, T_c, d), k_cache.stride()
        self._scores_shape = (L, T_c)
        self._q_shape, self._kq_shape, self._lse_shape = (Qn, H, d), (Qn, H_kv, d), (Qn, H)
        self._batch_key = (T_c, H, H_kv, d, self.dtype, self._index)

    @property
    def p(self):
        """The descriptor; its reference, which every call passes, changes with it."""
        return self._p

    @p.setter
    def p(self, problem):
        self._p, self._ref = problem, ctypes.byref(problem)

    # ---- sizes and buffers (device memory comes from torch)
    def workspace_bytes(self):
        return load().relaxkv_score_workspace_bytes(ctypes.byref(self.p))

    def sets_bytes(self):
        return load().relaxkv_sets_bytes(ctypes.byref(self.p))

    def alloc_workspace(self):
        return torch.empty(self.workspace_bytes(), dtype=torch.uint8, device=self.device)

    # ---- argument checks shared by the calls
    def _scores(self, scores):
        self._want(scores, "scores", torch.float32, self._scores_shape)

    def _want(self, t, name, dtype, shape):
        if not _dense(t, dtype, shape, self._index):
            _need(t, name, dtype, shape, self.device)

    def _caches(self, k_cache, v_cache):
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            if not (type(t) is _Tensor and t.dtype is self.dtype
                    and t.get_device() == self._index and t.shape == self._cache_shape
                    and t.stride() == self._cache_stride):
                _need_cache(t, name, self.dtype, self._cache_shape, self.device, self.kv_strides)

    def _sets(self, sets):
        if not isinstance(sets, SetsBuffer) or sets.buf.device != self.device or \
                (sets.s.L, sets.s.T_c, sets.s.k) != (self.L, self.T_c, self.k):
            raise ValueError("sets must come from alloc_sets() of a request of this shape")

    def _ws(self, ws, name="ws"):
        if type(ws) is _Tensor and ws.get_device() == self._index and ws.is_contiguous():
            return
        if not isinstance(ws, torch.Tensor) or ws.device != self.device or not ws.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor on {self.device}")

    def alloc_sets(self):
        """A device buffer for the sets and its bound descriptor."""
        nbytes = self.sets_bytes()
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = buf.data_ptr()
        pad = (-base) % 256
        s = Sets()
        _check(load().relaxkv_sets_bind(ctypes.byref(self.p), ctypes.c_void_p(base + pad),
                                        nbytes, ctypes.byref(s)), "relaxkv_sets_bind")
        return SetsBuffer(self, buf, s, pad)

    # ---- the four calls
    def score(self, ws, scores, stream=None):
        self._ws(ws)
        self._scores(scores)
        _check(self._lib.relaxkv_score(self._ref, _ptr(ws), _nbytes(ws), _ptr(scores),
                                    _stream(stream)), "relaxkv_score")

    def select(self, scores, sets, stream=None):
        self._scores(scores)
        self._sets(sets)
        _check(self._lib.relaxkv_select(self._ref, _ptr(scores), ctypes.byref(sets.s),
                                     _stream(stream)), "relaxkv_select")

    def build_sets(self, sets, stream=None):
        self._sets(sets)
        _check(self._lib.relaxkv_build_sets(self._ref, ctypes.byref(sets.s),
                                         _stream(stream)), "relaxkv_build_sets")

    def build_sets_context(self, scores, construction, sets, stream=None):
        """RelaxKV's anchors and targets with the context set replaced
        (CONTEXT_SETS_UNION / _GLOBAL / _LAYERWISE); scores [L][T_c] f32."""
        self._scores(scores)
        self._sets(sets)
        _check(self._lib.relaxkv_build_sets_context(self._ref, _ptr(scores),
                                                 int(construction), ctypes.byref(sets.s),
                                                 _stream(stream)), "relaxkv_build_sets_context")

    # ---- matched-target variants: one global target list for every layer
    def select_global(self, scores, target_ratio, sets, g, targets, n_targets, stream=None):
        """g [T_c] f32, targets [T_c] int32 and n_targets [1] int32 are outputs."""
        self._scores(scores)
        self._sets(sets)
        self._want(g, "g", torch.float32, (self.T_c,))
        self._want(targets, "targets", torch.int32, (self.T_c,))
        self._want(n_targets, "n_targets", torch.int32, (1,))
        _check(self._lib.relaxkv_select_global(self._ref, _ptr(scores),
                                            float(target_ratio), ctypes.byref(sets.s), _ptr(g),
                                            _ptr(targets), _ptr(n_targets), _stream(stream)),
               "relaxkv_select_global")

    def build_sets_global(self, sets, targets, n_targets, stream=None):
        """targets: int32 device [T_c], ascending in its first n_targets entries;
        n_targets: int32 device [1]."""
        self._sets(sets)
        self._want(targets, "targets", torch.int32, (self.T_c,))
        self._want(n_targets, "n_targets", torch.int32, (1,))
        _check(self._lib.relaxkv_build_sets_global(self._ref, ctypes.byref(sets.s),
                                                _ptr(targets), _ptr(n_targets), _stream(stream)),
               "relaxkv_build_sets_global")

    def sparse_attn(self, sets, layer, q_new, k_new, v_new, out, lse_out=None,
                    context_mode=CONTEXT_UNION, stream=None):
        """q_new/out [n][H][d], k_new/v_new [n][H_kv][d], lse_out [n][H] f32, with n
        rows allocated (normally |R_l|; targets past n are not computed and set the
        device error word)."""
        self._sets(sets)
        n = q_new.shape[0] if isinstance(q_new, torch.Tensor) and q_new.dim() == 3 else -1
        self._want(q_new, "q_new", self.dtype, (n, self.H, self.d))
        self._want(k_new, "k_new", self.dtype, (n, self.H_kv, self.d))
        self._want(v_new, "v_new", self.dtype, (n, self.H_kv, self.d))
        self._want(out, "out", self.dtype, (n, self.H, self.d))
        if lse_out is not None:
            self._want(lse_out, "lse_out", torch.float32, (n, self.H))
        _check(self._lib.relaxkv_sparse_attn(self._ref, ctypes.byref(sets.s), int(layer),
                                          _ptr(q_new), _ptr(k_new), _ptr(v_new), int(n),
                                          _ptr(out), _ptr(lse_out), int(context_mode),
                                          _stream(stream)),
               "relaxkv_sparse_attn")

    def update_cache(self, sets, layer, k_new, v_new, k_cache, v_cache, stream=None):
        """Fresh rows of R_l (k_new/v_new [n][H_kv][d]) into the cache
        (k_cache/v_cache: [L][H_kv][T_c][d] with the request's cache strides)."""
        self._sets(sets)
        n = k_new.shape[0] if isinstance(k_new, torch.Tensor) and k_new.dim() == 3 else -1
        self._want(k_new, "k_new", self.dtype, (n, self.H_kv, self.d))
        self._want(v_new, "v_new", self.dtype, (n, self.H_kv, self.d))
        self._caches(k_cache, v_cache)
        _check(self._lib.relaxkv_update_cache(self._ref, ctypes.byref(sets.s), int(layer),
                                           _ptr(k_new), _ptr(v_new), int(n), _ptr(k_cache),
                                           _ptr(v_cache), _stream(stream)),
               "relaxkv_update_cache")


    # ---- query-side completion (the query prefill after repair)
    def query_attn_workspace_bytes(self):
        return load().relaxkv_query_attn_workspace_bytes(ctypes.byref(self.p))

    def alloc_query_workspace(self):
        n = self.query_attn_workspace_bytes()
        return None if n == 0 else torch.empty(n, dtype=torch.uint8, device=self.device)

    def query_attn(self, layer, k_cache, v_cache, k_q, v_q, out, lse_out=None, ws=None,
                   stream=None):
        """k_cache/v_cache [L][H_kv][T_c][d] (the request's cache strides); k_q/v_q
        [n_query][H_kv][d]; out [n_query][H][d];
        lse_out [n_query][H] f32."""
        self._caches(k_cache, v_cache)
        self._want(k_q, "k_q", self.dtype, self._kq_shape)
        self._want(v_q, "v_q", self.dtype, self._kq_shape)
        self._want(out, "out", self.dtype, self._q_shape)
        if lse_out is not None:
            self._want(lse_out, "lse_out", torch.float32, self._lse_shape)
        if ws is not None:
            self._ws(ws)
        _check(self._lib.relaxkv_query_attn(self._ref, int(layer), _ptr(k_cache),
                                         _ptr(v_cache), _ptr(k_q), _ptr(v_q), _ptr(out),
                                         _ptr(lse_out), _ptr(ws), 0 if ws is None else _nbytes(ws),
                                         _stream(stream)), "relaxkv_query_attn")


    def query_attn_noalloc(self, layer, k_cache, v_cache, k_q, v_q, out, lse_out=None,
                           stream=None):
        """query_attn through the allocation-free entry point (the library's own
        per-GPU scratch; calls that overlap on one GPU race)."""
        self._caches(k_cache, v_cache)
        self._want(k_q, "k_q", self.dtype, self._kq_shape)
        self._want(v_q, "v_q", self.dtype, self._kq_shape)
        self._want(out, "out", self.dtype, self._q_shape)
        if lse_out is not None:
            self._want(lse_out, "lse_out", torch.float32, self._lse_shape)
        _check(self._lib.relaxkv_query_attn_noalloc(self._ref, int(layer), _ptr(k_cache),
                                                 _ptr(v_cache), _ptr(k_q), _ptr(v_q), _ptr(out),
                                                 _ptr(lse_out), _stream(stream)),
               "relaxkv_query_attn_noalloc")

    # ---- batched serving: many requests on this request's context cache
    def alloc_batch(self, n_seq, n_rows, max_suffix):
        """The maps of a step: n_seq requests with suffixes of up to max_suffix tokens, up to
        n_rows new tokens in a step."""
        n_seq, n_rows, max_suffix = int(n_seq), int(n_rows), int(max_suffix)
        nbytes = self._lib.relaxkv_batch_bytes(self._ref, n_seq, n_rows, max_suffix)
        if nbytes == 0:
            raise ValueError(f"no batch of {n_seq} requests, {n_rows} rows and suffixes of "
                             f"{max_suffix} tokens")
        buf = torch.zeros(nbytes + 256, dtype=torch.uint8, device=self.device)
        pad = (-buf.data_ptr()) % 256
        s = CBatch()
        _check(self._lib.relaxkv_batch_bind(self._ref, n_seq, n_rows, max_suffix,
                                            buf.data_ptr() + pad, nbytes, ctypes.byref(s)),
               "relaxkv_batch_bind")
        return Batch(self, buf, s, pad)

    def _here(self, stream):
        """The stream of a batched call, which runs on the request's GPU: the current device
        has to be that one."""
        if _current_device is not None and _current_device() != self._index:
            raise ValueError(f"the request is on {self.device}, the current device is "
                             f"cuda:{_current_device()}")
        if stream is not None and stream.device_index != self._index:
            raise ValueError(f"the stream is not on {self.device}")
        if stream is None and _raw_stream is not None:    # (the request's tensors are on the GPU)
            return _raw_stream(self._index)
        return _stream(stream)

    def _batch(self, batch):
        if type(batch) is not Batch or batch.key != self._batch_key:
            raise ValueError("batch must come from alloc_batch() of a request of this shape")

    def _suffix(self, batch, k, v):
        """The suffix caches' descriptor (the library checks the strides)."""
        shape = batch.suffix_shape
        for t, name in ((k, "k_suffix"), (v, "v_suffix")):
            if not (type(t) is _Tensor and t.dtype is self.dtype and t.shape == shape
                    and t.get_device() == self._index):
                _need_cache(t, name, self.dtype, shape, self.device)
        st = k.stride()
        if st != v.stride() or batch.flat or 0 in st or st[3] != 1:
            for t, name in ((k, "k_suffix"), (v, "v_suffix")):
                _need_cache(t, name, self.dtype, shape, self.device)
            st = _cache_strides(k)                        # (a dimension of size 1: any stride)
            if st != _cache_strides(v):
                raise ValueError("k_suffix and v_suffix must have the same strides")
        return CSuffix(k.data_ptr(), v.data_ptr(), st[0], st[1], st[2])

    def _projected(self, t, name, heads, n):
        """The row stride of a [n][heads][d] tensor whose rows are contiguous."""
        if t is None:
            return 0
        if type(t) is _Tensor and t.dtype is self.dtype and t.get_device() == self._index \
                and t.shape == (n, heads, self.d):
            st = t.stride()
            if st[2] == 1 and st[1] == self.d and n > 1 and st[0] > 0:
                return st[0]
        if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype != self.dtype:
            raise ValueError(f"{name} must be a {self.dtype} tensor on {self.device}")
        _need_shape(t, name, (n, heads, self.d))
        if n and ((heads > 1 and t.stride(1) != self.d) or t.stride(2) != 1):
            raise ValueError(f"{name} must have contiguous rows")
        if n > 1 and t.stride(0) == 0:
            raise ValueError(f"{name} must not be expanded (row stride 0)")
        return t.stride(0) if n > 1 else 0

    def _rows(self, q, k, v, n):
        return CRows(_ptr(q), _ptr(k), _ptr(v), self._projected(q, "q", self.H, n),
                     self._projected(k, "k", self.H_kv, n), self._projected(v, "v", self.H_kv, n), n)

    def _rope(self, rope):
        if type(rope) is not Rope:
            raise ValueError("rope must be a Rope")
        for device, dtype, d in rope.tensors:
            if device != self._index or dtype not in (None, self.dtype) or d not in (None, self.d):
                raise ValueError(f"rope's tensors must be on {self.device}, its norm weights "
                                 f"[{self.d}] {self.dtype}")
        return rope.ref

    def plan_batch(self, batch, past_len, new_len, stream=None):
        """past_len and new_len [n_seq] int32 device: tokens of each request's suffix before
        the step, and its new tokens."""
        self._batch(batch)
        self._want(past_len, "past_len", torch.int32, (batch.n_seq,))
        self._want(new_len, "new_len", torch.int32, (batch.n_seq,))
        _check(self._lib.relaxkv_batch_plan(self._ref, batch.ref, past_len.data_ptr(),
                                            new_len.data_ptr(), self._here(stream)),
               "relaxkv_batch_plan")

    def fresh_rows(self, rope, positions, q, k, v, q_out, k_out, v_out, stream=None):
        """Norm and rotation of projected rows at positions [n] int32, values copied: q
        [n][H][d], k and v [n][H_kv][d] (slices of one fused output, or None) into the dense
        rows q_out, k_out, v_out of the same shapes."""
        n = positions.shape[0] if isinstance(positions, torch.Tensor) and positions.dim() == 1 else -1
        self._want(positions, "positions", torch.int32, (n,))
        rows = self._rows(q, k, v, n)
        if (q is None) != (q_out is None) or (k is None) != (k_out is None) \
                or (v is None) != (v_out is None):
            raise ValueError("an output and its input must both be given, or neither")
        kv_shape = (n, self.H_kv, self.d)
        if q is not None:
            self._want(q_out, "q_out", self.dtype, (n, self.H, self.d))
        if k is not None:
            self._want(k_out, "k_out", self.dtype, kv_shape)
        if v is not None:
            self._want(v_out, "v_out", self.dtype, kv_shape)
        _check(self._lib.relaxkv_fresh_rows(self._ref, self._rope(rope), ctypes.byref(rows),
                                            positions.data_ptr(), _ptr(q_out), _ptr(k_out),
                                            _ptr(v_out), self._here(stream)), "relaxkv_fresh_rows")

    def batch_rows(self, rope, batch, q, k, v, q_out, k_suffix, v_suffix, stream=None):
        """fresh_rows for the rows of a planned step: queries to q_out [n_rows][H][d], keys and
        values to their tokens of the suffix caches [n_seq][H_kv][max_suffix][d] (any strides
        with contiguous rows)."""
        self._batch(batch)
        n = batch.n_rows
        rows = self._rows(q, k, v, n)
        if (q is None) != (q_out is None):
            raise ValueError("q_out and its input must both be given, or neither")
        if q_out is not None:
            self._want(q_out, "q_out", self.dtype, (n, self.H, self.d))
        suffix = self._suffix(batch, k_suffix, v_suffix)
        _check(self._lib.relaxkv_batch_rows(self._ref, self._rope(rope), batch.ref,
                                            ctypes.byref(rows), _ptr(q_out), ctypes.byref(suffix),
                                            self._here(stream)), "relaxkv_batch_rows")

    def shared_attn_workspace_bytes(self, batch):
        self._batch(batch)
        return self._lib.relaxkv_shared_attn_workspace_bytes(self._ref, batch.ref)

    def alloc_shared_workspace(self, batch):
        n = self.shared_attn_workspace_bytes(batch)
        return None if n == 0 else torch.empty(n, dtype=torch.uint8, device=self.device)

    def _batch_attn(self, batch, k_cache, v_cache, q, out, lse_out, ws):
        self._batch(batch)
        self._caches(k_cache, v_cache)
        shape, dtype, index = batch.q_shape, self.dtype, self._index
        if not (_dense(q, dtype, shape, index) and _dense(out, dtype, shape, index)):
            self._want(q, "q", dtype, shape)
            self._want(out, "out", dtype, shape)
        if lse_out is not None and not _dense(lse_out, torch.float32, batch.lse_shape, index):
            self._want(lse_out, "lse_out", torch.float32, batch.lse_shape)
        if ws is not None:
            self._ws(ws)

    def shared_attn(self, batch, layer, k_cache, v_cache, q, k_suffix, v_suffix, out, lse_out=None,
                    ws=None, stream=None):
        """Attention of a planned step's rows q [n_rows][H][d] over the context cache
        (k_cache/v_cache as in query_attn) and, causally, their request's suffix
        [n_seq][H_kv][max_suffix][d], which holds the step's tokens already; out
        [n_rows][H][d], lse_out [n_rows][H] f32."""
        self._batch_attn(batch, k_cache, v_cache, q, out, lse_out, ws)
        suffix = self._suffix(batch, k_suffix, v_suffix)
        _check(self._lib.relaxkv_shared_attn(self._ref, batch.ref, int(layer), _ptr(k_cache),
                                             _ptr(v_cache), _ptr(q), ctypes.byref(suffix),
                                             _ptr(out), _ptr(lse_out), _ptr(ws),
                                             0 if ws is None else _nbytes(ws), self._here(stream)),
               "relaxkv_shared_attn")

    # ---- attention over context blocks that a score selects for each row
    def block_count(self, block):
        return -(-self.T_c // int(block))

    def block_means(self, layer, k_cache, block, means, stream=None):
        """Key means over blocks of 16, 32, 64 or 128 positions of one layer of k_cache, or of
        all of them (layer None): means [n][H_kv][blocks][d]."""
        self._caches(k_cache, k_cache)
        if layer is not None and not 0 <= int(layer) < self.L:
            raise ValueError(f"layer must be None or in [0, {self.L})")
        if int(block) < 1:
            raise ValueError("block must be 16, 32, 64 or 128")
        self._want(means, "means", self.dtype, (self.L if layer is None else 1, self.H_kv,
                                                self.block_count(block), self.d))
        _check(self._lib.relaxkv_block_means(self._ref, -1 if layer is None else int(layer),
                                             _ptr(k_cache), int(block), _ptr(means),
                                             self._here(stream)), "relaxkv_block_means")

    def block_workspace_bytes(self, batch, block, n_sel):
        """Scratch of block_select and block_attn (one buffer serves both in turn)."""
        self._batch(batch)
        return max(self._lib.relaxkv_block_select_workspace_bytes(self._ref, batch.ref, int(block)),
                   self._lib.relaxkv_block_attn_workspace_bytes(self._ref, batch.ref, int(block),
                                                                int(n_sel)))

    def alloc_block_workspace(self, batch, block, n_sel):
        return torch.empty(self.block_workspace_bytes(batch, block, n_sel), dtype=torch.uint8,
                           device=self.device)

    def _lists(self, batch, blocks):
        n = blocks.shape[2] if isinstance(blocks, torch.Tensor) and blocks.dim() == 3 else -1
        self._want(blocks, "blocks", torch.int32, (batch.n_rows, self.H_kv, n))
        return n

    def block_select(self, batch, block, means, q, blocks, ws, stream=None):
        """The context blocks with the largest products of a row's summed group queries and
        the block means [H_kv][blocks][d] of its layer: blocks [n_rows][H_kv][n_sel] int32,
        ascending."""
        self._batch(batch)
        if int(block) < 1:
            raise ValueError("block must be 16, 32, 64 or 128")
        self._want(means, "means", self.dtype, (self.H_kv, self.block_count(block), self.d))
        self._want(q, "q", self.dtype, (batch.n_rows, self.H, self.d))
        n_sel = self._lists(batch, blocks)
        self._ws(ws)
        _check(self._lib.relaxkv_block_select(self._ref, batch.ref, int(block), _ptr(means), _ptr(q),
                                              n_sel, _ptr(blocks), _ptr(ws), _nbytes(ws),
                                              self._here(stream)), "relaxkv_block_select")

    def block_attn(self, batch, layer, k_cache, v_cache, block, blocks, q, k_suffix, v_suffix, out,
                   lse_out=None, ws=None, stream=None):
        """shared_attn over the listed blocks of each row and KV head (blocks
        [n_rows][H_kv][n_sel] int32, entries outside the blocks are none) instead of the whole
        context."""
        self._batch_attn(batch, k_cache, v_cache, q, out, lse_out, ws)
        n_sel = self._lists(batch, blocks)
        suffix = self._suffix(batch, k_suffix, v_suffix)
        _check(self._lib.relaxkv_block_attn(self._ref, batch.ref, int(layer), _ptr(k_cache),
                                            _ptr(v_cache), int(block), _ptr(blocks), n_sel, _ptr(q),
                                            ctypes.byref(suffix), _ptr(out), _ptr(lse_out),
                                            _ptr(ws), 0 if ws is None else _nbytes(ws),
                                            self._here(stream)), "relaxkv_block_attn")


class Rope:
    """Norm and rotation of a model (fresh_rows, batch_rows).

    inv_freq     [rot/2] f32: the angle of pair i at position P is P * inv_freq[i]; rot is a
                 multiple of 16 up to d (None: no rotation)
    q_weight, k_weight  [d] in the rows' dtype: RMS norm over each head, None for no norm
    interleaved  pairs (2i, 2i + 1) instead of (i, i + rot/2)
    """

    def __init__(self, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
        if inv_freq is not None and (not isinstance(inv_freq, torch.Tensor)
                                     or inv_freq.dtype != torch.float32 or inv_freq.dim() != 1
                                     or not inv_freq.is_contiguous()):
            raise ValueError("inv_freq must be a contiguous float32 tensor [rot/2]")
        for t, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None and not (isinstance(t, torch.Tensor) and t.dim() == 1
                                      and t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous tensor [d] or None")
        self.inv_freq, self.q_weight, self.k_weight = inv_freq, q_weight, k_weight
        # what a request checks: device (-1 for the host), dtype and length of each tensor
        self.tensors = [(t.get_device(), None if t is inv_freq else t.dtype,
                         None if t is inv_freq else t.shape[0])
                        for t in (inv_freq, q_weight, k_weight) if t is not None]
        self.s = CRope(_ptr(inv_freq), _ptr(q_weight), _ptr(k_weight), float(eps),
                       0 if inv_freq is None else 2 * inv_freq.shape[0], 1 if interleaved else 0)
        self.ref = ctypes.byref(self.s)


class Batch:
    """Device arrays of relaxkv_batch (views into one torch buffer)."""

    def __init__(self, req, buf, s, pad):
        self.buf, self.s, self.ref = buf, s, ctypes.byref(s)
        self.n_seq, self.n_rows, self.max_suffix = s.n_seq, s.n_rows, s.max_suffix
        self.key = (req.T_c, req.H, req.H_kv, req.d, req.dtype, req._index)
        self.suffix_shape = (s.n_seq, req.H_kv, s.max_suffix, req.d)
        self.flat = 1 in self.suffix_shape[:3]
        self.q_shape, self.lse_shape = (s.n_rows, req.H, req.d), (s.n_rows, req.H)
        base = buf.data_ptr()

        def view(ptr, n):
            off = ptr - base
            return buf[off:off + 4 * n].view(torch.int32)

        self.row_off = view(s.row_off, s.n_seq + 1)
        self.row_seq = view(s.row_seq, s.n_rows)
        self.row_pos = view(s.row_pos, s.n_rows)
        self.counts = view(s.counts, 4)

    def counts_to_host(self, stream=None, check=True):
        """[rows, row tiles, longest suffix, error word] of the planned step on the host; synchronises the
        stream.  With check=True a set error word raises RelaxKVError."""
        c = (c_int32 * 4)()
        st = load().relaxkv_batch_to_host(self.ref, c, _stream(stream))
        if check or st not in (OK, EINVAL):
            _check(st, "relaxkv_batch_to_host")
        return list(c)


class SetsBuffer:
    """Device arrays of relaxkv_sets (views into one torch buffer)."""

    def __init__(self, req, buf, s, pad):
        self.req, self.buf, self.s = req, buf, s
        L, T, k = req.L, req.T_c, req.k
        base = buf.data_ptr() + pad

        def view(ptr, n, dtype):
            off = ptr - base + pad
            esz = 8 if dtype == torch.int64 else 4
            return buf[off:off + n * esz].view(dtype)

        self.anchors = view(s.anchors, L * k, torch.int32).view(L, k)
        self.h = view(s.h, T, torch.int32)
        self.U = view(s.U, T, torch.int32)
        self.cidx = view(s.cidx, T, torch.int32)
        self.R_off = view(s.R_off, L + 1, torch.int32)
        self.R_idx = view(s.R_idx, L * T, torch.int32)
        self.R_u = view(s.R_u, L * T, torch.int32)
        self.src = view(s.src, L * T, torch.int32).view(L, T)
        self.rank = view(s.rank, L * T, torch.int32).view(L, T)
        self.counts = view(s.counts, L + 2, torch.int32)
        self.edges = view(s.edges, 2 * L, torch.int64)
        self.ctx = view(s.ctx, L * T, torch.int32).view(L, T)
        self.g = view(s.g, T, torch.float32)
        self.tiles = view(s.tiles, 2 * L * (req.H_kv + 1), torch.int32).view(2, L, req.H_kv + 1)

    def counts_to_host(self, stream=None, check=True):
        """(counts [L+2], edges [2L]) on the host; synchronises the stream.  With
        check=True a set device error word (counts[L+1], ERR_* bits) raises
        RelaxKVError; with check=False the counts are returned as they are."""
        L = self.req.L
        c = (c_int32 * (L + 2))()
        e = (c_int64 * (2 * L))()
        st = load().relaxkv_counts_to_host(ctypes.byref(self.s), c, e, _stream(stream))
        if check or st not in (OK, EINVAL):
            _check(st, "relaxkv_counts_to_host")
        return list(c), list(e)


def default_scale(d):
    return 1.0 / math.sqrt(d)
