"""Thin ctypes binding of libcosa.so: the C entry points under the same names.

Argument marshalling only: torch tensors supply device pointers (PyTorch is used for device memory
and streams), every computation runs in the library's HIP kernels. The binding raises if the
library was not built; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import re
from dataclasses import dataclass
from functools import cached_property
from typing import Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcosa.so")
HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "cosa.h")
DECODE_HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "cosa_decode.h")
SERVING_HEADER_PATH = os.path.join(os.path.dirname(_PKG), "include", "cosa_serving.h")

COSA_OK, COSA_ERR_INVALID_ARG, COSA_ERR_UNSUPPORTED, COSA_ERR_WORKSPACE, COSA_ERR_HIP = range(5)
SELECT_FRACTION, SELECT_TOP_P, SELECT_ALL = 0, 1, 2
ORDER_KAP, ORDER_ASCENDING = 0, 1
SKIP_NONE, SKIP_ROWMAX = 0, 1
VISIT_COMPUTED, VISIT_SKIPPED = 1, 2


class CosaProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
                ("stride", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("causal", ctypes.c_int32)]


class CosaSelect(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int), ("value", ctypes.c_float), ("order", ctypes.c_int)]


class CosaSkip(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int), ("delta", ctypes.c_float)]


class CosaWorkspaceLayout(ctypes.Structure):
    _fields_ = [("score", ctypes.c_size_t), ("hrm", ctypes.c_size_t), ("order", ctypes.c_size_t),
                ("count", ctypes.c_size_t), ("keys", ctypes.c_size_t), ("queue", ctypes.c_size_t),
                ("total", ctypes.c_size_t)]


class CosaPagedKv(ctypes.Structure):
    _fields_ = [("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int64)]


class CosaVarlen(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("cu_blocks", ctypes.POINTER(ctypes.c_int32))]


MAX_PACKED_SEQS = 128


class CosaDecodeProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("q_stride", ctypes.c_int64),
                ("sm_scale", ctypes.c_float)]


class CosaPageBudget(ctypes.Structure):
    _fields_ = [("fraction", ctypes.c_float), ("min_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("sink_pages", ctypes.c_int32),
                ("recent_pages", ctypes.c_int32)]


class CosaDecodeSparseLayout(ctypes.Structure):
    _fields_ = [("score", ctypes.c_size_t), ("pages", ctypes.c_size_t), ("count", ctypes.c_size_t),
                ("partial", ctypes.c_size_t), ("total", ctypes.c_size_t)]


class CosaChunkProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("sm_scale", ctypes.c_float)]


class CosaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


@dataclass(frozen=True)
class Problem:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    seq_len: int
    head_dim: int = 128
    block: int = 128
    stride: int = 16
    sm_scale: float = 0.0
    causal: int = 1

    @property
    def n_blocks(self) -> int:
        return -(-self.seq_len // self.block) if self.block > 0 else 0

    def c(self) -> CosaProblem:
        return CosaProblem(self.batch, self.n_q_heads, self.n_kv_heads, self.seq_len,
                           self.head_dim, self.block, self.stride, self.sm_scale, self.causal)


@dataclass(frozen=True)
class DecodeProblem:
    """One new token for each sequence of a batch (cosa_decode_problem). q_stride 0: the queries are
    dense, or a tensor passed as q brings its own stride."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    max_pages: int
    head_dim: int = 128
    q_stride: int = 0
    sm_scale: float = 0.0

    @cached_property
    def c(self) -> CosaDecodeProblem:
        return CosaDecodeProblem(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim,
                                 self.max_pages, self.q_stride, self.sm_scale)


@dataclass(frozen=True)
class ChunkProblem:
    """New tokens of a batch of sequences (cosa_chunk_problem): n_rows packed query rows. q_stride 0: they are
    dense, or a tensor passed as q brings its own stride."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    max_pages: int
    n_rows: int
    head_dim: int = 128
    q_stride: int = 0
    sm_scale: float = 0.0

    @cached_property
    def c(self) -> CosaChunkProblem:
        return CosaChunkProblem(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim,
                                self.max_pages, self.n_rows, self.q_stride, self.sm_scale)


_lib = None


def declared_symbols(header=None):
    """Names of the functions a header declares (include/cosa.h by default)."""
    text = open(header or HEADER_PATH).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\*?\s+\*?(cosa_[a-z_0-9]+)\(", text,
                                 re.M)))


def lib():
    """Load libcosa.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_25291_amd.build_lib`")
        # The library's HIP calls must bind to the HIP runtime that PyTorch loaded, so that the
        # tensors, streams and events it hands over belong to the same runtime. Importing torch
        # first puts that runtime in the process's global symbol scope, where the dynamic linker
        # resolves the library's HIP symbols; loaded the other way round, the library would start
        # a second HIP runtime of its own, which does not share torch's streams or device state.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        P, S, vp = ctypes.POINTER(CosaProblem), ctypes.c_int, ctypes.c_void_p
        L.cosa_status_string.restype = ctypes.c_char_p
        L.cosa_status_string.argtypes = [S]
        L.cosa_last_error.restype = ctypes.c_char_p
        L.cosa_last_error.argtypes = []
        L.cosa_kap_score.restype = S
        L.cosa_kap_score.argtypes = [P, vp, vp, vp, vp, vp]
        L.cosa_kap_select_ordered.restype = S
        L.cosa_kap_select_ordered.argtypes = [P, vp, vp, ctypes.POINTER(CosaSelect), vp, vp, vp]
        L.cosa_osk_attention.restype = S
        L.cosa_osk_attention.argtypes = [P, vp, vp, vp, vp, vp, ctypes.POINTER(CosaSkip), vp, vp,
                                         vp, vp, vp]
        L.cosa_osk_attention_queue_bytes.restype = ctypes.c_size_t
        L.cosa_osk_attention_queue_bytes.argtypes = []
        L.cosa_osk_attention_queued.restype = S
        L.cosa_osk_attention_queued.argtypes = [P, vp, vp, vp, vp, vp, ctypes.POINTER(CosaSkip), vp,
                                                vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.cosa_dense_attention.restype = S
        L.cosa_dense_attention.argtypes = [P, vp, vp, vp, vp, vp]
        L.cosa_prefill_workspace_bytes.restype = ctypes.c_size_t
        L.cosa_prefill_workspace_bytes.argtypes = [P]
        L.cosa_prefill_workspace_layout.restype = S
        L.cosa_prefill_workspace_layout.argtypes = [P, ctypes.POINTER(CosaWorkspaceLayout)]
        L.cosa_prefill.restype = S
        L.cosa_prefill.argtypes = [P, vp, vp, vp, ctypes.POINTER(CosaSelect),
                                   ctypes.POINTER(CosaSkip), vp, ctypes.c_size_t, vp, vp]
        L.cosa_prefill_noalloc.restype = S
        L.cosa_prefill_noalloc.argtypes = [P, vp, vp, vp, ctypes.POINTER(CosaSelect),
                                           ctypes.POINTER(CosaSkip), vp, vp]
        L.cosa_block_mass.restype = S
        L.cosa_block_mass.argtypes = [P, vp, vp, vp, vp]
        L.cosa_masked_attention.restype = S
        L.cosa_masked_attention.argtypes = [P, vp, vp, vp, vp, vp, vp]
        KV = ctypes.POINTER(CosaPagedKv)
        L.cosa_kap_score_paged.restype = S
        L.cosa_kap_score_paged.argtypes = [P, vp, KV, vp, vp, vp]
        L.cosa_osk_attention_paged.restype = S
        L.cosa_osk_attention_paged.argtypes = [P, vp, KV, vp, vp, ctypes.POINTER(CosaSkip), vp, vp,
                                               vp, vp, vp]
        L.cosa_prefill_paged.restype = S
        L.cosa_prefill_paged.argtypes = [P, vp, KV, ctypes.POINTER(CosaSelect),
                                         ctypes.POINTER(CosaSkip), vp, ctypes.c_size_t, vp, vp]
        L.cosa_kap_score_workspace_bytes.restype = ctypes.c_size_t
        L.cosa_kap_score_workspace_bytes.argtypes = [P]
        L.cosa_kap_score_staged.restype = S
        L.cosa_kap_score_staged.argtypes = [P, vp, vp, vp, ctypes.c_size_t, vp, vp, vp]
        VL = ctypes.POINTER(CosaVarlen)
        L.cosa_kap_score_varlen.restype = S
        L.cosa_kap_score_varlen.argtypes = [P, VL, vp, vp, vp, vp, vp]
        L.cosa_kap_select_ordered_varlen.restype = S
        L.cosa_kap_select_ordered_varlen.argtypes = [P, VL, vp, vp, ctypes.POINTER(CosaSelect), vp,
                                                     vp, vp]
        L.cosa_osk_attention_varlen.restype = S
        L.cosa_osk_attention_varlen.argtypes = [P, VL, vp, vp, vp, vp, vp, ctypes.POINTER(CosaSkip),
                                                vp, vp, vp, vp, vp]
        L.cosa_dense_attention_varlen.restype = S
        L.cosa_dense_attention_varlen.argtypes = [P, VL, vp, vp, vp, vp, vp]
        L.cosa_prefill_varlen.restype = S
        L.cosa_prefill_varlen.argtypes = [P, VL, vp, vp, vp, ctypes.POINTER(CosaSelect),
                                          ctypes.POINTER(CosaSkip), vp, ctypes.c_size_t, vp, vp]
        L.cosa_prefill_paged_varlen.restype = S
        L.cosa_prefill_paged_varlen.argtypes = [P, VL, vp, KV, ctypes.POINTER(CosaSelect),
                                                ctypes.POINTER(CosaSkip), vp, ctypes.c_size_t, vp,
                                                vp]
        D, PB = ctypes.POINTER(CosaDecodeProblem), ctypes.POINTER(CosaPageBudget)
        i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.cosa_page_map.restype = S
        L.cosa_page_map.argtypes = [i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp]
        L.cosa_kv_append.restype = S
        L.cosa_kv_append.argtypes = [i32, i32, i32, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp]
        L.cosa_page_score.restype = S
        L.cosa_page_score.argtypes = [D, vp, KV, vp, vp, vp, vp]
        L.cosa_page_select.restype = S
        L.cosa_page_select.argtypes = [D, i32, vp, vp, PB, vp, vp, vp]
        L.cosa_decode_workspace_bytes.restype = size
        L.cosa_decode_workspace_bytes.argtypes = [D]
        L.cosa_decode_attention.restype = S
        L.cosa_decode_attention.argtypes = [D, vp, KV, vp, vp, size, vp, vp, vp]
        L.cosa_decode_attention_listed.restype = S
        L.cosa_decode_attention_listed.argtypes = [D, vp, KV, vp, vp, vp, i32, vp, size, vp, vp, vp]
        L.cosa_decode_sparse_workspace_layout.restype = S
        L.cosa_decode_sparse_workspace_layout.argtypes = [D, PB,
                                                          ctypes.POINTER(CosaDecodeSparseLayout)]
        L.cosa_decode_sparse_workspace_bytes.restype = size
        L.cosa_decode_sparse_workspace_bytes.argtypes = [D, PB]
        L.cosa_decode_sparse.restype = S
        L.cosa_decode_sparse.argtypes = [D, vp, KV, vp, vp, PB, vp, size, vp, vp, vp]
        CH = ctypes.POINTER(CosaChunkProblem)
        L.cosa_chunk_workspace_bytes.restype = size
        L.cosa_chunk_workspace_bytes.argtypes = [CH]
        L.cosa_chunk_attention.restype = S
        L.cosa_chunk_attention.argtypes = [CH, vp, KV, vp, vp, vp, size, vp, vp, vp]
        L.cosa_page_fork.restype = S
        L.cosa_page_fork.argtypes = [i32, i32, i32, i32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cosa_page_copy.restype = S
        L.cosa_page_copy.argtypes = [i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.cosa_page_workspace_bytes.restype = size
        L.cosa_page_workspace_bytes.argtypes = [i64]
        L.cosa_page_release.restype = S
        L.cosa_page_release.argtypes = [i32, i32, i64, i32, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, size,
                                        vp]
        L.cosa_page_compact.restype = S
        L.cosa_page_compact.argtypes = [i32, i32, i32, i64, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, size, vp]
        _lib = L
    return _lib


def _check(status: int):
    if status != COSA_OK:
        raise CosaError(status, lib().cosa_last_error().decode())


def _ptr(t) -> Optional[int]:
    """Device pointer of a tensor (None -> NULL); integers are passed through as raw pointers."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("tensors must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _prob(problem) -> CosaProblem:
    return problem.c() if isinstance(problem, Problem) else problem


def select(mode: int = SELECT_FRACTION, value: float = 1.0, order: int = ORDER_KAP) -> CosaSelect:
    return CosaSelect(mode, value, order)


def skip(mode: int = SKIP_NONE, delta: float = 0.0) -> CosaSkip:
    return CosaSkip(mode, delta)


def cosa_status_string(status: int) -> str:
    return lib().cosa_status_string(status).decode()


def cosa_last_error() -> str:
    return lib().cosa_last_error().decode()


def cosa_kap_score(problem, q, k, score, hrm, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_score(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(score), _ptr(hrm),
                                _stream(stream)))


def cosa_kap_score_workspace_bytes(problem) -> int:
    p = _prob(problem)
    return int(lib().cosa_kap_score_workspace_bytes(ctypes.byref(p)))


def cosa_kap_score_staged(problem, q, k, workspace, workspace_bytes: int, score, hrm, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_score_staged(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(workspace),
                                       workspace_bytes, _ptr(score), _ptr(hrm), _stream(stream)))


def cosa_kap_select_ordered(problem, score, hrm, sel: CosaSelect, order, count, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_select_ordered(ctypes.byref(p), _ptr(score), _ptr(hrm), ctypes.byref(sel),
                                         _ptr(order), _ptr(count), _stream(stream)))


def cosa_osk_attention(problem, q, k, v, order, count, sk: Optional[CosaSkip], o, visit_log=None,
                       margin_log=None, n_computed=None, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_osk_attention(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(order),
                                    _ptr(count), skp, _ptr(o), _ptr(visit_log), _ptr(margin_log),
                                    _ptr(n_computed), _stream(stream)))


def cosa_osk_attention_queue_bytes() -> int:
    return int(lib().cosa_osk_attention_queue_bytes())


def cosa_osk_attention_queued(problem, q, k, v, order, count, sk: Optional[CosaSkip], o, queue,
                              queue_bytes: int, visit_log=None, margin_log=None, n_computed=None,
                              stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_osk_attention_queued(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(order),
                                           _ptr(count), skp, _ptr(o), _ptr(visit_log),
                                           _ptr(margin_log), _ptr(n_computed), _ptr(queue),
                                           queue_bytes, _stream(stream)))


def cosa_dense_attention(problem, q, k, v, o, stream=None):
    p = _prob(problem)
    _check(lib().cosa_dense_attention(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                      _stream(stream)))


def cosa_block_mass(problem, q, k, mass, stream=None):
    p = _prob(problem)
    _check(lib().cosa_block_mass(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(mass), _stream(stream)))


def cosa_masked_attention(problem, q, k, v, mask, o, stream=None):
    p = _prob(problem)
    _check(lib().cosa_masked_attention(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(mask),
                                       _ptr(o), _stream(stream)))


def cosa_prefill_workspace_bytes(problem) -> int:
    p = _prob(problem)
    n = lib().cosa_prefill_workspace_bytes(ctypes.byref(p))
    if n == 0 and not (p.batch == 0 or p.seq_len == 0):
        raise CosaError(COSA_ERR_INVALID_ARG, cosa_last_error())
    return n


def cosa_prefill_workspace_layout(problem) -> CosaWorkspaceLayout:
    p = _prob(problem)
    out = CosaWorkspaceLayout()
    _check(lib().cosa_prefill_workspace_layout(ctypes.byref(p), ctypes.byref(out)))
    return out


def cosa_prefill(problem, q, k, v, sel: CosaSelect, sk: Optional[CosaSkip], workspace,
                 workspace_bytes: int, o, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_prefill(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), ctypes.byref(sel), skp,
                              _ptr(workspace), workspace_bytes, _ptr(o), _stream(stream)))


NOALLOC_SCRATCH_BYTES = 128 * 1024 * 1024


def cosa_prefill_noalloc(problem, q, k, v, sel: CosaSelect, sk: Optional[CosaSkip], o,
                         stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_prefill_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v),
                                      ctypes.byref(sel), skp, _ptr(o), _stream(stream)))


def _kvref(kv):
    return ctypes.byref(kv) if kv is not None else None


def paged_kv(k_cache, v_cache, page_table, page_size: int, n_pages: int) -> CosaPagedKv:
    """cosa_paged_kv from device tensors (v_cache may be None for the proxy-only call)."""
    return CosaPagedKv(_ptr(k_cache), _ptr(v_cache), _ptr(page_table), page_size, n_pages)


def cosa_kap_score_paged(problem, q, kv: CosaPagedKv, score, hrm, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_score_paged(ctypes.byref(p), _ptr(q), _kvref(kv), _ptr(score),
                                      _ptr(hrm), _stream(stream)))


def cosa_osk_attention_paged(problem, q, kv: CosaPagedKv, order, count, sk: Optional[CosaSkip], o,
                             visit_log=None, margin_log=None, n_computed=None, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_osk_attention_paged(ctypes.byref(p), _ptr(q), _kvref(kv), _ptr(order),
                                          _ptr(count), skp, _ptr(o), _ptr(visit_log),
                                          _ptr(margin_log), _ptr(n_computed), _stream(stream)))


def cosa_prefill_paged(problem, q, kv: CosaPagedKv, sel: CosaSelect, sk: Optional[CosaSkip],
                       workspace, workspace_bytes: int, o, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_prefill_paged(ctypes.byref(p), _ptr(q), _kvref(kv), ctypes.byref(sel),
                                    skp, _ptr(workspace), workspace_bytes, _ptr(o),
                                    _stream(stream)))


def varlen(cu_blocks) -> CosaVarlen:
    """cosa_varlen from host block offsets [0, ..., nb] of the packed sequences (the struct keeps
    its own copy of the array alive)."""
    vals = [int(x) for x in cu_blocks]
    arr = (ctypes.c_int32 * max(len(vals), 1))(*vals)
    v = CosaVarlen(len(vals) - 1, ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)))
    v._host_offsets = arr
    return v


def _vlref(vl):
    return ctypes.byref(vl) if vl is not None else None


def cosa_kap_score_varlen(problem, vl: CosaVarlen, q, k, score, hrm, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_score_varlen(ctypes.byref(p), _vlref(vl), _ptr(q), _ptr(k), _ptr(score),
                                       _ptr(hrm), _stream(stream)))


def cosa_kap_select_ordered_varlen(problem, vl: CosaVarlen, score, hrm, sel: CosaSelect, order,
                                   count, stream=None):
    p = _prob(problem)
    _check(lib().cosa_kap_select_ordered_varlen(ctypes.byref(p), _vlref(vl), _ptr(score), _ptr(hrm),
                                                ctypes.byref(sel), _ptr(order), _ptr(count),
                                                _stream(stream)))


def cosa_osk_attention_varlen(problem, vl: CosaVarlen, q, k, v, order, count,
                              sk: Optional[CosaSkip], o, visit_log=None, margin_log=None,
                              n_computed=None, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_osk_attention_varlen(ctypes.byref(p), _vlref(vl), _ptr(q), _ptr(k), _ptr(v),
                                           _ptr(order), _ptr(count), skp, _ptr(o), _ptr(visit_log),
                                           _ptr(margin_log), _ptr(n_computed), _stream(stream)))


def cosa_dense_attention_varlen(problem, vl: CosaVarlen, q, k, v, o, stream=None):
    p = _prob(problem)
    _check(lib().cosa_dense_attention_varlen(ctypes.byref(p), _vlref(vl), _ptr(q), _ptr(k), _ptr(v),
                                             _ptr(o), _stream(stream)))


def cosa_prefill_varlen(problem, vl: CosaVarlen, q, k, v, sel: CosaSelect, sk: Optional[CosaSkip],
                        workspace, workspace_bytes: int, o, stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_prefill_varlen(ctypes.byref(p), _vlref(vl), _ptr(q), _ptr(k), _ptr(v),
                                     ctypes.byref(sel), skp, _ptr(workspace), workspace_bytes,
                                     _ptr(o), _stream(stream)))


def cosa_prefill_paged_varlen(problem, vl: CosaVarlen, q, kv: CosaPagedKv, sel: CosaSelect,
                              sk: Optional[CosaSkip], workspace, workspace_bytes: int, o,
                              stream=None):
    p = _prob(problem)
    skp = ctypes.byref(sk) if sk is not None else None
    _check(lib().cosa_prefill_paged_varlen(ctypes.byref(p), _vlref(vl), _ptr(q), _kvref(kv),
                                           ctypes.byref(sel), skp, _ptr(workspace),
                                           workspace_bytes, _ptr(o), _stream(stream)))


# ---- decode-side operators (include/cosa_decode.h)

def _place(stream, *tensors):
    """Stream of a call for _run (None: the current one of the device that holds the tensors) and the tensors'
    device pointers. They must be contiguous and share one device; None and raw pointers pass through."""
    device, out = None, []
    for t in tensors:
        if t is not None and t.__class__ is not int:
            d = t.get_device()
            if d != device:
                device = _same_device(d, device)
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
            t = t.data_ptr()
        out.append(t)
    return _stream_of(stream, device), out


def _same_device(d: int, device: Optional[int]) -> int:
    if d < 0:
        raise ValueError("tensors must live on the GPU")
    if device is not None and d != device:
        raise ValueError(f"tensors must live on one device, not on cuda:{device} and cuda:{d}")
    return d


def _raw_stream(device: int) -> int:
    # the handle alone: torch.cuda.current_stream() takes 1 us to build a Stream around it
    global _raw_stream
    import torch
    _raw_stream = torch._C._cuda_getCurrentRawStream
    return _raw_stream(device)


def _get_device() -> int:
    global _get_device
    import torch
    if not torch.cuda.is_available():
        return 0
    _get_device = torch._C._cuda_getDevice
    return _get_device()


def _stream_of(stream, device: Optional[int]):
    """A stream's handle, or (handle, device) where that device has to be made current for the call."""
    if device is None:
        return _stream(stream)
    if stream is None:
        handle = _raw_stream(device)
    elif isinstance(stream, int):
        handle = stream
    else:
        if stream.device.index != device:
            raise ValueError(f"the stream belongs to {stream.device}, the tensors to cuda:{device}")
        handle = stream.cuda_stream
    # the null stream, the legacy and the per-thread one are those of whichever device is current
    if handle <= 2 and device != _get_device():
        return handle, device
    return handle


def _run(call, on, *args):
    """Calls an entry point with its stream as the last argument."""
    if on.__class__ is tuple:
        import torch
        with torch.cuda.device(on[1]):
            status = call(*args, on[0])
    else:
        status = call(*args, on)
    if status:
        _check(status)


def _rows(t, stride: int, like=None, want=None):
    """Pointer and row stride (elements) of rows [n, heads, head_dim]: a tensor whose rows are dense
    but may lie apart, on the device of the tensor `like`, or a raw pointer with the given stride.
    want: the rows (at least), heads and head_dim that a call reads."""
    if t is None or isinstance(t, int):
        return t, stride
    d = t.get_device()
    if d < 0 or (like is not None and like.__class__ is not int and like.get_device() != d):
        _same_device(d, like.get_device() if d >= 0 else None)
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("rows must be [n, heads, head_dim]")
    n, heads, dim = shape
    if want is not None and (n < want[0] or heads != want[1] or dim != want[2] or t.element_size() != 2):
        raise ValueError(f"rows of {want[1]} heads of {want[2]} bf16 elements (or their bits), at least {want[0]} of "
                         f"them, expected; got {tuple(shape)} of {t.dtype}")
    row = heads * dim
    if not t.is_contiguous():
        apart, head, elem = t.stride()
        if (elem != 1 and dim > 1) or (head != dim and heads > 1):
            raise ValueError("rows must be dense in heads and head_dim")
        if n > 1:
            if apart < row:
                raise ValueError("rows must not overlap")
            row = apart
    if stride and stride != row and n > 1:
        raise ValueError(f"row stride {stride} given for a tensor with row stride {row}")
    return t.data_ptr(), row


def _dprob(problem, q=None, like=None):
    """C problem and query pointer; the query tensor's own row stride goes into the problem."""
    p = problem.c if isinstance(problem, DecodeProblem) else problem
    ptr, stride = _rows(q, p.q_stride, like, (p.batch, p.n_q_heads, p.head_dim))
    if stride != p.q_stride and stride != p.n_q_heads * p.head_dim:
        p = CosaDecodeProblem(p.batch, p.n_q_heads, p.n_kv_heads, p.head_dim, p.max_pages, stride,
                              p.sm_scale)
    return ctypes.byref(p), ptr


def page_budget(max_pages: int, min_pages: int = 1, fraction: float = 1.0, sink_pages: int = 1,
                recent_pages: int = 1) -> CosaPageBudget:
    """cosa_page_budget; by default up to max_pages pages of every sequence."""
    return CosaPageBudget(fraction, min_pages, max_pages, sink_pages, recent_pages)


def cosa_page_map(batch: int, page_size: int, max_pages: int, cached_lens, new_lens, free_pages,
                  free_capacity: int, n_free, page_table, seq_lens, cu_new, slots, max_new: int,
                  n_taken, stream=None):
    s, (cached, new, free, nf, table, lens, cu, sl, taken) = _place(
        stream, cached_lens, new_lens, free_pages, n_free, page_table, seq_lens, cu_new, slots, n_taken)
    _run(lib().cosa_page_map, s, batch, page_size, max_pages, cached, new, free, free_capacity, nf, table,
         lens, cu, sl, max_new, taken)


def cosa_kv_append(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, k_cache, v_cache,
                   bounds, n_tokens: int, k, v, slots, k_stride: int = 0, v_stride: int = 0,
                   stream=None):
    """k and v: [n_tokens (or more), n_kv_heads, head_dim] tensors, slices of a fused projection among them
    (their row strides are taken from the tensors)."""
    s, (kc, vc, b, sl) = _place(stream, k_cache, v_cache, bounds, slots)
    want = (n_tokens, n_kv_heads, head_dim)
    kp, k_stride = _rows(k, k_stride, k_cache, want)
    vp, v_stride = _rows(v, v_stride, k_cache, want)
    _run(lib().cosa_kv_append, s, n_kv_heads, head_dim, page_size, n_pages, kc, vc, b, n_tokens, kp,
         k_stride, vp, v_stride, sl)


def cosa_page_score(problem, q, kv: CosaPagedKv, bounds, seq_lens, score, stream=None):
    s, (b, lens, out) = _place(stream, bounds, seq_lens, score)
    p, qp = _dprob(problem, q, score)
    _run(lib().cosa_page_score, s, p, qp, _kvref(kv), b, lens, out)


def cosa_page_select(problem, page_size: int, seq_lens, score, budget: CosaPageBudget, pages, count,
                     stream=None):
    s, (lens, sc, pg, cnt) = _place(stream, seq_lens, score, pages, count)
    p, _ = _dprob(problem)
    _run(lib().cosa_page_select, s, p, page_size, lens, sc, _kvref(budget), pg, cnt)


def cosa_decode_workspace_bytes(problem) -> int:
    p, _ = _dprob(problem)
    n = int(lib().cosa_decode_workspace_bytes(p))
    if n == 0:
        raise CosaError(COSA_ERR_INVALID_ARG, cosa_last_error())
    return n


def cosa_decode_attention(problem, q, kv: CosaPagedKv, seq_lens, workspace, workspace_bytes: int, o,
                          lse=None, stream=None):
    s, (lens, ws, out, ls) = _place(stream, seq_lens, workspace, o, lse)
    p, qp = _dprob(problem, q, o)
    _run(lib().cosa_decode_attention, s, p, qp, _kvref(kv), lens, ws, workspace_bytes, out, ls)


def cosa_decode_attention_listed(problem, q, kv: CosaPagedKv, seq_lens, pages, count,
                                 list_pages: int, workspace, workspace_bytes: int, o, lse=None,
                                 stream=None):
    s, (lens, pg, cnt, ws, out, ls) = _place(stream, seq_lens, pages, count, workspace, o, lse)
    p, qp = _dprob(problem, q, o)
    _run(lib().cosa_decode_attention_listed, s, p, qp, _kvref(kv), lens, pg, cnt, list_pages, ws,
         workspace_bytes, out, ls)


def cosa_decode_sparse_workspace_layout(problem, budget: CosaPageBudget) -> CosaDecodeSparseLayout:
    p, _ = _dprob(problem)
    out = CosaDecodeSparseLayout()
    _check(lib().cosa_decode_sparse_workspace_layout(p, _kvref(budget), ctypes.byref(out)))
    return out


def cosa_decode_sparse_workspace_bytes(problem, budget: CosaPageBudget) -> int:
    return int(cosa_decode_sparse_workspace_layout(problem, budget).total)


def cosa_decode_sparse(problem, q, kv: CosaPagedKv, bounds, seq_lens, budget: CosaPageBudget,
                       workspace, workspace_bytes: int, o, lse=None, stream=None):
    s, (b, lens, ws, out, ls) = _place(stream, bounds, seq_lens, workspace, o, lse)
    p, qp = _dprob(problem, q, o)
    _run(lib().cosa_decode_sparse, s, p, qp, _kvref(kv), b, lens, _kvref(budget), ws, workspace_bytes,
         out, ls)


# ---- serving operators (include/cosa_serving.h)

def _cprob(problem, q=None, like=None):
    """C problem and query pointer; the query tensor's own row stride goes into the problem."""
    p = problem.c if isinstance(problem, ChunkProblem) else problem
    ptr, stride = _rows(q, p.q_stride, like, (p.n_rows, p.n_q_heads, p.head_dim))
    if stride != p.q_stride and stride != p.n_q_heads * p.head_dim:
        p = CosaChunkProblem(p.batch, p.n_q_heads, p.n_kv_heads, p.head_dim, p.max_pages, p.n_rows, stride,
                             p.sm_scale)
    return ctypes.byref(p), ptr


def cosa_chunk_workspace_bytes(problem) -> int:
    p, _ = _cprob(problem)
    n = int(lib().cosa_chunk_workspace_bytes(p))
    if n == 0:
        raise CosaError(COSA_ERR_INVALID_ARG, cosa_last_error())
    return n


def cosa_chunk_attention(problem, q, kv: CosaPagedKv, seq_lens, cu_new, workspace, workspace_bytes: int, o,
                         lse=None, stream=None):
    """q: [n_rows (or more), n_q_heads, head_dim], a slice of a fused projection among them."""
    s, (lens, cu, ws, out, ls) = _place(stream, seq_lens, cu_new, workspace, o, lse)
    p, qp = _cprob(problem, q, o)
    _run(lib().cosa_chunk_attention, s, p, qp, _kvref(kv), lens, cu, ws, workspace_bytes, out, ls)


def cosa_page_fork(n_parents: int, n_children: int, page_size: int, max_pages: int, parent, page_table, seq_lens,
                   copy_all: int, free_pages, free_capacity: int, n_free, new_table, new_lens, src, dst, rows, n_taken,
                   stream=None):
    s, (par, table, lens, free, nf, nt, nl, a, b, r, taken) = _place(
        stream, parent, page_table, seq_lens, free_pages, n_free, new_table, new_lens, src, dst, rows, n_taken)
    _run(lib().cosa_page_fork, s, n_parents, n_children, page_size, max_pages, par, table, lens, copy_all, free,
         free_capacity, nf, nt, nl, a, b, r, taken)


def cosa_page_copy(n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, k_cache, v_cache, bounds, src, dst, rows,
                   max_pairs: int, n_pairs, stream=None):
    s, (kc, vc, b, a, d, r, n) = _place(stream, k_cache, v_cache, bounds, src, dst, rows, n_pairs)
    _run(lib().cosa_page_copy, s, n_kv_heads, head_dim, page_size, n_pages, kc, vc, b, a, d, r, max_pairs, n)


def cosa_page_workspace_bytes(n_pages: int) -> int:
    n = int(lib().cosa_page_workspace_bytes(n_pages))
    if n == 0:
        raise CosaError(COSA_ERR_INVALID_ARG, cosa_last_error())
    return n


def cosa_page_release(page_size: int, max_pages: int, n_pages: int, old_batch: int, old_table, old_lens, new_batch: int,
                      new_table, new_lens, free_pages, free_capacity: int, n_free, n_taken, free_out, out_capacity: int,
                      n_free_out, workspace, workspace_bytes: int, stream=None):
    s, (ot, ol, nt, nl, free, nf, taken, out, nfo, ws) = _place(
        stream, old_table, old_lens, new_table, new_lens, free_pages, n_free, n_taken, free_out, n_free_out, workspace)
    _run(lib().cosa_page_release, s, page_size, max_pages, n_pages, old_batch, ot, ol, new_batch, nt, nl, free,
         free_capacity, nf, taken, out, out_capacity, nfo, ws, workspace_bytes)


def cosa_page_compact(batch: int, page_size: int, max_pages: int, n_pages: int, page_table, seq_lens, max_moves: int,
                      new_table, src, dst, n_moves, free_pages, free_capacity: int, n_free, workspace,
                      workspace_bytes: int, stream=None):
    s, (table, lens, nt, a, b, nm, free, nf, ws) = _place(
        stream, page_table, seq_lens, new_table, src, dst, n_moves, free_pages, n_free, workspace)
    _run(lib().cosa_page_compact, s, batch, page_size, max_pages, n_pages, table, lens, max_moves, nt, a, b, nm, free,
         free_capacity, nf, ws, workspace_bytes)
