"""ctypes binding of libprism.so — argument marshalling only.

Every function has the name of the C entry point it calls (include/prism.h).  PyTorch is
used for device memory (`torch.empty`) and the current HIP stream; all computation happens
inside the library's kernels.  There is no fallback: if the library is missing or a call
returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

# PRISM_LIBRARY names another build of the same library (the measurement-only variants that
# `python -m paper_2602_08426_amd.build --ablation` writes); there is still no fallback.
_LIB_PATH = os.environ.get("PRISM_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                            "libprism.so")
_lib: Optional[ctypes.CDLL] = None

PRISM_FLAG_NO_CALIBRATION = 1
PRISM_FLAG_BIDIRECTIONAL = 2
PRISM_FLAG_FORCE_DIAGONAL = 4
PRISM_FLAG_FORCE_SINK = 8
PRISM_FLAG_PAIR_KERNEL = 0x10000000
PRISM_FLAG_GENERAL_KERNEL = 0x20000000
PRISM_FLAG_STREAM_ONLY = 0x40000000
PRISM_MAX_SEGMENTS = 8
PRISM_ROPE_INTERLEAVED = 0
PRISM_ROPE_HALF = 1
PRISM_ROTATE_BACKWARD = 1
PRISM_CACHE_BF16 = 0
PRISM_CACHE_E4M3 = 1


class PrismError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _load().prism_status_string(status).decode()
        super().__init__(f"{where} failed with status {status}: {msg}")


class prism_params(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("seq_len", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block", ctypes.c_int32), ("d_high", ctypes.c_int32), ("d_low", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("flags", ctypes.c_uint32)]

    @property
    def n_blocks(self) -> int:
        return -(-self.seq_len // self.block)

    @property
    def words_per_row(self) -> int:
        return (self.n_blocks + 63) // 64


class prism_band(ctypes.Structure):
    _fields_ = [("n_segments", ctypes.c_int32), ("start", ctypes.c_int32 * PRISM_MAX_SEGMENTS),
                ("width", ctypes.c_int32 * PRISM_MAX_SEGMENTS)]


class prism_bands(ctypes.Structure):
    _fields_ = [("high", prism_band), ("low", prism_band)]


class prism_rope(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("position_offset", ctypes.c_int32),
                ("yarn_native_len", ctypes.c_int32), ("yarn_scale", ctypes.c_double),
                ("yarn_alpha", ctypes.c_double), ("yarn_beta", ctypes.c_double)]


class prism_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class prism_rotary(ctypes.Structure):
    _fields_ = [("freq", prism_rope), ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("magnitude", ctypes.c_float)]


class prism_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("page", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class prism_batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_tokens", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("cu_tokens", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p)]


class prism_cache_attn_params(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("scale", ctypes.c_float)]


EXPORTS = ("prism_version", "prism_status_string", "prism_estimate_workspace_bytes",
           "prism_estimate", "prism_estimate_static", "prism_estimate_bands", "prism_rope_estimate", "prism_block_scores",
           "prism_block_scores_bands", "prism_mask_to_csr", "prism_causal_csr", "prism_dense_csr",
           "prism_sparse_attn_workspace_bytes", "prism_sparse_attn", "prism_v_image",
           "prism_sparse_attn_pre", "prism_varlen_layout", "prism_estimate_varlen_workspace_bytes",
           "prism_estimate_varlen", "prism_sparse_attn_varlen_workspace_bytes", "prism_sparse_attn_varlen",
           "prism_rotate", "prism_cache_append", "prism_cache_attn_workspace_bytes", "prism_cache_attn")


def _load() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} not found: build it first (python -m paper_2602_08426_amd.build "
            "or __graft_entry__.build())")
    lib = ctypes.CDLL(_LIB_PATH)
    P, vp, i64, sz = ctypes.POINTER(prism_params), ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    PB = ctypes.POINTER(prism_bands)
    lib.prism_version.restype = ctypes.c_int
    lib.prism_version.argtypes = []
    lib.prism_status_string.restype = ctypes.c_char_p
    lib.prism_status_string.argtypes = [ctypes.c_int]
    lib.prism_estimate_workspace_bytes.argtypes = [P, ctypes.POINTER(sz)]
    lib.prism_estimate.argtypes = [P, vp, vp, vp, vp, vp, i64, vp, vp, sz, vp]
    lib.prism_estimate_static.argtypes = [P, vp, vp, vp, vp, vp, i64, vp, vp]
    lib.prism_estimate_bands.argtypes = [P, PB, vp, vp, vp, vp, vp, i64, vp, vp, sz, vp]
    lib.prism_rope_estimate.argtypes = [P, ctypes.POINTER(prism_rope), PB, vp, vp, vp, vp, vp, vp, vp,
                                        i64, vp, vp, sz, vp]
    lib.prism_block_scores.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.prism_block_scores_bands.argtypes = [P, PB, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.prism_dense_csr.argtypes = [P, vp, vp, i64, vp]
    lib.prism_mask_to_csr.argtypes = [P, vp, vp, vp, i64, vp, vp]
    lib.prism_causal_csr.argtypes = [P, vp, vp, i64, vp]
    lib.prism_sparse_attn_workspace_bytes.argtypes = [P, ctypes.POINTER(sz)]
    lib.prism_sparse_attn.argtypes = [P, vp, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.prism_v_image.argtypes = [P, vp, vp, sz, vp]
    lib.prism_sparse_attn_pre.argtypes = [P, vp, vp, vp, sz, vp, vp, i64, vp, vp, vp]
    I32P, I64P = ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64)
    lib.prism_varlen_layout.argtypes = [P, I32P, ctypes.c_int, I64P, I64P, I64P]
    lib.prism_estimate_varlen_workspace_bytes.argtypes = [P, I32P, ctypes.c_int, ctypes.POINTER(sz)]
    lib.prism_estimate_varlen.argtypes = [P, I32P, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.prism_sparse_attn_varlen_workspace_bytes.argtypes = [P, I32P, ctypes.c_int, ctypes.POINTER(sz)]
    lib.prism_sparse_attn_varlen.argtypes = [P, I32P, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    PR, PC, PT = ctypes.POINTER(prism_rows), ctypes.POINTER(prism_cache), ctypes.POINTER(prism_batch)
    PY, i32 = ctypes.POINTER(prism_rotary), ctypes.c_int
    lib.prism_rotate.argtypes = [PY, i32, i32, vp, i32, PR, PR, i32, PR, PR, ctypes.c_uint32, vp]
    lib.prism_cache_append.argtypes = [PC, PT, PY, PR, PR, i32, PR, PR, vp]
    lib.prism_cache_attn_workspace_bytes.argtypes = [PC, PT, i32, ctypes.POINTER(sz)]
    lib.prism_cache_attn.argtypes = [PC, PT, ctypes.POINTER(prism_cache_attn_params), PR, PR, vp, vp, sz, vp]
    for name in EXPORTS[2:]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def library_path() -> str:
    return _LIB_PATH


def make_params(n_q_heads: int, n_kv_heads: int, seq_len: int, block: int, d_high: int = 64,
                d_low: int = 96, top_p: float = 0.95, flags: int = 0, head_dim: int = 128) -> prism_params:
    return prism_params(n_q_heads, n_kv_heads, seq_len, head_dim, block, d_high, d_low, top_p, flags)


def make_bands(high, low) -> prism_bands:
    """Band descriptors from two lists of (start, width) slices of the head dim."""
    b = prism_bands()
    for band, segs in ((b.high, high), (b.low, low)):
        segs = list(segs)
        if len(segs) > PRISM_MAX_SEGMENTS:
            raise ValueError(f"at most {PRISM_MAX_SEGMENTS} slices per band")
        band.n_segments = len(segs)
        for i, (start, width) in enumerate(segs):
            band.start[i], band.width[i] = start, width
    return b


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


# handle of the current stream: the call behind torch.cuda.current_stream(), without the object around it (host time of a
# small call 14.3 -> 9 us together with the argument checks below reading each property once)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _check(status: int, where: str) -> None:
    if status != 0:
        raise PrismError(status, where)


def prism_version() -> int:
    return _load().prism_version()


def prism_status_string(status: int) -> str:
    return _load().prism_status_string(status).decode()


def prism_estimate_workspace_bytes(params: prism_params) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().prism_estimate_workspace_bytes(ctypes.byref(params), ctypes.byref(n)),
           "prism_estimate_workspace_bytes")
    return n.value


def prism_sparse_attn_workspace_bytes(params: prism_params) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().prism_sparse_attn_workspace_bytes(ctypes.byref(params), ctypes.byref(n)),
           "prism_sparse_attn_workspace_bytes")
    return n.value


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """256-byte aligned scratch (torch's caching allocator aligns to 512 B)."""
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def alloc_estimate_outputs(params: prism_params, col_capacity: Optional[int] = None, device="cuda"):
    N, W, h = params.n_blocks, params.words_per_row, params.n_q_heads
    if col_capacity is None:
        col_capacity = h * N * N if params.flags & PRISM_FLAG_BIDIRECTIONAL else h * N * (N + 1) // 2
    mask_bits = torch.empty((h, N, W), dtype=torch.int64, device=device)
    row_ptr = torch.empty(h * N + 1, dtype=torch.int32, device=device)
    col_idx = torch.empty(max(col_capacity, 1), dtype=torch.int32, device=device)
    info = torch.empty(4, dtype=torch.int32, device=device)
    return mask_bits, row_ptr, col_idx, info


def prism_estimate(params: prism_params, q: torch.Tensor, k: torch.Tensor, mask_bits: torch.Tensor,
                   row_ptr: torch.Tensor, col_idx: torch.Tensor, col_capacity: int,
                   info: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(_load().prism_estimate(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(mask_bits),
                                  _ptr(row_ptr), _ptr(col_idx), col_capacity, _ptr(info),
                                  _ptr(workspace), workspace.numel(), _stream()), "prism_estimate")


def prism_estimate_static(params: prism_params, q: torch.Tensor, k: torch.Tensor,
                          mask_bits: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                          col_capacity: int, info: torch.Tensor) -> None:
    _check(_load().prism_estimate_static(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(mask_bits),
                                         _ptr(row_ptr), _ptr(col_idx), col_capacity, _ptr(info),
                                         _stream()), "prism_estimate_static")


def prism_estimate_bands(params: prism_params, bands: prism_bands, q: torch.Tensor, k: torch.Tensor,
                         mask_bits: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                         col_capacity: int, info: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(_load().prism_estimate_bands(ctypes.byref(params), ctypes.byref(bands), _ptr(q), _ptr(k),
                                        _ptr(mask_bits), _ptr(row_ptr), _ptr(col_idx), col_capacity,
                                        _ptr(info), _ptr(workspace), workspace.numel(), _stream()),
           "prism_estimate_bands")


def make_rope(base: float, position_offset: int = 0, yarn_native_len: int = 0, yarn_scale: float = 1.0,
              yarn_alpha: float = 1.0, yarn_beta: float = 32.0) -> prism_rope:
    return prism_rope(base, position_offset, yarn_native_len, yarn_scale, yarn_alpha, yarn_beta)


def prism_rope_estimate(params: prism_params, rope: prism_rope, bands: Optional[prism_bands],
                        q_in: torch.Tensor, k_in: torch.Tensor, q_out: torch.Tensor, k_out: torch.Tensor,
                        mask_bits: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                        col_capacity: int, info: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(_load().prism_rope_estimate(ctypes.byref(params), ctypes.byref(rope),
                                       ctypes.byref(bands) if bands is not None else None,
                                       _ptr(q_in), _ptr(k_in), _ptr(q_out), _ptr(k_out), _ptr(mask_bits),
                                       _ptr(row_ptr), _ptr(col_idx), col_capacity, _ptr(info),
                                       _ptr(workspace), workspace.numel(), _stream()),
           "prism_rope_estimate")


def prism_block_scores(params: prism_params, q: torch.Tensor, k: torch.Tensor,
                       pooled_q: Optional[torch.Tensor], pooled_k: Optional[torch.Tensor],
                       scales: Optional[torch.Tensor], logits_high: Optional[torch.Tensor],
                       logits_low: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(_load().prism_block_scores(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(pooled_q),
                                      _ptr(pooled_k), _ptr(scales), _ptr(logits_high),
                                      _ptr(logits_low), _ptr(workspace), workspace.numel(),
                                      _stream()), "prism_block_scores")


def prism_block_scores_bands(params: prism_params, bands: prism_bands, q: torch.Tensor,
                             k: torch.Tensor, pooled_q: Optional[torch.Tensor],
                             pooled_k: Optional[torch.Tensor], scales: Optional[torch.Tensor],
                             logits_high: Optional[torch.Tensor], logits_low: Optional[torch.Tensor],
                             workspace: torch.Tensor) -> None:
    _check(_load().prism_block_scores_bands(ctypes.byref(params), ctypes.byref(bands), _ptr(q),
                                            _ptr(k), _ptr(pooled_q), _ptr(pooled_k), _ptr(scales),
                                            _ptr(logits_high), _ptr(logits_low), _ptr(workspace),
                                            workspace.numel(), _stream()), "prism_block_scores_bands")


def prism_mask_to_csr(params: prism_params, mask_bits: torch.Tensor, row_ptr: torch.Tensor,
                      col_idx: torch.Tensor, col_capacity: int, info: torch.Tensor) -> None:
    _check(_load().prism_mask_to_csr(ctypes.byref(params), _ptr(mask_bits), _ptr(row_ptr),
                                     _ptr(col_idx), col_capacity, _ptr(info), _stream()),
           "prism_mask_to_csr")


def prism_causal_csr(params: prism_params, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                     col_capacity: int) -> None:
    _check(_load().prism_causal_csr(ctypes.byref(params), _ptr(row_ptr), _ptr(col_idx),
                                    col_capacity, _stream()), "prism_causal_csr")


def prism_dense_csr(params: prism_params, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                    col_capacity: int) -> None:
    _check(_load().prism_dense_csr(ctypes.byref(params), _ptr(row_ptr), _ptr(col_idx),
                                   col_capacity, _stream()), "prism_dense_csr")


def prism_sparse_attn(params: prism_params, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      row_ptr: torch.Tensor, col_idx: torch.Tensor, col_count: int,
                      out: torch.Tensor, lse: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(_load().prism_sparse_attn(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v), _ptr(row_ptr),
                                     _ptr(col_idx), col_count, _ptr(out), _ptr(lse),
                                     _ptr(workspace), workspace.numel(), _stream()),
           "prism_sparse_attn")


def prism_v_image(params: prism_params, v: torch.Tensor, v_image: torch.Tensor) -> None:
    _check(_load().prism_v_image(ctypes.byref(params), _ptr(v), _ptr(v_image), v_image.numel(),
                                 _stream()), "prism_v_image")


def prism_sparse_attn_pre(params: prism_params, q: torch.Tensor, k: torch.Tensor,
                          v_image: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                          col_count: int, out: torch.Tensor, lse: Optional[torch.Tensor]) -> None:
    _check(_load().prism_sparse_attn_pre(ctypes.byref(params), _ptr(q), _ptr(k), _ptr(v_image),
                                         v_image.numel(), _ptr(row_ptr), _ptr(col_idx), col_count,
                                         _ptr(out), _ptr(lse), _stream()), "prism_sparse_attn_pre")


# ---- packed variable-length batches ---------------------------------------------------------
def _cu(cu_seqlens):
    """host int32 array of sequence offsets -> (ctypes array, number of sequences)"""
    vals = [int(x) for x in cu_seqlens]
    return (ctypes.c_int32 * len(vals))(*vals), len(vals) - 1


def prism_varlen_layout(params: prism_params, cu_seqlens):
    """(mask_offsets, row_offsets, col_offsets): lists of n_seqs + 1 ints, last = total."""
    cu, n = _cu(cu_seqlens)
    outs = [(ctypes.c_int64 * (n + 1))() for _ in range(3)]
    _check(_load().prism_varlen_layout(ctypes.byref(params), cu, n, *outs), "prism_varlen_layout")
    return tuple(list(o) for o in outs)


def prism_estimate_varlen_workspace_bytes(params: prism_params, cu_seqlens) -> int:
    cu, n = _cu(cu_seqlens)
    nb = ctypes.c_size_t(0)
    _check(_load().prism_estimate_varlen_workspace_bytes(ctypes.byref(params), cu, n, ctypes.byref(nb)),
           "prism_estimate_varlen_workspace_bytes")
    return nb.value


def prism_estimate_varlen(params: prism_params, cu_seqlens, q: torch.Tensor, k: torch.Tensor,
                          mask_bits: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                          info: torch.Tensor, workspace: torch.Tensor) -> None:
    cu, n = _cu(cu_seqlens)
    _check(_load().prism_estimate_varlen(ctypes.byref(params), cu, n, _ptr(q), _ptr(k), _ptr(mask_bits),
                                         _ptr(row_ptr), _ptr(col_idx), _ptr(info), _ptr(workspace),
                                         workspace.numel(), _stream()), "prism_estimate_varlen")


def prism_sparse_attn_varlen_workspace_bytes(params: prism_params, cu_seqlens) -> int:
    cu, n = _cu(cu_seqlens)
    nb = ctypes.c_size_t(0)
    _check(_load().prism_sparse_attn_varlen_workspace_bytes(ctypes.byref(params), cu, n, ctypes.byref(nb)),
           "prism_sparse_attn_varlen_workspace_bytes")
    return nb.value


def prism_sparse_attn_varlen(params: prism_params, cu_seqlens, q: torch.Tensor, k: torch.Tensor,
                             v: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                             out: torch.Tensor, lse: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    cu, n = _cu(cu_seqlens)
    _check(_load().prism_sparse_attn_varlen(ctypes.byref(params), cu, n, _ptr(q), _ptr(k), _ptr(v),
                                            _ptr(row_ptr), _ptr(col_idx), _ptr(out), _ptr(lse),
                                            _ptr(workspace), workspace.numel(), _stream()),
           "prism_sparse_attn_varlen")


# ---- serving: rotary positions, a paged cache, attention over it -------------------------------
def _on_current(t: torch.Tensor, dtype, what: str) -> None:
    if t.dtype is not dtype or not t.is_cuda:
        raise ValueError(f"{what}: expected a device tensor of {dtype}, got {t.dtype} on {t.device}")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{what} is on {t.device}, calls go to the current device, cuda:{torch.cuda.current_device()}")


def _rows(t: Optional[torch.Tensor], what: str, shape=None) -> Optional[prism_rows]:
    """[heads, tokens, d] bf16, contiguous in d, any strides of the library's in front"""
    if t is None:
        return None
    _on_current(t, torch.bfloat16, what)
    strides = t.stride()
    if len(strides) != 3 or (strides[2] != 1 and t.numel() > 0) or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: expected [heads, tokens, head_dim]" + (f" = {tuple(shape)}" if shape is not None else "") +
                         f" with a contiguous last axis, got {tuple(t.shape)} with strides {strides}")
    return prism_rows(t.data_ptr(), strides[0], strides[1])


def _dense(t: Optional[torch.Tensor], dtype, shape, what: str) -> Optional[int]:
    if t is None:
        return None
    _on_current(t, dtype, what)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor {tuple(shape)}, got {tuple(t.shape)} with strides {t.stride()}")
    return t.data_ptr()


def _ref(s: Optional[ctypes.Structure]):
    return ctypes.byref(s) if s is not None else None


def make_rotary(base: float, rot_dim: int, layout: int = PRISM_ROPE_INTERLEAVED, position_offset: int = 0,
                magnitude: float = 1.0, yarn_native_len: int = 0, yarn_scale: float = 1.0, yarn_alpha: float = 1.0,
                yarn_beta: float = 32.0) -> prism_rotary:
    return prism_rotary(make_rope(base, position_offset, yarn_native_len, yarn_scale, yarn_alpha, yarn_beta), rot_dim,
                        layout, magnitude)


def prism_rotate(rotary: prism_rotary, q_in: Optional[torch.Tensor], k_in: Optional[torch.Tensor],
                 q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor],
                 positions: Optional[torch.Tensor] = None, flags: int = 0) -> None:
    some = q_in if q_in is not None else k_in
    if some is None or (q_in is None) != (q_out is None) or (k_in is None) != (k_out is None):
        raise ValueError("prism_rotate: expected Q, K or both, each with its output")
    heads, tokens, d = [0, 0], *some.shape[1:]
    rows = []
    for i, (x, y, a, b) in enumerate(((q_in, q_out, "q_in", "q_out"), (k_in, k_out, "k_in", "k_out"))):
        if x is None:
            rows += [None, None]
            continue
        heads[i] = x.shape[0]
        shape = (heads[i], tokens, d)
        rows += [ctypes.byref(_rows(x, a, shape)), ctypes.byref(_rows(y, b, shape))]
    _check(_load().prism_rotate(ctypes.byref(rotary), d, tokens, _dense(positions, torch.int32, (tokens,), "positions"),
                                heads[0], rows[0], rows[1], heads[1], rows[2], rows[3], flags, _stream()), "prism_rotate")


def alloc_cache(n_pages: int, n_kv_heads: int, page: int, head_dim: int, dtype: int = PRISM_CACHE_BF16, device="cuda"):
    """(k, v, k_scale, v_scale) of a cache; the scales are None in bf16"""
    t = torch.float8_e4m3fn if dtype == PRISM_CACHE_E4M3 else torch.bfloat16
    k, v = (torch.empty((n_pages, n_kv_heads, page, head_dim), dtype=t, device=device) for _ in range(2))
    if dtype != PRISM_CACHE_E4M3:
        return k, v, None, None
    return k, v, *(torch.empty((n_pages, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2))


def make_cache(k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
               v_scale: Optional[torch.Tensor] = None) -> prism_cache:
    """Descriptor of a cache in tensors [n_pages, n_kv_heads, page, head_dim]; keeps them alive.  The pages of k and v may
    be apart by the same stride, as in one tensor [n_pages, 2, n_kv_heads, page, head_dim]."""
    if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
        raise ValueError(f"expected k and v [n_pages, n_kv_heads, page, head_dim] in bfloat16 or float8_e4m3fn, got "
                         f"{tuple(k.shape)} {k.dtype} and {tuple(v.shape)} {v.dtype}")
    n_pages, h_kv, page, d = k.shape
    for t, what in ((k, "k"), (v, "v")):
        _on_current(t, k.dtype, what)
        if any(n > 1 and a != b for n, a, b in zip(t.shape[1:], t.stride()[1:], (page * d, d, 1))):
            raise ValueError(f"{what}: the pages are contiguous [n_kv_heads, page, head_dim], got strides {t.stride()}")
    if n_pages > 1 and k.stride(0) != v.stride(0):
        raise ValueError(f"the pages of k and v lie {k.stride(0)} and {v.stride(0)} elements apart, expected the same")
    e4m3 = k.dtype == torch.float8_e4m3fn
    if e4m3 != (k_scale is not None) or e4m3 != (v_scale is not None):
        raise ValueError("k_scale and v_scale belong to a cache in float8_e4m3fn, and only there")
    c = prism_cache(k.data_ptr(), v.data_ptr(), _dense(k_scale, torch.float32, (n_pages, h_kv), "k_scale"),
                    _dense(v_scale, torch.float32, (n_pages, h_kv), "v_scale"), k.stride(0) if n_pages > 1 else 0, n_pages,
                    h_kv, page, d, PRISM_CACHE_E4M3 if e4m3 else PRISM_CACHE_BF16)
    c._keep, c._device = (k, v, k_scale, v_scale), k.get_device()
    return c


def make_batch(lengths: torch.Tensor, page_table: torch.Tensor, max_tokens: int = 1,
               cu_tokens: Optional[torch.Tensor] = None, n_tokens: Optional[int] = None) -> prism_batch:
    """Descriptor of a batch; keeps its int32 device tensors alive.  Without cu_tokens every sequence has max_tokens new
    tokens; with them n_tokens (rows of q, k, v and out) is given too."""
    n = lengths.numel()
    if page_table.dim() != 2 or page_table.shape[0] != n:
        raise ValueError(f"expected page_table [{n}, max_pages], got {tuple(page_table.shape)}")
    if cu_tokens is not None and n_tokens is None:
        raise ValueError("cu_tokens lives on the device: n_tokens has to be given with it")
    if cu_tokens is None and n_tokens not in (None, n * max_tokens):
        raise ValueError(f"{n} sequences of {max_tokens} new tokens are not {n_tokens}")
    b = prism_batch(n, n * max_tokens if cu_tokens is None else n_tokens, max_tokens, page_table.shape[1],
                    _dense(cu_tokens, torch.int32, (n + 1,), "cu_tokens"), _dense(lengths, torch.int32, (n,), "lengths"),
                    _dense(page_table, torch.int32, page_table.shape, "page_table"))
    b._keep, b._device = (lengths, page_table, cu_tokens), lengths.get_device()
    return b


def _made_on_current(cache: prism_cache, batch: prism_batch) -> None:
    here = torch._C._cuda_getDevice()
    for s, what in ((cache, "cache"), (batch, "batch")):
        if getattr(s, "_device", here) != here:          # descriptors filled in by hand have none
            raise ValueError(f"the {what} is on cuda:{s._device}, calls go to the current device, cuda:{here}")


def prism_cache_append(cache: prism_cache, batch: prism_batch, rotary: Optional[prism_rotary], k: torch.Tensor,
                       v: torch.Tensor, q_in: Optional[torch.Tensor] = None,
                       q_out: Optional[torch.Tensor] = None) -> None:
    _made_on_current(cache, batch)
    kv = (cache.n_kv_heads, batch.n_tokens, cache.head_dim)
    heads = 0 if q_in is None else q_in.shape[0]
    q = (heads, batch.n_tokens, cache.head_dim)
    _check(_load().prism_cache_append(ctypes.byref(cache), ctypes.byref(batch), _ref(rotary), _ref(_rows(k, "k", kv)),
                                      _ref(_rows(v, "v", kv)), heads, _ref(_rows(q_in, "q_in", q)),
                                      _ref(_rows(q_out, "q_out", q)), _stream()), "prism_cache_append")


def prism_cache_attn_workspace_bytes(cache: prism_cache, batch: prism_batch, n_q_heads: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().prism_cache_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), n_q_heads, ctypes.byref(n)),
           "prism_cache_attn_workspace_bytes")
    return n.value


def prism_cache_attn(cache: prism_cache, batch: prism_batch, q: torch.Tensor, out: torch.Tensor,
                     lse: Optional[torch.Tensor], workspace: torch.Tensor, window: int = 0, sinks: int = 0,
                     scale: float = 0.0) -> None:
    _made_on_current(cache, batch)
    _on_current(workspace, workspace.dtype, "workspace")
    heads = q.shape[0]
    shape = (heads, batch.n_tokens, cache.head_dim)
    params = prism_cache_attn_params(heads, window, sinks, scale)
    _check(_load().prism_cache_attn(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(params),
                                    _ref(_rows(q, "q", shape)), _ref(_rows(out, "out", shape)),
                                    _dense(lse, torch.float32, shape[:2], "lse"), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream()), "prism_cache_attn")


# ---- conveniences for callers holding numpy bf16 bit patterns --------------------------
def bf16_bits_to_device(bits, device="cuda") -> torch.Tensor:
    """numpy uint16 bf16 bit patterns -> device bf16 tensor (a copy, no arithmetic)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def device_bf16_to_bits(t: torch.Tensor):
    """device bf16 tensor -> numpy uint16 bit patterns."""
    import numpy as np
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
