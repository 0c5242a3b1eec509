"""Python binding of libdessert_hip.so (the C ABI declared in include/dessert.h).

Argument marshalling only: torch supplies device memory and the HIP stream,
every step of hashing, scoring and top-k runs in the library's gfx950 kernels.
There is no CPU path: loading fails loudly if the shared library has not been
built (run ``python -m paper_2210_15748_amd.build`` or ``__graft_entry__.build()``).

Function names mirror the C entry points without the ``dessert_`` prefix:
``create`` / ``destroy`` / ``hash`` / ``build_index`` / ``search`` / ``scores`` /
``set_algo`` / ``set_score_transform`` / ``get_projection`` / ``enable_timing`` / ``get_timing``, and beside the
search ``quantize_rows`` / ``scaled_matmul`` / ``token_logprobs`` / ``head_logprobs``, and on the paged cache of a reading model
``cache`` / ``cache_batch`` (what the calls take) with ``cache_append`` / ``cache_attention`` / ``cache_select`` / ``cache_advance`` /
``cache_compact``.
"""
from __future__ import annotations

import ctypes as C
import os
import pathlib
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = pathlib.Path(__file__).resolve().parent
LIB_PATH = _HERE / "libdessert_hip.so"

OK, EINVAL, ENOMEM, EHIP, ESTATE = range(5)
I8, F16, BF16, F32 = 0, 1, 2, 3
SCALE_MAXABS, SCALE_UNIT = 0, 1
PROJ_RADEMACHER_I8, PROJ_GAUSSIAN_F32 = 0, 1
HASH_AUTO, HASH_SCALAR, HASH_MFMA = 0, 1, 2
SCORE_AUTO, SCORE_BYTECMP, SCORE_MASKLUT = 0, 1, 2

SCORE_RAW_COUNTS, SCORE_EQ1_Q16 = 0, 1
SCORE_MAX_IDENTITY_Q16, SCORE_MAX_EXPM1_Q16, SCORE_MAX_SIGMOID_Q16 = 2, 3, 4
SCORE_MEAN_IDENTITY_Q16, SCORE_MEAN_EXPM1_Q16, SCORE_MEAN_SIGMOID_Q16 = 5, 6, 7

EXPORTS = [
    "dessert_create", "dessert_destroy", "dessert_get_projection", "dessert_set_algo", "dessert_set_score_transform",
    "dessert_set_query_weights",
    "dessert_code_bytes",
    "dessert_hash", "dessert_build_index", "dessert_attach_index", "dessert_search_workspace_bytes", "dessert_search", "dessert_scores",
    "dessert_noalloc_scratch_bytes", "dessert_search_noalloc", "dessert_set_debug", "dessert_last_score_kernel",
    "dessert_filter_kmeans_workspace_bytes", "dessert_filter_kmeans",
    "dessert_filter_build", "dessert_filter_workspace_bytes", "dessert_filter_query",
    "dessert_filter_search_workspace_bytes", "dessert_filter_search",
    "dessert_quantize_rows", "dessert_scaled_matmul_workspace_bytes", "dessert_scaled_matmul",
    "dessert_token_logprobs_workspace_bytes", "dessert_token_logprobs",
    "dessert_head_logprobs_workspace_bytes", "dessert_head_logprobs",
    "dessert_cache_append", "dessert_cache_attention_workspace_bytes", "dessert_cache_attention",
    "dessert_cache_select_workspace_bytes", "dessert_cache_select", "dessert_cache_advance_workspace_bytes", "dessert_cache_advance",
    "dessert_cache_compact_workspace_bytes", "dessert_cache_compact",
    "dessert_enable_timing", "dessert_get_timing", "dessert_probe_read_bandwidth", "dessert_probe_mix_bandwidth", "dessert_last_error",
    "dessert_version",
]


class Config(C.Structure):
    _fields_ = [("d", C.c_uint32), ("L", C.c_uint32), ("C", C.c_uint32), ("dtype", C.c_uint32),
                ("proj_kind", C.c_uint32), ("device", C.c_int32), ("seed", C.c_uint64),
                ("proj_dev", C.c_void_p), ("stream", C.c_void_p)]


class _CacheStruct(C.Structure):
    _fields_ = [("k_codes_dev", C.c_void_p), ("v_codes_dev", C.c_void_p), ("k_scales_dev", C.c_void_p), ("v_scales_dev", C.c_void_p),
                ("bounds_dev", C.c_void_p), ("n_pages", C.c_uint32), ("n_heads", C.c_uint32), ("page_tokens", C.c_uint32), ("dim", C.c_uint32)]


class _BatchStruct(C.Structure):
    _fields_ = [("tables_dev", C.c_void_p), ("lengths_dev", C.c_void_p), ("starts_dev", C.c_void_p), ("n_seqs", C.c_uint32),
                ("table_pages", C.c_uint32), ("n_tokens", C.c_uint32), ("max_tokens", C.c_uint32), ("max_length", C.c_uint32)]


class DessertError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"dessert status {status}: {message}")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    """Load the shared library (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2210_15748_amd.build`; "
                          "there is no fallback implementation")
    l = C.CDLL(os.fspath(LIB_PATH))
    vp, u32, u64, sz = C.c_void_p, C.c_uint32, C.c_uint64, C.c_size_t
    l.dessert_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    l.dessert_destroy.argtypes = [vp]
    l.dessert_destroy.restype = None
    l.dessert_get_projection.argtypes = [vp, vp]
    l.dessert_set_algo.argtypes = [vp, C.c_int, C.c_int]
    l.dessert_set_score_transform.argtypes = [vp, C.c_int]
    l.dessert_set_query_weights.argtypes = [vp, vp, u64]
    l.dessert_code_bytes.argtypes = [vp, u64]
    l.dessert_code_bytes.restype = sz
    l.dessert_hash.argtypes = [vp, vp, u64, vp]
    l.dessert_build_index.argtypes = [vp, vp, u64, vp, u64, vp, vp]
    l.dessert_attach_index.argtypes = [vp, vp, vp, u64, u64, u64]
    l.dessert_search_workspace_bytes.argtypes = [vp, u32, u64, u64, u32]
    l.dessert_search_workspace_bytes.restype = sz
    l.dessert_search.argtypes = [vp, vp, vp, u32, vp, vp, u32, vp, sz, vp, vp]
    l.dessert_scores.argtypes = [vp, vp, vp, u32, vp, vp, vp, sz, vp]
    l.dessert_noalloc_scratch_bytes.argtypes = []
    l.dessert_noalloc_scratch_bytes.restype = sz
    l.dessert_search_noalloc.argtypes = [vp, vp, u32, u32, vp, u64, u32, vp, vp]
    l.dessert_set_debug.argtypes = [vp, C.c_int]
    l.dessert_last_score_kernel.argtypes = [vp]
    l.dessert_last_score_kernel.restype = C.c_char_p
    l.dessert_filter_kmeans_workspace_bytes.argtypes = [vp, u64, u32]
    l.dessert_filter_kmeans_workspace_bytes.restype = sz
    l.dessert_filter_kmeans.argtypes = [vp, vp, u64, vp, u32, u32, vp, sz]
    l.dessert_filter_build.argtypes = [vp, vp, u32, vp, vp, vp, vp]
    l.dessert_filter_workspace_bytes.argtypes = [vp, u32, u64, u32, u32]
    l.dessert_filter_workspace_bytes.restype = sz
    l.dessert_filter_query.argtypes = [vp, vp, vp, u32, u32, u32, vp, sz, vp, vp]
    l.dessert_filter_search_workspace_bytes.argtypes = [vp, u32, u64, u32, u32, u32, u32]
    l.dessert_filter_search_workspace_bytes.restype = sz
    l.dessert_filter_search.argtypes = [vp, vp, vp, u32, u32, u32, u32, vp, sz, vp, vp]
    l.dessert_quantize_rows.argtypes = [vp, vp, u32, u64, u32, u64, C.c_int, vp, vp]
    l.dessert_scaled_matmul_workspace_bytes.argtypes = [vp, u64, u64, u32]
    l.dessert_scaled_matmul_workspace_bytes.restype = sz
    l.dessert_scaled_matmul.argtypes = [vp, vp, u64, vp, u64, vp, u64, vp, vp, u64, u32, u32, vp, u64, vp, sz]
    l.dessert_token_logprobs_workspace_bytes.argtypes = [vp, u64, u32, u32]
    l.dessert_token_logprobs_workspace_bytes.restype = sz
    l.dessert_token_logprobs.argtypes = [vp, vp, u32, u64, u32, u64, vp, u32, vp, sz, vp, vp, vp, vp]
    l.dessert_head_logprobs_workspace_bytes.argtypes = [vp, u64, u32, u32, u32]
    l.dessert_head_logprobs_workspace_bytes.restype = sz
    l.dessert_head_logprobs.argtypes = [vp, vp, u64, vp, u64, vp, u64, vp, u32, u32, vp, u32, vp, sz, vp, vp, vp, vp]
    l.dessert_cache_append.argtypes = [vp, vp, vp, vp, u64, vp, u64, u32]
    l.dessert_cache_attention_workspace_bytes.argtypes = [vp, vp, vp, u32, u32]
    l.dessert_cache_attention_workspace_bytes.restype = sz
    l.dessert_cache_attention.argtypes = [vp, vp, vp, vp, u32, u64, u32, C.c_float, u32, vp, u32, vp, sz, vp, vp]
    l.dessert_cache_select_workspace_bytes.argtypes = [vp, vp, vp]
    l.dessert_cache_select_workspace_bytes.restype = sz
    l.dessert_cache_select.argtypes = [vp, vp, vp, vp, vp, u32, u32, u32, u32, vp, sz, vp]
    l.dessert_cache_advance_workspace_bytes.argtypes = [vp, u32, u32]
    l.dessert_cache_advance_workspace_bytes.restype = sz
    l.dessert_cache_advance.argtypes = [vp, vp, u32, vp, vp, u32, vp, u32, vp, vp, u32, vp, sz, vp, vp, vp]
    l.dessert_cache_compact_workspace_bytes.argtypes = [vp, u32]
    l.dessert_cache_compact_workspace_bytes.restype = sz
    l.dessert_cache_compact.argtypes = [vp, vp, u32, vp, vp, u32, vp, u32, vp, sz, vp, vp]
    l.dessert_enable_timing.argtypes = [vp, C.c_int]
    l.dessert_get_timing.argtypes = [vp, u32, C.POINTER(C.c_float)]
    l.dessert_probe_read_bandwidth.argtypes = [vp, sz, C.c_int, vp, C.c_int, C.POINTER(C.c_float)]
    l.dessert_probe_mix_bandwidth.argtypes = [vp, vp, sz, C.c_int, vp, C.c_int, C.POINTER(C.c_float)]
    l.dessert_last_error.restype = C.c_char_p
    l.dessert_version.restype = C.c_char_p
    _lib = l
    return l


def last_error() -> str:
    return lib().dessert_last_error().decode()


def version() -> str:
    return lib().dessert_version().decode()


def _check(status: int):
    if status != OK:
        raise DessertError(status, last_error())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _host_u32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a.cpu() if isinstance(a, torch.Tensor) else a), dtype=np.uint32)


def _host_u64(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a.cpu() if isinstance(a, torch.Tensor) else a), dtype=np.uint64)


class Index:
    """Owner of one dessert_index_t handle plus the torch buffers the index lives in."""

    def __init__(self, handle: int, cfg: Config, device: torch.device):
        self.handle = handle
        self.cfg = cfg
        self.device = device
        self.codes: Optional[torch.Tensor] = None
        self.offsets: Optional[torch.Tensor] = None
        self.n_docs = 0
        self._keep = []

    def __del__(self):
        try:
            destroy(self)
        except Exception:
            pass


def create(d: int, L: int, C_bits: int, dtype: int = I8, proj_kind: int = PROJ_RADEMACHER_I8,
           proj: Optional[torch.Tensor] = None, seed: int = 0, device: Optional[torch.device] = None,
           stream: Optional[torch.cuda.Stream] = None) -> Index:
    """dessert_create.  ``proj``: device tensor [L*C, d] (int8 or float32) or None (seed-derived)."""
    if device is None:
        device = proj.device if proj is not None else torch.device("cuda", torch.cuda.current_device())
    device = torch.device(device)
    dev_index = device.index if device.index is not None else torch.cuda.current_device()
    if stream is None:
        stream = torch.cuda.current_stream(device)
    cfg = Config(d=d, L=L, C=C_bits, dtype=dtype, proj_kind=proj_kind, device=dev_index, seed=seed,
                 proj_dev=_ptr(proj.contiguous() if proj is not None else None), stream=stream.cuda_stream)
    if proj is not None:
        want = torch.int8 if proj_kind == PROJ_RADEMACHER_I8 else torch.float32
        if proj.dtype != want or tuple(proj.shape) != (L * C_bits, d) or not proj.is_cuda:
            raise ValueError("proj must be a device tensor [L*C, d] of dtype " + str(want))
    handle = C.c_void_p()
    _check(lib().dessert_create(C.byref(cfg), C.byref(handle)))
    return Index(handle.value, cfg, torch.device("cuda", dev_index))


def destroy(ix: Index) -> None:
    if ix.handle:
        lib().dessert_destroy(ix.handle)
        ix.handle = None


def set_algo(ix: Index, hash_algo: int = HASH_AUTO, score_algo: int = SCORE_AUTO) -> None:
    _check(lib().dessert_set_algo(ix.handle, hash_algo, score_algo))


def set_score_transform(ix: Index, transform: int) -> None:
    _check(lib().dessert_set_score_transform(ix.handle, transform))


def set_query_weights(ix: Index, weights: Optional[torch.Tensor]) -> None:
    """dessert_set_query_weights: a device tensor of Q16 weights (uint32 / int32 values in 0..65536), one per query
    vector of the following batches, or None."""
    if weights is None:
        ix._weights = None
        _check(lib().dessert_set_query_weights(ix.handle, None, 0))
        return
    if not weights.is_cuda or weights.dtype not in (torch.int32, torch.uint32) or weights.dim() != 1:
        raise ValueError("weights must be a 1-d device tensor of int32 / uint32")
    ix._weights = weights.contiguous()
    _check(lib().dessert_set_query_weights(ix.handle, ix._weights.data_ptr(), ix._weights.numel()))


def get_projection(ix: Index) -> torch.Tensor:
    dt = torch.int8 if ix.cfg.proj_kind == PROJ_RADEMACHER_I8 else torch.float32
    out = torch.empty(ix.cfg.L * ix.cfg.C, ix.cfg.d, dtype=dt, device=ix.device)
    _check(lib().dessert_get_projection(ix.handle, out.data_ptr()))
    return out


def _check_vectors(ix: Index, v: torch.Tensor) -> torch.Tensor:
    want = torch.int8 if ix.cfg.dtype == I8 else torch.float16
    if not v.is_cuda or v.dtype != want or v.dim() != 2 or v.shape[1] != ix.cfg.d:
        raise ValueError(f"vectors must be a device tensor [n, {ix.cfg.d}] of dtype {want}")
    return v.contiguous()


def code_dtype(ix: Index) -> torch.dtype:
    """Element type of the code arrays: uint8, or uint16 when C > 8."""
    return torch.uint16 if ix.cfg.C > 8 else torch.uint8


def hash(ix: Index, vectors: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:  # noqa: A001
    """dessert_hash: codes [n, L] of code_dtype(ix)."""
    vectors = _check_vectors(ix, vectors)
    n = vectors.shape[0]
    if out is None:
        out = torch.empty(n, ix.cfg.L, dtype=code_dtype(ix), device=ix.device)
    _check(lib().dessert_hash(ix.handle, vectors.data_ptr(), n, out.data_ptr()))
    return out


def build_index(ix: Index, vectors: torch.Tensor, lengths, codes: Optional[torch.Tensor] = None,
                offsets: Optional[torch.Tensor] = None):
    """dessert_build_index.  Returns (codes [V, L] of code_dtype(ix), offsets [N+1] int64), both on the device."""
    vectors = _check_vectors(ix, vectors)
    lens = _host_u32(lengths)
    n_docs, V = lens.shape[0], vectors.shape[0]
    if codes is None:
        codes = torch.empty(V, ix.cfg.L, dtype=code_dtype(ix), device=ix.device)
    if offsets is None:
        offsets = torch.empty(n_docs + 1, dtype=torch.int64, device=ix.device)
    _check(lib().dessert_build_index(ix.handle, vectors.data_ptr(), V, lens.ctypes.data, n_docs,
                                     codes.data_ptr(), offsets.data_ptr()))
    ix.codes, ix.offsets, ix.n_docs = codes, offsets, n_docs
    return codes, offsets


def attach_index(ix: Index, codes: torch.Tensor, offsets: torch.Tensor, max_length: Optional[int] = None) -> None:
    """dessert_attach_index: make arrays written by an earlier build_index (same configuration and projection matrix) this
    handle's index.  max_length (longest document) is computed from the offsets if not given."""
    if not codes.is_cuda or not offsets.is_cuda or offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1:
        raise ValueError("codes and offsets must be device tensors, offsets int64 [n_docs + 1]")
    if codes.dtype != code_dtype(ix) or codes.dim() != 2 or codes.shape[1] != ix.cfg.L:
        raise ValueError(f"codes must be [n_vectors, {ix.cfg.L}] of {code_dtype(ix)}")
    codes, offsets = codes.contiguous(), offsets.contiguous()
    n_docs = offsets.numel() - 1
    if max_length is None:
        max_length = int((offsets[1:] - offsets[:-1]).max().item()) if n_docs else 0
    _check(lib().dessert_attach_index(ix.handle, codes.data_ptr(), offsets.data_ptr(), n_docs, codes.shape[0], max_length))
    ix.codes, ix.offsets, ix.n_docs = codes, offsets, n_docs


def _batch(ix: Index, q_vectors, q_lengths, cand_ids, cand_offsets):
    q_vectors = _check_vectors(ix, q_vectors)
    ql = _host_u32(q_lengths)
    B = ql.shape[0]
    if int(ql.sum()) != q_vectors.shape[0]:
        raise ValueError("sum(q_lengths) != number of query vectors")
    if cand_ids is not None:
        if cand_ids.dim() == 2 and cand_offsets is None:
            cand_offsets = np.arange(B + 1, dtype=np.uint64) * cand_ids.shape[1]
        if cand_ids.dtype != torch.int32 and cand_ids.dtype != torch.uint32:
            cand_ids = cand_ids.to(torch.int32)
        cand_ids = cand_ids.contiguous().reshape(-1)
        co = _host_u64(cand_offsets)
        if co.shape[0] != B + 1 or int(co[-1]) != cand_ids.numel():
            raise ValueError("cand_offsets must have n_queries+1 entries ending at len(cand_ids)")
        total = int(co[-1])
    else:
        co = None
        total = B * ix.n_docs
    return q_vectors, ql, B, cand_ids, co, total


def workspace_bytes(ix: Index, n_queries: int, total_q_vectors: int, total_scored: int, k: int) -> int:
    return int(lib().dessert_search_workspace_bytes(ix.handle, n_queries, total_q_vectors, total_scored, k))


def search(ix: Index, q_vectors: torch.Tensor, q_lengths, k: int, cand_ids: Optional[torch.Tensor] = None,
           cand_offsets=None, workspace: Optional[torch.Tensor] = None, out_ids: Optional[torch.Tensor] = None,
           out_scores: Optional[torch.Tensor] = None):
    """dessert_search.  Returns (ids [B, k] int64 view of uint32, scores [B, k] int32)."""
    q_vectors, ql, B, cand_ids, co, total = _batch(ix, q_vectors, q_lengths, cand_ids, cand_offsets)
    if workspace is None:
        workspace = torch.empty(workspace_bytes(ix, B, q_vectors.shape[0], total, k), dtype=torch.uint8,
                                device=ix.device)
    if out_ids is None:
        out_ids = torch.empty(B, k, dtype=torch.uint32, device=ix.device)
    if out_scores is None:
        out_scores = torch.empty(B, k, dtype=torch.int32, device=ix.device)
    _check(lib().dessert_search(ix.handle, q_vectors.data_ptr(), ql.ctypes.data, B, _ptr(cand_ids),
                                None if co is None else co.ctypes.data, k, workspace.data_ptr(), workspace.numel(),
                                out_ids.data_ptr(), out_scores.data_ptr()))
    return out_ids, out_scores


def search_noalloc(ix: Index, q_vectors: torch.Tensor, q_length: int, k: int, cand_ids: Optional[torch.Tensor] = None,
                   out_ids: Optional[torch.Tensor] = None, out_scores: Optional[torch.Tensor] = None):
    """dessert_search_noalloc: query sets of q_length vectors each, candidate lists [B, cand_length] (or None: every
    document); the library's built-in scratch array is the workspace.  Outputs are allocated here only if not given."""
    q_vectors = _check_vectors(ix, q_vectors)
    if q_length <= 0 or q_vectors.shape[0] % q_length:
        raise ValueError("the number of query vectors must be a multiple of q_length")
    B = q_vectors.shape[0] // q_length
    cand_len = 0
    if cand_ids is not None:
        if cand_ids.dim() != 2 or cand_ids.shape[0] != B or cand_ids.dtype not in (torch.int32, torch.uint32):
            raise ValueError("cand_ids must be a device tensor [B, cand_length] of int32 / uint32")
        cand_ids = cand_ids.contiguous()
        cand_len = cand_ids.shape[1]
    if out_ids is None:
        out_ids = torch.empty(B, k, dtype=torch.uint32, device=ix.device)
    if out_scores is None:
        out_scores = torch.empty(B, k, dtype=torch.int32, device=ix.device)
    _check(lib().dessert_search_noalloc(ix.handle, q_vectors.data_ptr(), q_length, B, _ptr(cand_ids), cand_len, k,
                                        out_ids.data_ptr(), out_scores.data_ptr()))
    return out_ids, out_scores


def noalloc_scratch_bytes() -> int:
    return int(lib().dessert_noalloc_scratch_bytes())


def last_score_kernel(ix: Index) -> str:
    return lib().dessert_last_score_kernel(ix.handle).decode()


def set_debug(ix: Index, enable: bool = True) -> None:
    _check(lib().dessert_set_debug(ix.handle, int(bool(enable))))


def scores(ix: Index, q_vectors: torch.Tensor, q_lengths, cand_ids: Optional[torch.Tensor] = None,
           cand_offsets=None, workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """dessert_scores: raw int32 scores, [total candidates] or [B, n_docs]."""
    q_vectors, ql, B, cand_ids, co, total = _batch(ix, q_vectors, q_lengths, cand_ids, cand_offsets)
    if workspace is None:
        workspace = torch.empty(workspace_bytes(ix, B, q_vectors.shape[0], total, 0), dtype=torch.uint8,
                                device=ix.device)
    if out is None:
        out = torch.empty(total, dtype=torch.int32, device=ix.device)
    _check(lib().dessert_scores(ix.handle, q_vectors.data_ptr(), ql.ctypes.data, B, _ptr(cand_ids),
                                None if co is None else co.ctypes.data, workspace.data_ptr(), workspace.numel(),
                                out.data_ptr()))
    return out if co is not None else out.view(B, ix.n_docs)


def filter_kmeans(ix: Index, sample: torch.Tensor, init_centroids: torch.Tensor, iterations: int) -> torch.Tensor:
    """dessert_filter_kmeans: Lloyd iterations from init_centroids on the sample; returns the new centroids [K, d] int8."""
    sample = _check_vectors(ix, sample)
    if not init_centroids.is_cuda or init_centroids.dtype != torch.int8 or init_centroids.dim() != 2 \
            or init_centroids.shape[1] != ix.cfg.d:
        raise ValueError("init_centroids must be a device int8 tensor [K, d]")
    cent = init_centroids.contiguous().clone()
    K, n = cent.shape[0], sample.shape[0]
    nbytes = int(lib().dessert_filter_kmeans_workspace_bytes(ix.handle, n, K))
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ix.device)
    _check(lib().dessert_filter_kmeans(ix.handle, sample.data_ptr(), n, cent.data_ptr(), K, iterations,
                                       ws.data_ptr(), ws.numel()))
    return cent


def filter_build(ix: Index, centroids: torch.Tensor, vectors: torch.Tensor):
    """dessert_filter_build.  Returns (assign [V] int32, bucket_offsets [K+1] int32, bucket_docs [V] int32);
    only bucket_docs[: bucket_offsets[-1]] is meaningful."""
    vectors = _check_vectors(ix, vectors)
    if not centroids.is_cuda or centroids.dtype != torch.int8 or centroids.dim() != 2 or centroids.shape[1] != ix.cfg.d:
        raise ValueError("centroids must be a device int8 tensor [K, d]")
    centroids = centroids.contiguous()
    K, V = centroids.shape[0], vectors.shape[0]
    assign = torch.empty(V, dtype=torch.int32, device=ix.device)
    bucket_offsets = torch.empty(K + 1, dtype=torch.int32, device=ix.device)
    bucket_docs = torch.empty(max(V, 1), dtype=torch.int32, device=ix.device)
    _check(lib().dessert_filter_build(ix.handle, centroids.data_ptr(), K, vectors.data_ptr(), assign.data_ptr(),
                                      bucket_offsets.data_ptr(), bucket_docs.data_ptr()))
    ix._keep = [bucket_offsets, bucket_docs]
    return assign, bucket_offsets, bucket_docs


def filter_query(ix: Index, q_vectors: torch.Tensor, q_lengths, filter_probe: int, filter_k: int,
                 workspace: Optional[torch.Tensor] = None):
    """dessert_filter_query.  Returns (ids [B, filter_k] uint32 with 0xFFFFFFFF padding, counts [B, filter_k] int32)."""
    q_vectors = _check_vectors(ix, q_vectors)
    ql = _host_u32(q_lengths)
    B = ql.shape[0]
    if int(ql.sum()) != q_vectors.shape[0]:
        raise ValueError("sum(q_lengths) != number of query vectors")
    if workspace is None:
        nbytes = int(lib().dessert_filter_workspace_bytes(ix.handle, B, q_vectors.shape[0], int(ql.max()), filter_probe))
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ix.device)
    ids = torch.empty(B, filter_k, dtype=torch.uint32, device=ix.device)
    counts = torch.empty(B, filter_k, dtype=torch.int32, device=ix.device)
    _check(lib().dessert_filter_query(ix.handle, q_vectors.data_ptr(), ql.ctypes.data, B, filter_probe, filter_k,
                                      workspace.data_ptr(), workspace.numel(), ids.data_ptr(), counts.data_ptr()))
    return ids, counts


def filter_search(ix: Index, q_vectors: torch.Tensor, q_lengths, filter_probe: int, filter_k: int, k: int,
                  workspace: Optional[torch.Tensor] = None, out_ids: Optional[torch.Tensor] = None,
                  out_scores: Optional[torch.Tensor] = None):
    """dessert_filter_search: filter, then search among the filter's candidates.  Returns (ids [B, k] uint32, scores [B, k] int32)."""
    q_vectors = _check_vectors(ix, q_vectors)
    ql = _host_u32(q_lengths)
    B = ql.shape[0]
    if int(ql.sum()) != q_vectors.shape[0]:
        raise ValueError("sum(q_lengths) != number of query vectors")
    if workspace is None:
        nbytes = int(lib().dessert_filter_search_workspace_bytes(ix.handle, B, q_vectors.shape[0], int(ql.max()) if B else 0,
                                                                 filter_probe, filter_k, k))
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=ix.device)
    if out_ids is None:
        out_ids = torch.empty(B, k, dtype=torch.uint32, device=ix.device)
    if out_scores is None:
        out_scores = torch.empty(B, k, dtype=torch.int32, device=ix.device)
    _check(lib().dessert_filter_search(ix.handle, q_vectors.data_ptr(), ql.ctypes.data, B, filter_probe, filter_k, k,
                                       workspace.data_ptr(), workspace.numel(), out_ids.data_ptr(), out_scores.data_ptr()))
    return out_ids, out_scores


# ---- beside the search ----------------------------------------------------------------------------------------------------
_FLOAT_TYPES = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
_HALF_TYPES = (torch.float16, torch.bfloat16)
_INT8, _FLOAT32, _TOKEN_TYPES = (torch.int8,), (torch.float32,), (torch.int32, torch.uint32)
_MOST = 0x7FFFFFFF


def _lend(ix: Index, made) -> None:
    """Tensors that were allocated or copied on the current stream go to work on the index's stream: it waits for them, and
    they are not handed out again before it is done with them."""
    made = [t for t in made if t is not None]
    if not made:
        return
    current = torch.cuda.current_stream(ix.device)
    if current.cuda_stream == (ix.cfg.stream or 0):
        return
    stream = torch.cuda.ExternalStream(ix.cfg.stream, device=ix.device) if ix.cfg.stream else torch.cuda.default_stream(ix.device)
    stream.wait_stream(current)
    for t in made:
        t.record_stream(stream)


def _rows(ix: Index, t: torch.Tensor, name: str, made, dtypes):
    """A matrix on the index's device as the library reads it, elements of a row side by side and rows in order: the tensor, its address,
    rows, columns and the elements from row to row.  (The checks of a small call take longer than its kernels: each is made once.)"""
    shape = t.shape
    if len(shape) != 2 or t.dtype not in dtypes or t.device != ix.device:
        raise ValueError(f"{name} must be a matrix on {ix.device} of dtype " + " / ".join(str(d) for d in dtypes))
    n_rows, n_cols = shape
    if n_rows > _MOST or n_cols > _MOST:      # the library's limit of rows; it takes columns and vocabulary in 32 bits
        raise ValueError(f"{name} has {n_rows} rows of {n_cols}, at most 2^31 - 1 of each are taken")
    apart, step = t.stride()
    if (n_cols > 1 and step != 1) or (n_rows > 1 and apart < n_cols):
        t = t.contiguous()
        made.append(t)
        apart = n_cols
    return t, t.data_ptr(), n_rows, n_cols, apart if n_rows > 1 else n_cols


def _vector(ix: Index, t: torch.Tensor, n: int, name: str, made, dtypes) -> int:
    if t.shape != (n,) or t.dtype not in dtypes or t.device != ix.device:
        raise ValueError(f"{name} must be [{n}] on {ix.device} of dtype " + " / ".join(str(d) for d in dtypes))
    if n > 1 and t.stride(0) != 1:
        t = t.contiguous()
        made.append(t)
    return t.data_ptr()


def _output(ix: Index, t: Optional[torch.Tensor], shape, name: str, made, dtype) -> torch.Tensor:
    if t is None:
        t = torch.empty(shape, dtype=dtype, device=ix.device)
        made.append(t)
        return t
    if t.shape != shape or t.dtype != dtype or t.device != ix.device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} on {ix.device} of dtype {dtype}")
    return t


def _workspace(ix: Index, workspace: Optional[torch.Tensor], made, nbytes, *sizes):
    """(address, bytes) of the given workspace, or of one of nbytes(ix, *sizes) bytes"""
    if workspace is None:
        need = nbytes(ix, *sizes)
        if need == 0:
            return None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=ix.device)
        made.append(workspace)
    elif workspace.device != ix.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous on {ix.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def quantize_rows(ix: Index, x: torch.Tensor, scaling: int = SCALE_MAXABS, out: Optional[torch.Tensor] = None,
                  out_scales: Optional[torch.Tensor] = None):
    """dessert_quantize_rows: x [n, c] of float16 / bfloat16 / float32 (rows may lie apart).  Returns (codes [n, c] int8,
    scales [n] float32)."""
    made = []
    x, x_ptr, n, c, apart = _rows(ix, x, "x", made, _FLOAT_TYPES)
    out = _output(ix, out, (n, c), "out", made, torch.int8)
    out_scales = _output(ix, out_scales, (n,), "out_scales", made, torch.float32)
    _lend(ix, made)
    _check(lib().dessert_quantize_rows(ix.handle, x_ptr, _FLOAT_TYPES[x.dtype], n, c, apart, scaling, out.data_ptr(), out_scales.data_ptr()))
    return out, out_scales


def scaled_matmul_workspace_bytes(ix: Index, n_rows: int, n_channels: int, n_cols: int) -> int:
    return int(lib().dessert_scaled_matmul_workspace_bytes(ix.handle, n_rows, n_channels, n_cols))


def scaled_matmul(ix: Index, a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dessert_scaled_matmul: a [m, k] and b [n, k] int8 (rows may lie apart), scales [m] and [n] float32, bias [n] float32
    or None.  Returns [m, n] of out_dtype; ``out`` (rows may lie apart) decides the type if given."""
    made = []
    _, a_ptr, m, k, a_apart = _rows(ix, a, "a", made, _INT8)
    _, b_ptr, n, b_cols, b_apart = _rows(ix, b, "b", made, _INT8)
    if b_cols != k:
        raise ValueError(f"a has {k} columns, b has {b_cols}")
    sa_ptr = _vector(ix, a_scales, m, "a_scales", made, _FLOAT32)
    sb_ptr = _vector(ix, b_scales, n, "b_scales", made, _FLOAT32)
    bias_ptr = None if bias is None else _vector(ix, bias, n, "bias", made, _FLOAT32)
    if out is None:
        if out_dtype not in _FLOAT_TYPES:
            raise ValueError("out_dtype must be float16, bfloat16 or float32")
        out = _output(ix, None, (m, n), "out", made, out_dtype)
    kept, out_ptr, out_rows, out_cols, out_apart = _rows(ix, out, "out", [], _FLOAT_TYPES)
    if kept is not out or out_rows != m or out_cols != n:
        raise ValueError(f"out must be [{m}, {n}] with the elements of a row side by side")
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, scaled_matmul_workspace_bytes, m, n, k)
    _lend(ix, made)
    _check(lib().dessert_scaled_matmul(ix.handle, a_ptr, a_apart, sa_ptr, m, b_ptr, b_apart, sb_ptr, bias_ptr, n, k, _FLOAT_TYPES[out.dtype],
                                       out_ptr, out_apart, ws_ptr, ws_bytes))
    return out


def _tokens(ix: Index, tokens: Optional[torch.Tensor], n: int, made) -> Optional[int]:
    if tokens is None:
        return None
    if tokens.dtype == torch.int64:     # ids outside 32 bits are ids outside any vocabulary; -1 is the padding mark
        tokens = torch.where((tokens < -1) | (tokens > 0x7FFFFFFF), 0x7FFFFFFF, tokens).to(torch.int32)
        made.append(tokens)
    return _vector(ix, tokens, n, "tokens", made, _TOKEN_TYPES)


def _logprob_outputs(ix: Index, n: int, n_top: int, tokens, outs, made):
    if not 0 <= n_top <= _MOST:
        raise ValueError(f"n_top is {n_top}")
    o = (None,) * 4 if outs is None else outs
    return (None if tokens is None else _output(ix, o[0], (n,), "outs[0]", made, torch.float32),
            _output(ix, o[1], (n,), "outs[1]", made, torch.float32),
            _output(ix, o[2], (n, n_top), "outs[2]", made, torch.uint32),
            _output(ix, o[3], (n, n_top), "outs[3]", made, torch.float32))


def token_logprobs_workspace_bytes(ix: Index, n_rows: int, n_vocab: int, n_top: int) -> int:
    return int(lib().dessert_token_logprobs_workspace_bytes(ix.handle, n_rows, n_vocab, n_top))


def token_logprobs(ix: Index, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, n_top: int = 0,
                   workspace: Optional[torch.Tensor] = None, outs=None):
    """dessert_token_logprobs: logits [n, V] of float16 / bfloat16 / float32 (rows may lie apart), tokens [n] int32 / uint32 /
    int64 (-1: padded position) or None.  Returns (logprobs [n] or None, entropy [n], top ids [n, n_top] uint32, top logprobs
    [n, n_top]); ``outs``: the four tensors to write."""
    made = []
    logits, l_ptr, n, V, apart = _rows(ix, logits, "logits", made, _FLOAT_TYPES)
    tokens = _tokens(ix, tokens, n, made)
    o = _logprob_outputs(ix, n, n_top, tokens, outs, made)
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, token_logprobs_workspace_bytes, n, V, n_top)
    _lend(ix, made)
    _check(lib().dessert_token_logprobs(ix.handle, l_ptr, _FLOAT_TYPES[logits.dtype], n, V, apart, tokens, n_top, ws_ptr, ws_bytes,
                                        *map(_ptr, o)))
    return o


def head_logprobs_workspace_bytes(ix: Index, n_rows: int, n_vocab: int, n_cols: int, n_top: int) -> int:
    return int(lib().dessert_head_logprobs_workspace_bytes(ix.handle, n_rows, n_vocab, n_cols, n_top))


def head_logprobs(ix: Index, a: torch.Tensor, a_scales: torch.Tensor, vocab: torch.Tensor, vocab_scales: torch.Tensor,
                  tokens: Optional[torch.Tensor] = None, n_top: int = 0, workspace: Optional[torch.Tensor] = None, outs=None):
    """dessert_head_logprobs: states a [n, k] and vocabulary matrix [V, k] int8 with scales [n] and [V] float32; the rest as
    token_logprobs."""
    made = []
    _, a_ptr, n, k, a_apart = _rows(ix, a, "a", made, _INT8)
    _, v_ptr, V, v_cols, v_apart = _rows(ix, vocab, "vocab", made, _INT8)
    if v_cols != k:
        raise ValueError(f"a has {k} columns, vocab has {v_cols}")
    sa_ptr = _vector(ix, a_scales, n, "a_scales", made, _FLOAT32)
    sv_ptr = _vector(ix, vocab_scales, V, "vocab_scales", made, _FLOAT32)
    tokens = _tokens(ix, tokens, n, made)
    o = _logprob_outputs(ix, n, n_top, tokens, outs, made)
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, head_logprobs_workspace_bytes, n, V, k, n_top)
    _lend(ix, made)
    _check(lib().dessert_head_logprobs(ix.handle, a_ptr, a_apart, sa_ptr, n, v_ptr, v_apart, sv_ptr, V, k, tokens, n_top, ws_ptr, ws_bytes,
                                       *map(_ptr, o)))
    return o


# ---- what a model keeps of its tokens ---------------------------------------------------------------------------------------
class Cache:
    """One layer's paged int8 cache, as the calls take it: the tensors (kept alive here) and dessert_cache_t."""

    def __init__(self, tensors, struct: _CacheStruct):
        self.k_codes, self.v_codes, self.k_scales, self.v_scales, self.bounds = tensors
        self.struct = struct
        self.n_pages, self.n_heads, self.page_tokens, self.dim = struct.n_pages, struct.n_heads, struct.page_tokens, struct.dim
        self.address, self.raw = C.addressof(struct), bytes(struct)


class CacheBatch:
    """The sequences of a call: the tensors (kept alive here; their contents may change from call to call) and dessert_cache_batch_t."""

    def __init__(self, tensors, struct: _BatchStruct):
        self.tables, self.lengths, self.starts = tensors
        self.struct = struct
        self.n_seqs, self.n_tokens = struct.n_seqs, struct.n_tokens
        self.address = C.addressof(struct)


def _kept(ix: Index, t: torch.Tensor, shape, name: str, dtypes) -> int:
    """A tensor that a call reads or writes where it lies: None in a shape is any size."""
    if (len(t.shape) != len(shape) or any(w is not None and w != n for n, w in zip(t.shape, shape)) or t.dtype not in dtypes
            or t.device != ix.device or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {list(shape)} on {ix.device} of dtype " + " / ".join(str(d) for d in dtypes))
    return t.data_ptr()


def _size(n: int, name: str, most: int = _MOST) -> int:
    if not 0 <= n <= most:
        raise ValueError(f"{name} is {n}, 0 to {most} is taken")
    return n


def cache(ix: Index, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor,
          bounds: Optional[torch.Tensor] = None) -> Cache:
    """dessert_cache_t: k_codes [pages, heads, page tokens, dim] int8, v_codes [pages, heads, dim, page tokens] int8, scales
    [pages, heads] float32, bounds [pages, heads, 2, dim] int8 or None.  Nothing is copied: calls read and write these tensors."""
    k_ptr = _kept(ix, k_codes, (None,) * 4, "k_codes", _INT8)
    P, H, T, D = k_codes.shape
    for n in (P, H, T, D):
        _size(n, "a size of k_codes")
    struct = _CacheStruct(k_ptr, _kept(ix, v_codes, (P, H, D, T), "v_codes", _INT8), _kept(ix, k_scales, (P, H), "k_scales", _FLOAT32),
                          _kept(ix, v_scales, (P, H), "v_scales", _FLOAT32),
                          None if bounds is None else _kept(ix, bounds, (P, H, 2, D), "bounds", _INT8), P, H, T, D)
    return Cache((k_codes, v_codes, k_scales, v_scales, bounds), struct)


def cache_batch(ix: Index, tables: torch.Tensor, lengths: torch.Tensor, starts: Optional[torch.Tensor] = None,
                n_tokens: Optional[int] = None, max_tokens: Optional[int] = None, max_length: Optional[int] = None) -> CacheBatch:
    """dessert_cache_batch_t: tables [seqs, table pages] and lengths [seqs] int32 / uint32 (-1: no page), starts [seqs + 1] or None (one new token
    each).  With starts, n_tokens (rows of the arrays of tokens) is needed; max_tokens (new tokens of a sequence, at most)
    is taken to be that where it is not given (the form of attention goes by it: a few
    tokens each are done sooner where it says so), max_length (which decides how work is divided) what the tables hold."""
    t_ptr = _kept(ix, tables, (None, None), "tables", _TOKEN_TYPES)
    n, width = tables.shape
    l_ptr = _kept(ix, lengths, (n,), "lengths", _TOKEN_TYPES)
    s_ptr = None if starts is None else _kept(ix, starts, (n + 1,), "starts", _TOKEN_TYPES)
    if n_tokens is None:
        if starts is not None:
            raise ValueError("n_tokens is needed with starts")
        n_tokens = n
    if max_tokens is None:
        max_tokens = n_tokens if starts is not None else 1
    struct = _BatchStruct(t_ptr, l_ptr, s_ptr, _size(n, "the number of sequences"), _size(width, "the tables' width"), _size(n_tokens, "n_tokens"),
                          _size(max_tokens, "max_tokens"), _MOST if max_length is None else _size(max_length, "max_length"))
    return CacheBatch((tables, lengths, starts), struct)


def _states(ix: Index, t: torch.Tensor, n: int, heads: Optional[int], dim: int, name: str, made, dtypes):
    """[n, heads, dim], a token's heads side by side: address, heads, elements from token to token"""
    shape = t.shape
    if (len(shape) != 3 or shape[0] != n or shape[2] != dim or (heads is not None and shape[1] != heads) or shape[1] > _MOST
            or t.dtype not in dtypes or t.device != ix.device):
        raise ValueError(f"{name} must be [{n}, {'heads' if heads is None else heads}, {dim}] on {ix.device} of dtype " + " / ".join(str(d) for d in dtypes))
    heads, wide = shape[1], shape[1] * dim
    apart, between, step = t.stride()
    if step != 1 or (heads > 1 and between != dim) or (n > 1 and apart < wide):
        t = t.contiguous()
        made.append(t)
        apart = wide
    return t.data_ptr(), heads, apart if n > 1 else wide


def cache_append(ix: Index, cache: Cache, batch: CacheBatch, k: torch.Tensor, v: torch.Tensor) -> None:
    """dessert_cache_append: k and v [tokens, heads, dim] of float16 / bfloat16 / float32 (tokens may lie apart)."""
    made = []
    if k.dtype != v.dtype:
        raise ValueError("k and v must be of one dtype")
    k_ptr, _, k_apart = _states(ix, k, batch.n_tokens, cache.n_heads, cache.dim, "k", made, _FLOAT_TYPES)
    v_ptr, _, v_apart = _states(ix, v, batch.n_tokens, cache.n_heads, cache.dim, "v", made, _FLOAT_TYPES)
    _lend(ix, made)
    _check(lib().dessert_cache_append(ix.handle, cache.address, batch.address, k_ptr, k_apart, v_ptr, v_apart, _FLOAT_TYPES[k.dtype]))


def cache_attention_workspace_bytes(ix: Index, cache: Cache, batch: CacheBatch, n_q_heads: int, n_select: int = 0) -> int:
    return int(lib().dessert_cache_attention_workspace_bytes(ix.handle, cache.address, batch.address, n_q_heads, n_select))


def cache_attention(ix: Index, cache: Cache, batch: CacheBatch, q: torch.Tensor, scale: Optional[float] = None, window: int = 0,
                    pages: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None):
    """dessert_cache_attention: q [tokens, query heads, dim] of float16 / bfloat16 (tokens may lie apart), scale 1 / sqrt(dim) unless given, pages
    [tokens, heads, n] int32 / uint32 as cache_select gives them, or None.  Returns (out like q without gaps, lse [tokens,
    query heads] float32)."""
    made = []
    n = batch.n_tokens
    q_ptr, heads, apart = _states(ix, q, n, None, cache.dim, "q", made, _HALF_TYPES)
    window = _size(window, "window")
    if pages is None:
        p_ptr, n_select = None, 0
    else:
        p_ptr, n_select = _kept(ix, pages, (n, cache.n_heads, None), "pages", _TOKEN_TYPES), _size(pages.shape[2], "the number of pages")
        if n_select == 0:
            raise ValueError("pages has no places")
    out = _output(ix, out, (n, heads, cache.dim), "out", made, q.dtype)
    out_lse = _output(ix, out_lse, (n, heads), "out_lse", made, torch.float32)
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, cache_attention_workspace_bytes, cache, batch, heads, n_select)
    _lend(ix, made)
    _check(lib().dessert_cache_attention(ix.handle, cache.address, batch.address, q_ptr, _FLOAT_TYPES[q.dtype], apart, heads,
                                         cache.dim ** -0.5 if scale is None else scale, window, p_ptr, n_select, ws_ptr, ws_bytes,
                                         out.data_ptr(), out_lse.data_ptr()))
    return out, out_lse


def cache_select_workspace_bytes(ix: Index, cache: Cache, batch: CacheBatch) -> int:
    return int(lib().dessert_cache_select_workspace_bytes(ix.handle, cache.address, batch.address))


def cache_select(ix: Index, cache: Cache, batch: CacheBatch, q_codes: torch.Tensor, q_scales: torch.Tensor, n_select: int,
                 n_first: int = 0, n_last: int = 0, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dessert_cache_select: q_codes [tokens * query heads, dim] int8 and q_scales [tokens * query heads] as quantize_rows gives them.
    Returns places [tokens, heads, n_select] uint32, ascending, 0xFFFFFFFF behind the last."""
    made = []
    n = batch.n_tokens
    q_ptr = _kept(ix, q_codes, (None, cache.dim), "q_codes", _INT8)
    rows = q_codes.shape[0]
    if rows % n if n else rows:
        raise ValueError(f"q_codes has {rows} rows for {n} tokens")
    heads = rows // n if n else cache.n_heads      # of no tokens: any number of heads
    s_ptr = _vector(ix, q_scales, rows, "q_scales", made, _FLOAT32)
    n_first, n_last = _size(n_first, "n_first"), _size(n_last, "n_last")
    out = _output(ix, out, (n, cache.n_heads, _size(n_select, "n_select")), "out", made, torch.uint32)
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, cache_select_workspace_bytes, cache, batch)
    _lend(ix, made)
    _check(lib().dessert_cache_select(ix.handle, cache.address, batch.address, q_ptr, s_ptr, heads, n_select, n_first, n_last, ws_ptr, ws_bytes, out.data_ptr()))
    return out


def _layers(caches):
    """(dessert_cache_t of each layer side by side, how many, pages)"""
    if isinstance(caches, Cache):
        return caches.raw, 1, caches.n_pages
    raw = [c.raw for c in caches]
    if not raw:
        raise ValueError("no layers")
    return b"".join(raw), len(raw), caches[0].n_pages


def _numbers(ix: Index, t: torch.Tensor, n: Optional[int], name: str) -> int:
    """The address of a vector of 32-bit numbers that a call reads or writes where it lies (n = None: of any length)."""
    shape = t.shape
    if len(shape) != 1 or (n is not None and shape[0] != n) or t.dtype not in _TOKEN_TYPES or t.device != ix.device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{'any' if n is None else n}] on {ix.device} of dtype int32 / uint32")
    return t.data_ptr()


def _tables(ix: Index, tables: torch.Tensor, lengths: torch.Tensor):
    """(address of tables, of lengths, sequences, width)"""
    shape = tables.shape
    if len(shape) != 2 or tables.dtype not in _TOKEN_TYPES or tables.device != ix.device or not tables.is_contiguous():
        raise ValueError(f"tables must be a contiguous matrix on {ix.device} of dtype int32 / uint32")
    n, width = shape
    if n > _MOST or width > _MOST:
        raise ValueError(f"tables of {n} rows of {width}, at most 2^31 - 1 of each are taken")
    return tables.data_ptr(), _numbers(ix, lengths, n, "lengths"), n, width


def _page_output(ix: Index, t: Optional[torch.Tensor], shape, name: str, made) -> torch.Tensor:
    return _output(ix, t, shape, name, made, torch.uint32 if t is not None and t.dtype == torch.uint32 else torch.int32)


def cache_advance_workspace_bytes(ix: Index, n_pages: int, n_new: int) -> int:
    return int(lib().dessert_cache_advance_workspace_bytes(ix.handle, n_pages, n_new))


def cache_advance(ix: Index, caches, refs: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor, add: torch.Tensor,
                  parents: Optional[torch.Tensor] = None, outs=None, workspace: Optional[torch.Tensor] = None):
    """dessert_cache_advance: caches a Cache or one for each layer, refs [pages] (changed), tables [seqs, table pages], lengths [seqs], add and parents [new
    seqs] (-1: none) or None, all int32 / uint32.  Returns (tables [new seqs, table pages], lengths [new seqs], status [2]: free
    pages, sequences without room); ``outs``: the three tensors to write, apart from the old ones."""
    made = []
    layers, n_layers, pages = _layers(caches)
    r_ptr = _numbers(ix, refs, pages, "refs")
    t_ptr, l_ptr, n, width = _tables(ix, tables, lengths)
    a_ptr = _numbers(ix, add, None, "add")
    new = add.shape[0]
    p_ptr = None if parents is None else _numbers(ix, parents, new, "parents")
    o = (None, None, None) if outs is None else outs
    o = (_page_output(ix, o[0], (new, width), "outs[0]", made), _page_output(ix, o[1], (new,), "outs[1]", made),
         _page_output(ix, o[2], (2,), "outs[2]", made))
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, cache_advance_workspace_bytes, pages, new)
    _lend(ix, made)
    _check(lib().dessert_cache_advance(ix.handle, layers, n_layers, r_ptr, t_ptr, width, l_ptr, n, p_ptr, a_ptr, _size(new, "the number of sequences"),
                                       ws_ptr, ws_bytes, o[0].data_ptr(), o[1].data_ptr(), o[2].data_ptr()))
    return o


def cache_compact_workspace_bytes(ix: Index, n_pages: int) -> int:
    return int(lib().dessert_cache_compact_workspace_bytes(ix.handle, n_pages))


def cache_compact(ix: Index, caches, refs: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor, outs=None,
                  workspace: Optional[torch.Tensor] = None):
    """dessert_cache_compact: caches as for cache_advance, refs [pages] and tables [seqs, table pages] (both changed), lengths [seqs], all int32 / uint32.
    Returns (new numbers [pages], pages in use [1])."""
    made = []
    layers, n_layers, pages = _layers(caches)
    r_ptr = _numbers(ix, refs, pages, "refs")
    t_ptr, l_ptr, n, width = _tables(ix, tables, lengths)
    o = (None, None) if outs is None else outs
    o = (_page_output(ix, o[0], (pages,), "outs[0]", made), _page_output(ix, o[1], (1,), "outs[1]", made))
    ws_ptr, ws_bytes = _workspace(ix, workspace, made, cache_compact_workspace_bytes, pages)
    _lend(ix, made)
    _check(lib().dessert_cache_compact(ix.handle, layers, n_layers, r_ptr, t_ptr, width, l_ptr, n, ws_ptr, ws_bytes, o[0].data_ptr(),
                                       o[1].data_ptr()))
    return o


def enable_timing(ix: Index, enable=True) -> None:
    """dessert_enable_timing: False/0 off, True/1 every call, n > 1 every n-th call."""
    _check(lib().dessert_enable_timing(ix.handle, int(enable)))


def get_timing(ix: Index, calls_back: int = 0):
    ms = (C.c_float * 4)()
    _check(lib().dessert_get_timing(ix.handle, calls_back, ms))
    return {"hash_ms": ms[0], "score_ms": ms[1], "topk_ms": ms[2], "total_ms": ms[3]}


def probe_read_bandwidth(buf: torch.Tensor, reps: int = 10) -> float:
    """dessert_probe_read_bandwidth: GB/s of a plain streaming read over `buf` (measurement aid)."""
    ms = C.c_float()
    nbytes = buf.numel() * buf.element_size()
    stream = torch.cuda.current_stream(buf.device).cuda_stream
    _check(lib().dessert_probe_read_bandwidth(buf.data_ptr(), nbytes, buf.device.index or 0, stream, reps, C.byref(ms)))
    return nbytes / (ms.value * 1e-3) / 1e9


def probe_mix_bandwidth(src: torch.Tensor, dst: torch.Tensor, reps: int = 10) -> float:
    """dessert_probe_mix_bandwidth: GB/s (read + written) of a kernel that reads 4 bytes of `src` for every byte it
    writes to `dst` and computes nothing (measurement aid: the ceiling for the index build's traffic)."""
    out_bytes = dst.numel() * dst.element_size()
    if src.numel() * src.element_size() < 4 * out_bytes:
        raise ValueError("src must hold four times the bytes of dst")
    ms = C.c_float()
    stream = torch.cuda.current_stream(dst.device).cuda_stream
    _check(lib().dessert_probe_mix_bandwidth(src.data_ptr(), dst.data_ptr(), out_bytes, dst.device.index or 0, stream, reps,
                                             C.byref(ms)))
    return 5 * out_bytes / (ms.value * 1e-3) / 1e9
