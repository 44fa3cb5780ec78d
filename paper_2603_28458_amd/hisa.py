"""ctypes binding of libhisa.so (C ABI in include/hisa.h).  Argument marshalling only: every
step of the indexer runs in the HIP kernels.  PyTorch supplies device memory and the stream.

The functions carry the names of the C entry points.  There is no CPU fallback: if the compiled
library is missing, the first call raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

HISA_F32, HISA_BF16, HISA_FP8_E4M3 = 0, 1, 2
HISA_WEIGHTS_16BIT, HISA_WEIGHTS_8BIT = 0, 1
OP_POOL, OP_BLOCK_SCORE_TOPK, OP_TOKEN_REFINE_TOPK, OP_FLAT_TOPK = 0, 1, 2, 3
DTYPE_CODE = {"f32": HISA_F32, "bf16": HISA_BF16, "fp8_e4m3": HISA_FP8_E4M3}
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libhisa.so")

EXPORTS = ["hisa_pool_blocks", "hisa_pool_append", "hisa_block_score_topk", "hisa_token_refine_topk",
           "hisa_block_sparse_tokens", "hisa_index_iou", "dsa_flat_indexer_topk", "hisa_workspace_bytes",
           "hisa_status_string", "hisa_version", "hisa_probe_copy", "hisa_probe_mfma", "hisa_probe_mfma_fp8", "hisa_probe_mfma_toggling", "hisa_indexer_topk", "hisa_pool_blocks_max",
           "hisa_token_refine_topk_static", "hisa_page_tables", "hisa_cache_append", "hisa_paged_attention",
           "hisa_sparse_attention", "hisa_attention_workspace_bytes"]
STATIC_SCRATCH_BYTES = 16 << 20


class HisaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


class _Keys(C.Structure):
    _fields_ = [("k", C.c_void_p), ("k_scale", C.c_void_p), ("seq_len", C.c_void_p),
                ("n_seq", C.c_int32), ("s_max", C.c_int32), ("d", C.c_int32), ("k_dtype", C.c_int32)]


class _Queries(C.Structure):
    _fields_ = [("q", C.c_void_p), ("w", C.c_void_p), ("q_seq", C.c_void_p), ("q_pos", C.c_void_p),
                ("q_lo", C.c_void_p), ("T", C.c_int32), ("H", C.c_int32), ("q_pos0", C.c_int32),
                ("q_dtype", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("block_table", C.c_void_p), ("seq_len", C.c_void_p), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("n_pages", C.c_int32), ("page", C.c_int32),
                ("n_seq", C.c_int32), ("max_pages", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32),
                ("dtype", C.c_int32), ("weights", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (python -m paper_2603_28458_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               f"`python -m paper_2603_28458_amd.build` (there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.hisa_pool_blocks.argtypes = [C.POINTER(_Keys), i32, i32, i32, vp, i32, vp]
        L.hisa_pool_blocks.restype = C.c_int
        L.hisa_pool_blocks_max.argtypes = [C.POINTER(_Keys), i32, i32, i32, vp, i32, vp]
        L.hisa_pool_blocks_max.restype = C.c_int
        L.hisa_pool_append.argtypes = [C.POINTER(_Keys), i32, vp, i32, vp, i32, vp]
        L.hisa_pool_append.restype = C.c_int
        L.hisa_block_sparse_tokens.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), i32, i32, vp, vp, vp]
        L.hisa_block_sparse_tokens.restype = C.c_int
        L.hisa_index_iou.argtypes = [vp, vp, i32, i32, vp, vp]
        L.hisa_index_iou.restype = C.c_int
        L.hisa_block_score_topk.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), vp, i32, i32, i32,
                                            vp, vp, vp, sz, vp]
        L.hisa_block_score_topk.restype = C.c_int
        L.hisa_token_refine_topk.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), i32, i32, vp, i32,
                                             vp, vp, vp, vp, sz, vp]
        L.hisa_token_refine_topk.restype = C.c_int
        L.hisa_token_refine_topk_static.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), i32, i32, vp, i32,
                                                    vp, vp, vp]
        L.hisa_token_refine_topk_static.restype = C.c_int
        L.dsa_flat_indexer_topk.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), i32, vp, vp, vp,
                                            sz, vp]
        L.dsa_flat_indexer_topk.restype = C.c_int
        L.hisa_workspace_bytes.argtypes = [C.c_int, C.POINTER(_Queries), C.POINTER(_Keys), i32, i32,
                                           i32, i32]
        L.hisa_workspace_bytes.restype = sz
        L.hisa_indexer_topk.argtypes = [C.POINTER(_Queries), C.POINTER(_Keys), vp, i32, i32, i32, i32, vp, vp,
                                        vp, vp]
        L.hisa_indexer_topk.restype = C.c_int
        L.hisa_probe_copy.argtypes = [vp, vp, sz, vp]
        L.hisa_probe_copy.restype = C.c_int
        L.hisa_probe_mfma.argtypes = [vp, i32, C.POINTER(C.c_double), vp]
        L.hisa_probe_mfma.restype = C.c_int
        L.hisa_probe_mfma_fp8.argtypes = [vp, i32, C.POINTER(C.c_double), vp]
        L.hisa_probe_mfma_fp8.restype = C.c_int
        L.hisa_probe_mfma_toggling.argtypes = [vp, i32, i32, C.POINTER(C.c_double), vp]
        L.hisa_probe_mfma_toggling.restype = C.c_int
        L.hisa_page_tables.argtypes = [vp, vp, i32, vp, i32, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.hisa_page_tables.restype = C.c_int
        L.hisa_cache_append.argtypes = [C.POINTER(_Cache), vp, vp, vp, i32, C.c_int64, i32, vp]
        L.hisa_cache_append.restype = C.c_int
        L.hisa_paged_attention.argtypes = [C.POINTER(_Queries), C.POINTER(_Cache), vp, C.c_float, vp, vp, vp, sz, vp]
        L.hisa_paged_attention.restype = C.c_int
        L.hisa_sparse_attention.argtypes = [C.POINTER(_Queries), C.POINTER(_Cache), vp, i32, C.c_float, vp, vp, vp, sz,
                                            vp]
        L.hisa_sparse_attention.restype = C.c_int
        L.hisa_attention_workspace_bytes.argtypes = [C.POINTER(_Queries), C.POINTER(_Cache), i32]
        L.hisa_attention_workspace_bytes.restype = sz
        L.hisa_status_string.argtypes = [C.c_int]
        L.hisa_status_string.restype = C.c_char_p
        L.hisa_version.argtypes = []
        L.hisa_version.restype = C.c_char_p
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().hisa_status_string(int(status)).decode()


def version() -> str:
    return lib().hisa_version().decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to the library must be contiguous"
    return t.data_ptr()


# The handle alone: torch.cuda.current_stream() builds a Stream object around it on every call.  (Not part of
# torch's documented interface: without it the object is built.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


@dataclass
class Keys:
    """Token-level indexing keys: k [n_seq, s_max, d] (float32 / bfloat16 / uint8 or float8 codes),
    k_scale [n_seq, s_max] float32 for fp8, seq_len [n_seq] int32; all on the GPU."""
    k: Optional[torch.Tensor]
    seq_len: torch.Tensor
    dtype: int
    k_scale: Optional[torch.Tensor] = None
    n_seq: int = 0
    s_max: int = 0
    d: int = 0

    def __post_init__(self):
        if self.k is not None:
            self.n_seq, self.s_max, self.d = self.k.shape

    def c(self) -> _Keys:
        return _Keys(_ptr(self.k), _ptr(self.k_scale), _ptr(self.seq_len), self.n_seq, self.s_max,
                     self.d, self.dtype)


@dataclass
class Queries:
    """Indexing queries q [T, H, d] (float32 / bfloat16), gates w [T, H] float32, optional
    q_seq / q_pos / q_lo [T] int32; all on the GPU.  (The attention calls read no gates: w may be None there.)"""
    q: torch.Tensor
    w: Optional[torch.Tensor]
    dtype: int
    q_seq: Optional[torch.Tensor] = None
    q_pos: Optional[torch.Tensor] = None
    q_pos0: int = 0
    q_lo: Optional[torch.Tensor] = None

    @property
    def T(self) -> int:
        return self.q.shape[0]

    @property
    def H(self) -> int:
        return self.q.shape[1]

    def c(self) -> _Queries:
        return _Queries(_ptr(self.q), _ptr(self.w), _ptr(self.q_seq), _ptr(self.q_pos), _ptr(self.q_lo),
                        self.T, self.H, self.q_pos0, self.dtype)


def _check(status: int, where: str):
    if status != 0:
        raise HisaError(status, where)


def hisa_workspace_bytes(op: int, queries: Queries, keys: Keys, B: int = 1, m: int = 0, k: int = 0,
                         want_scores: bool = False) -> int:
    qc, kc = queries.c(), keys.c()
    return int(lib().hisa_workspace_bytes(op, C.byref(qc), C.byref(kc), B, m, k, int(want_scores)))


def _ws(op: int, qc: _Queries, kc: _Keys, B: int, m: int, k: int, want_scores: bool, device) -> Optional[torch.Tensor]:
    """A workspace for a call that was not given one."""
    nbytes = int(lib().hisa_workspace_bytes(op, qc, kc, B, m, k, int(want_scores)))
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


_POOLED_TORCH = {HISA_F32: torch.float32, HISA_BF16: torch.bfloat16}


def hisa_pool_blocks(keys: Keys, B: int, pooled: Optional[torch.Tensor] = None,
                     pooled_dtype: int = HISA_BF16, blk_begin: int = 0, blk_end: Optional[int] = None,
                     stream=None, max_pool: bool = False) -> torch.Tensor:
    """Eq. 4: pooled [n_seq, s_max / B, d] (max_pool: hisa_pool_blocks_max, the maximum instead of the mean)."""
    M = keys.s_max // B
    if pooled is None:
        pooled = torch.zeros((keys.n_seq, M, keys.d), dtype=_POOLED_TORCH[pooled_dtype],
                             device=keys.k.device)
    kc = keys.c()
    fn = lib().hisa_pool_blocks_max if max_pool else lib().hisa_pool_blocks
    st = fn(C.byref(kc), B, blk_begin, M if blk_end is None else blk_end, _ptr(pooled), pooled_dtype,
            _stream(stream))
    _check(st, "hisa_pool_blocks_max" if max_pool else "hisa_pool_blocks")
    return pooled


def hisa_pool_blocks_max(keys: Keys, B: int, pooled: Optional[torch.Tensor] = None, pooled_dtype: int = HISA_BF16,
                         blk_begin: int = 0, blk_end: Optional[int] = None, stream=None) -> torch.Tensor:
    """Eq. 4 with Pool = per-dimension maximum."""
    return hisa_pool_blocks(keys, B, pooled, pooled_dtype, blk_begin, blk_end, stream, max_pool=True)


def hisa_pool_append(keys: Keys, B: int, prev_len: torch.Tensor, max_new_tokens: int, pooled: torch.Tensor,
                     pooled_dtype: int = HISA_BF16, stream=None) -> torch.Tensor:
    """Section 4.1, incremental pooled cache: re-pools the blocks that grew since prev_len."""
    kc = keys.c()
    st = lib().hisa_pool_append(C.byref(kc), B, _ptr(prev_len), max_new_tokens, _ptr(pooled), pooled_dtype,
                                _stream(stream))
    _check(st, "hisa_pool_append")
    return pooled


def hisa_block_sparse_tokens(queries: Queries, keys: Keys, B: int, m: int, block_idx: torch.Tensor,
                             tokens: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Block-Sparse baseline (Section 5): tokens [T, m*B] int32, -1 where not visible."""
    if tokens is None:
        tokens = torch.empty((queries.T, m * B), dtype=torch.int32, device=block_idx.device)
    qc, kc = queries.c(), keys.c()
    st = lib().hisa_block_sparse_tokens(C.byref(qc), C.byref(kc), B, m, _ptr(block_idx), _ptr(tokens),
                                        _stream(stream))
    _check(st, "hisa_block_sparse_tokens")
    return tokens


def hisa_index_iou(a_idx: torch.Tensor, b_idx: torch.Tensor, iou: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """Eq. 12 per row of two [T, k] index tensors (ascending rows, -1 padding)."""
    T, k = a_idx.shape
    assert b_idx.shape == a_idx.shape
    if iou is None:
        iou = torch.empty((T,), dtype=torch.float32, device=a_idx.device)
    st = lib().hisa_index_iou(_ptr(a_idx), _ptr(b_idx), T, k, _ptr(iou), _stream(stream))
    _check(st, "hisa_index_iou")
    return iou


def hisa_block_score_topk(queries: Queries, keys: Keys, pooled: torch.Tensor, pooled_dtype: int, B: int,
                          m: int, block_idx: Optional[torch.Tensor] = None,
                          block_scores: Optional[torch.Tensor] = None, want_scores: bool = False,
                          ws: Optional[torch.Tensor] = None, stream=None):
    """Stage 1 (Eqs. 5-6).  Returns (block_idx [T, m] int32, block_scores [T, s_max/B] or None)."""
    dev = queries.q.device
    T, M = queries.T, keys.s_max // B
    if block_idx is None:
        block_idx = torch.empty((T, m), dtype=torch.int32, device=dev)
    if want_scores and block_scores is None:
        block_scores = torch.empty((T, M), dtype=torch.float32, device=dev)
    qc, kc = queries.c(), keys.c()
    if ws is None:
        ws = _ws(OP_BLOCK_SCORE_TOPK, qc, kc, B, m, 0, block_scores is not None, dev)
    st = lib().hisa_block_score_topk(C.byref(qc), C.byref(kc), _ptr(pooled), pooled_dtype, B, m,
                                     _ptr(block_idx), _ptr(block_scores), _ptr(ws),
                                     0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "hisa_block_score_topk")
    return block_idx, block_scores


def hisa_token_refine_topk(queries: Queries, keys: Keys, B: int, m: int, block_idx: torch.Tensor, k: int,
                           topk_idx: Optional[torch.Tensor] = None,
                           topk_scores: Optional[torch.Tensor] = None,
                           cand_scores: Optional[torch.Tensor] = None, want_topk_scores: bool = False,
                           want_cand_scores: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """Stage 2 (Eqs. 7-9).  Returns (topk_idx [T, k] int32, topk_scores or None, cand_scores or None)."""
    dev = queries.q.device
    T = queries.T
    if topk_idx is None:
        topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if want_topk_scores and topk_scores is None:
        topk_scores = torch.empty((T, k), dtype=torch.float32, device=dev)
    if want_cand_scores and cand_scores is None:
        cand_scores = torch.empty((T, m * B), dtype=torch.float32, device=dev)
    qc, kc = queries.c(), keys.c()
    if ws is None:
        ws = _ws(OP_TOKEN_REFINE_TOPK, qc, kc, B, m, k, cand_scores is not None, dev)
    st = lib().hisa_token_refine_topk(C.byref(qc), C.byref(kc), B, m, _ptr(block_idx), k, _ptr(topk_idx),
                                      _ptr(topk_scores), _ptr(cand_scores), _ptr(ws),
                                      0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "hisa_token_refine_topk")
    return topk_idx, topk_scores, cand_scores


def hisa_token_refine_topk_static(queries: Queries, keys: Keys, B: int, m: int, block_idx: torch.Tensor, k: int,
                                  topk_idx: torch.Tensor, topk_scores: Optional[torch.Tensor] = None,
                                  stream=None):
    """Stage 2 (Eqs. 7-9) through the library's static scratch array: nothing is allocated, here or
    in the library, so the outputs must be passed in.  Returns (topk_idx, topk_scores)."""
    qc, kc = queries.c(), keys.c()
    st = lib().hisa_token_refine_topk_static(C.byref(qc), C.byref(kc), B, m, _ptr(block_idx), k, _ptr(topk_idx),
                                             _ptr(topk_scores), _stream(stream))
    _check(st, "hisa_token_refine_topk_static")
    return topk_idx, topk_scores


def dsa_flat_indexer_topk(queries: Queries, keys: Keys, k: int, topk_idx: Optional[torch.Tensor] = None,
                          topk_scores: Optional[torch.Tensor] = None, want_topk_scores: bool = False,
                          ws: Optional[torch.Tensor] = None, stream=None):
    """Flat DSA indexer (Eqs. 1-2).  Returns (topk_idx [T, k] int32, topk_scores or None)."""
    dev = queries.q.device
    T = queries.T
    if topk_idx is None:
        topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if want_topk_scores and topk_scores is None:
        topk_scores = torch.empty((T, k), dtype=torch.float32, device=dev)
    qc, kc = queries.c(), keys.c()
    if ws is None:
        ws = _ws(OP_FLAT_TOPK, qc, kc, 1, 0, k, False, dev)
    st = lib().dsa_flat_indexer_topk(C.byref(qc), C.byref(kc), k, _ptr(topk_idx), _ptr(topk_scores),
                                     _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "dsa_flat_indexer_topk")
    return topk_idx, topk_scores


def hisa_indexer_topk(queries: Queries, keys: Keys, pooled: torch.Tensor, pooled_dtype: int, B: int, m: int,
                      k: int, block_idx: Optional[torch.Tensor] = None, want_block_idx: bool = False,
                      topk_idx: Optional[torch.Tensor] = None, topk_scores: Optional[torch.Tensor] = None,
                      want_topk_scores: bool = False, stream=None):
    """Algorithm 1 in one launch.  Returns (block_idx or None, topk_idx, topk_scores or None)."""
    dev = queries.q.device
    T = queries.T
    if want_block_idx and block_idx is None:
        block_idx = torch.empty((T, m), dtype=torch.int32, device=dev)
    if topk_idx is None:
        topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if want_topk_scores and topk_scores is None:
        topk_scores = torch.empty((T, k), dtype=torch.float32, device=dev)
    qc, kc = queries.c(), keys.c()
    st = lib().hisa_indexer_topk(C.byref(qc), C.byref(kc), _ptr(pooled), pooled_dtype, B, m, k, _ptr(block_idx),
                                 _ptr(topk_idx), _ptr(topk_scores), _stream(stream))
    _check(st, "hisa_indexer_topk")
    return block_idx, topk_idx, topk_scores


# ---------------------------------------------------------------- the paged cache and its attention
def _on_gpu(t: torch.Tensor) -> bool:
    return t.is_cuda


def _need(t, name: str, dtypes, shape=None, device=None, contiguous: bool = True):
    """A tensor that a kernel can take as it is: on the GPU (the same one as the others), of the type and shape that the
    call goes by."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor is needed, got {type(t).__name__}")
    if not _on_gpu(t):
        raise ValueError(f"{name}: not on the GPU ({t.device})")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, the other tensors are on {device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: {t.dtype}, needed is {' or '.join(str(d) for d in dtypes)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, needed is {tuple(shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")
    return t


def _fits(t, dtype, shape, dev: int) -> bool:
    """What _need asks of a tensor, in one go: most calls pass, and a small call's time is its host side."""
    return (isinstance(t, torch.Tensor) and t.dtype is dtype and (shape is None or t.shape == shape)
            and t.get_device() == dev and t.is_contiguous())


def _gpu_of(t, name: str) -> int:
    """Index of the GPU that a call's first tensor lives on."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor is needed, got {type(t).__name__}")
    if not _on_gpu(t):
        raise ValueError(f"{name}: not on the GPU ({t.device})")
    return t.get_device()


_numel, _data_ptr, _is_contiguous = torch.Tensor.numel, torch.Tensor.data_ptr, torch.Tensor.is_contiguous
_I32 = (torch.int32,)
_F32 = (torch.float32,)
_STORED = {HISA_F32: (torch.float32,), HISA_BF16: (torch.bfloat16,),
           HISA_FP8_E4M3: (torch.float8_e4m3fn, torch.uint8)}


class _on:
    """The GPU that the tensors live on as the current one while a call is enqueued (a no-op if it is already)."""

    def __init__(self, index: int):
        self.guard = torch.cuda.device(index) if index != torch.cuda.current_device() else None

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)
        return False


def _call(fn, dev: int, stream, *args) -> int:
    """fn(*args, stream) with GPU `dev` current."""
    if dev == torch.cuda.current_device():
        return fn(*args, _stream(stream))
    with _on(dev):
        return fn(*args, _stream(stream))


def _allocating(stream, device):
    """Where a call allocates what it was not given: on the stream that it runs on, so that the memory is not handed out
    again before the kernels are done with it."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream(stream)
        stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


@dataclass
class Cache:
    """A paged cache: k, v [n_pages, page, H_kv, d] (float32 / bfloat16 / uint8 or float8 codes; any strides that k and v
    share, the last dimension contiguous, so a transposed [n_pages, H_kv, page, d] or a slice of an array that holds both
    fits), k_scale / v_scale [n_pages, page, H_kv] float32 for fp8, block_table [n_seq, max_pages] and seq_len [n_seq]
    int32; all on the GPU.  v None: keys alone, block_table and seq_len None: to append to only.  weights: what the attention
    rounds its weights to (bf16 and fp8 caches): 16 bits, or 8, which is faster where prompts are long."""
    k: torch.Tensor
    v: Optional[torch.Tensor]
    dtype: int
    block_table: Optional[torch.Tensor] = None
    seq_len: Optional[torch.Tensor] = None
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None
    weights: int = HISA_WEIGHTS_16BIT

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_c", None)

    def __getstate__(self):  # (copies build a struct of their own)
        return {name: value for name, value in self.__dict__.items() if not name.startswith("_")}

    def __post_init__(self):
        self.check()

    def check(self):
        if self.dtype not in _STORED:
            raise ValueError(f"dtype: unknown code {self.dtype}")
        if self.weights not in (HISA_WEIGHTS_16BIT, HISA_WEIGHTS_8BIT):
            raise ValueError(f"weights: unknown code {self.weights}")
        if self.k.dim() != 4:
            raise ValueError(f"k: shape {tuple(self.k.shape)}, needed is [n_pages, page, H_kv, d]")
        dev = self.k.device
        for name, t in (("k", self.k), ("v", self.v)):
            if t is None:
                continue
            _need(t, name, _STORED[self.dtype], self.k.shape, dev, contiguous=False)
            if t.stride(3) != 1 and t.shape[3] > 1:
                raise ValueError(f"{name}: the last dimension is not contiguous")
            if t.stride() != self.k.stride():
                raise ValueError(f"v: strides {t.stride()}, those of k are {self.k.stride()}")
        for name, t in (("k_scale", self.k_scale), ("v_scale", self.v_scale)):
            if t is not None:
                _need(t, name, _F32, self.k.shape[:3], dev)
        if self.block_table is not None:
            _need(self.block_table, "block_table", _I32, None, dev)
            if self.block_table.dim() != 2:
                raise ValueError("block_table: needed is [n_seq, max_pages]")
        if self.seq_len is not None:
            _need(self.seq_len, "seq_len", _I32, None if self.block_table is None else self.block_table.shape[:1], dev)

    def c(self) -> _Cache:
        k, v, ks, vs, table, length = self.k, self.v, self.k_scale, self.v_scale, self.block_table, self.seq_len
        laid = (k.shape, k.stride(), v is None or (v.shape, v.stride()),
                table is None or (table.shape, table.is_contiguous()),
                length is None or (length.shape, length.is_contiguous()),
                ks is None or (ks.shape, ks.is_contiguous()), vs is None or (vs.shape, vs.is_contiguous()))
        c = self.__dict__.get("_c")
        if c is None or self._laid != laid:
            self.check()
            n_seq, max_pages = (0, 0) if table is None else table.shape
            c = _Cache(None, None, None, None, None, None, *laid[1][:3], *laid[0][:2], n_seq, max_pages, *laid[0][2:],
                       self.dtype, self.weights)
            self.__dict__.update(_laid=laid, _c=c)
        # The sizes stay while all tensors keep theirs (the struct costs 3 us to build); where memory lies is asked anew.
        c.k = k.data_ptr()
        c.v = None if v is None else v.data_ptr()
        c.k_scale = None if ks is None else ks.data_ptr()
        c.v_scale = None if vs is None else vs.data_ptr()
        c.block_table = None if table is None else table.data_ptr()
        c.seq_len = None if length is None else length.data_ptr()
        return c


@dataclass
class PageTables:
    """What hisa_page_tables writes: seq_len [n_seq], q_start and page_start [n_seq + 1], q_seq, q_pos, slots and (or
    None) key_rows [rows], all int32."""
    seq_len: torch.Tensor
    q_start: torch.Tensor
    page_start: torch.Tensor
    q_seq: torch.Tensor
    q_pos: torch.Tensor
    slots: torch.Tensor
    key_rows: Optional[torch.Tensor] = None

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_checked", None)

    def pointers(self, n_seq: int, rows: int, dev: int, device) -> list:
        """Where the seven tensors lie.  Their types and layout are checked once for a batch's sizes, and again if a
        tensor is replaced, resized or laid out otherwise."""
        checked = self.__dict__.get("_checked")
        if (checked is None or checked[0] != (n_seq, rows, dev) or tuple(map(_numel, checked[1])) != checked[2]
                or not all(map(_is_contiguous, checked[1]))):
            names = ("seq_len", "q_start", "page_start", "q_seq", "q_pos", "slots", "key_rows")[:6 + (self.key_rows is not None)]
            sizes = (n_seq, n_seq + 1, n_seq + 1, rows, rows, rows, rows)[:len(names)]
            tensors = tuple(_need(getattr(self, name), name, _I32, (n,), device) for name, n in zip(names, sizes))
            checked = self.__dict__["_checked"] = ((n_seq, rows, dev), tensors, sizes)
        lie = list(map(_data_ptr, checked[1]))
        return lie if len(lie) == 7 else lie + [None]

    @property
    def pages_used(self) -> torch.Tensor:
        """[1]: how many of the free pages are in use now (more than there were: too few)."""
        return self.page_start[-1:]

    @staticmethod
    def empty(n_seq: int, rows: int, device, key_rows: bool = False) -> "PageTables":
        def new(n):
            return torch.empty((n,), dtype=torch.int32, device=device)

        return PageTables(new(n_seq), new(n_seq + 1), new(n_seq + 1), new(rows), new(rows), new(rows),
                          new(rows) if key_rows else None)


def hisa_page_tables(ctx_len: torch.Tensor, new_len: torch.Tensor, block_table: torch.Tensor, page: int,
                     free_pages: torch.Tensor, rows: int, s_max: int = 0, out: Optional[PageTables] = None,
                     stream=None) -> PageTables:
    """Block tables (updated in place) and slot maps of a batch from its requests' lengths; s_max > 0: key_rows too, the
    tokens' rows in a padded key array [n_seq, s_max, d]."""
    i32 = torch.int32
    dev = _gpu_of(ctx_len, "ctx_len")
    n_seq = ctx_len.numel()
    seqs, device = (n_seq,), ctx_len.device
    _fits(ctx_len, i32, seqs, dev) or _need(ctx_len, "ctx_len", _I32, seqs)
    _fits(new_len, i32, seqs, dev) or _need(new_len, "new_len", _I32, seqs, device)
    n_free = free_pages.numel()
    _fits(free_pages, i32, (n_free,), dev) or _need(free_pages, "free_pages", _I32, (n_free,), device)
    if block_table.dim() != 2 or block_table.shape[0] != n_seq:
        raise ValueError(f"block_table: shape {tuple(block_table.shape)}, needed is [{n_seq}, max_pages]")
    _fits(block_table, i32, None, dev) or _need(block_table, "block_table", _I32, None, device)
    if rows < 1:
        raise ValueError(f"rows: {rows}")
    if out is None:
        with _allocating(stream, device):
            out = PageTables.empty(n_seq, rows, device, key_rows=s_max > 0)
    st = _call(lib().hisa_page_tables, dev, stream, ctx_len.data_ptr(), new_len.data_ptr(), n_seq, block_table.data_ptr(),
               block_table.shape[1], page, free_pages.data_ptr(), n_free, rows, s_max,
               *out.pointers(n_seq, rows, dev, device))
    _check(st, "hisa_page_tables")
    return out


def hisa_cache_append(cache: Cache, slots: torch.Tensor, k_new: torch.Tensor, v_new: Optional[torch.Tensor] = None,
                      stream=None) -> None:
    """Rows k_new (and v_new) [T, H_kv, d] into the slots [T] of the cache, converted to its type.  The rows of a token
    are contiguous, tokens may lie further apart (a slice of a wider projection), keys and values alike."""
    k = cache.k
    dev = _gpu_of(k, "k")
    T = slots.numel()
    _fits(slots, torch.int32, (T,), dev) or _need(slots, "slots", _I32, (T,), k.device)
    H_kv, d = k.shape[2:]
    shape, dtype = (T, H_kv, d), k_new.dtype
    stride = H_kv * d
    if not (_fits(k_new, dtype, shape, dev) and (dtype is torch.bfloat16 or dtype is torch.float32)
            and (v_new is None or _fits(v_new, dtype, shape, dev))):
        # tokens further apart, or something that does not fit
        stride = k_new.stride(0) if k_new.dim() == 3 and T > 1 else stride
        for name, t in (("k_new", k_new), ("v_new", v_new)):
            if t is None:
                continue
            _need(t, name, (torch.float32, torch.bfloat16), shape, k.device, contiguous=False)
            if t.dtype != dtype:
                raise ValueError(f"v_new: {t.dtype}, k_new is {dtype}")
            if T and not t[0].is_contiguous():
                raise ValueError(f"{name}: the rows of a token are not contiguous")
            if T > 1 and t.stride(0) != stride:
                raise ValueError(f"v_new: tokens {t.stride(0)} elements apart, those of k_new {stride}")
    st = _call(lib().hisa_cache_append, dev, stream, cache.c(), slots.data_ptr(), k_new.data_ptr(),
               None if v_new is None else v_new.data_ptr(), HISA_F32 if dtype is torch.float32 else HISA_BF16, stride, T)
    _check(st, "hisa_cache_append")


def hisa_attention_workspace_bytes(queries: Queries, cache: Cache, k: int = 0) -> int:
    """Workspace of hisa_paged_attention (k == 0) or hisa_sparse_attention (k positions per query).  A smaller batch may
    need more than a larger one: a program with several sizes takes the largest of their answers."""
    qc, cc = queries.c(), cache.c()
    return int(lib().hisa_attention_workspace_bytes(C.byref(qc), C.byref(cc), k))


def _attention(name: str, queries: Queries, cache: Cache, index: torch.Tensor, k: int, scale, out, lse, want_lse, ws,
               stream):
    q, ck = queries.q, cache.k
    dev, device = _gpu_of(ck, "k"), ck.device
    dtype = torch.float32 if queries.dtype == HISA_F32 else torch.bfloat16
    _fits(q, dtype, None, dev) or _need(q, "q", (dtype,), None, device)
    if q.dim() != 3 or q.shape[2] != ck.shape[3]:
        raise ValueError(f"q: shape {tuple(q.shape)}, needed is [T, H, {ck.shape[3]}]")
    T, H, d = q.shape
    rows, ptrs = (T,), []
    for what, t in (("q_seq", queries.q_seq), ("q_pos", queries.q_pos), ("q_lo", queries.q_lo)):
        if t is not None:
            _fits(t, torch.int32, rows, dev) or _need(t, what, _I32, rows, device)
        ptrs.append(None if t is None else t.data_ptr())
    if out is None:
        with _allocating(stream, device):
            out = torch.empty_like(q)
    else:
        _fits(out, dtype, q.shape, dev) or _need(out, "out", (dtype,), q.shape, device)
    if lse is not None:
        _fits(lse, torch.float32, (T, H), dev) or _need(lse, "lse", _F32, (T, H), device)
    elif want_lse:
        with _allocating(stream, device):
            lse = torch.empty((T, H), dtype=torch.float32, device=device)
    qc, cc = _Queries(q.data_ptr(), None, *ptrs, T, H, 0, queries.dtype), cache.c()
    L = lib()
    if ws is None:
        size = int(L.hisa_attention_workspace_bytes(qc, cc, k))
        with _allocating(stream, device):
            ws = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    else:
        size = ws.numel()
        _fits(ws, torch.uint8, None, dev) or _need(ws, "ws", (torch.uint8,), None, device)
    scale = d ** -0.5 if scale is None else float(scale)
    ptrs = (scale, out.data_ptr(), None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(), size)
    if k:
        st = _call(L.hisa_sparse_attention, dev, stream, qc, cc, index.data_ptr(), k, *ptrs)
    else:
        st = _call(L.hisa_paged_attention, dev, stream, qc, cc, index.data_ptr(), *ptrs)
    _check(st, name)
    return out, lse


def hisa_paged_attention(queries: Queries, cache: Cache, q_start: torch.Tensor, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                         ws: Optional[torch.Tensor] = None, stream=None):
    """Attention of new tokens over the paged cache; scale: d ** -0.5 unless given.  Returns (out [T, H, d], lse [T, H]
    or None)."""
    if cache.block_table is None or cache.seq_len is None or cache.v is None:
        raise ValueError("cache: values, block_table and seq_len are needed")
    shape = (cache.block_table.shape[0] + 1,)
    _fits(q_start, torch.int32, shape, cache.k.get_device()) or _need(q_start, "q_start", _I32, shape, cache.k.device)
    return _attention("hisa_paged_attention", queries, cache, q_start, 0, scale, out, lse, want_lse, ws, stream)


def hisa_sparse_attention(queries: Queries, cache: Cache, topk_idx: torch.Tensor, scale: Optional[float] = None,
                          out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                          ws: Optional[torch.Tensor] = None, stream=None):
    """Attention over the positions topk_idx [T, k] of each query (entries outside the sequence, -1 among them, are
    skipped).  Returns (out [T, H, d], lse [T, H] or None)."""
    if cache.block_table is None or cache.seq_len is None or cache.v is None:
        raise ValueError("cache: values, block_table and seq_len are needed")
    _fits(topk_idx, torch.int32, None, cache.k.get_device()) or _need(topk_idx, "topk_idx", _I32, None,
                                                                                 cache.k.device)
    if topk_idx.dim() != 2 or topk_idx.shape[0] != queries.T or topk_idx.shape[1] < 1:
        raise ValueError(f"topk_idx: shape {tuple(topk_idx.shape)}, needed is [{queries.T}, k]")
    return _attention("hisa_sparse_attention", queries, cache, topk_idx, topk_idx.shape[1], scale, out, lse, want_lse, ws,
                      stream)


def hisa_probe_copy(src: torch.Tensor, dst: torch.Tensor, stream=None) -> int:
    """Streaming copy probe; returns the bytes moved (read + written)."""
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    _check(lib().hisa_probe_copy(_ptr(src), _ptr(dst), nbytes, _stream(stream)), "hisa_probe_copy")
    return 2 * nbytes


def hisa_probe_mfma(out: torch.Tensor, iters: int, stream=None) -> float:
    """MFMA-only probe; `out` holds at least 512 * 256 floats; returns the flop count of the launch."""
    assert out.dtype == torch.float32 and out.numel() >= 512 * 256
    flop = C.c_double(0.0)
    _check(lib().hisa_probe_mfma(_ptr(out), iters, C.byref(flop), _stream(stream)), "hisa_probe_mfma")
    return flop.value


def hisa_probe_mfma_fp8(out: torch.Tensor, iters: int, stream=None) -> float:
    """The same probe on the fp8 MFMA (e4m3 x e4m3)."""
    assert out.dtype == torch.float32 and out.numel() >= 512 * 256
    flop = C.c_double(0.0)
    _check(lib().hisa_probe_mfma_fp8(_ptr(out), iters, C.byref(flop), _stream(stream)), "hisa_probe_mfma_fp8")
    return flop.value


def hisa_probe_mfma_toggling(out: torch.Tensor, iters: int, fp8: bool = False, stream=None) -> float:
    """Either MFMA probe on operands that differ per lane and per instruction (pseudo-random values)."""
    assert out.dtype == torch.float32 and out.numel() >= 512 * 256
    flop = C.c_double(0.0)
    _check(lib().hisa_probe_mfma_toggling(_ptr(out), iters, 1 if fp8 else 0, C.byref(flop), _stream(stream)),
           "hisa_probe_mfma_toggling")
    return flop.value


# ---------------------------------------------------------------- moving a workload to the GPU
def to_device(wl, device="cuda:0"):
    """(Queries, Keys) on the GPU from a workloads.Workload (host numpy bits): copies only."""
    import numpy as np

    def dev(a, view=None):
        if a is None:
            return None
        t = torch.from_numpy(np.ascontiguousarray(a))
        if view is not None:
            t = t.view(view)
        return t.to(device)

    kview = {"f32": None, "bf16": torch.bfloat16, "fp8_e4m3": None}[wl.k_dtype]
    kk = wl.keys.view(np.int16) if wl.k_dtype == "bf16" else wl.keys
    qq = wl.q.view(np.int16) if wl.q_dtype == "bf16" else wl.q
    keys = Keys(k=dev(kk, kview), seq_len=dev(wl.seq_len.astype(np.int32)), dtype=DTYPE_CODE[wl.k_dtype],
                k_scale=dev(wl.k_scale))
    queries = Queries(q=dev(qq, torch.bfloat16 if wl.q_dtype == "bf16" else None), w=dev(wl.w),
                      dtype=DTYPE_CODE[wl.q_dtype], q_seq=dev(wl.q_seq), q_pos=dev(wl.q_pos),
                      q_pos0=wl.q_pos0, q_lo=dev(getattr(wl, "q_lo", None)))
    return queries, keys
