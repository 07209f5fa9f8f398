"""Python face of the C-ABI library `libgvote.so` (declared in include/gvote.h).

Argument marshalling only: every function takes torch tensors (for device memory and the
current stream), checks dtype/device, and passes raw pointers, strides and sizes to the
entry point of the same name.  No step of the pass is computed here, and there is no
fallback: a missing library raises at the first call.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libgvote.so")
_lib = None

GVOTE_OK = 0
SEL_TOPK_C0, SEL_TOPP = 0, 1
DTYPE_F32, DTYPE_BF16 = 0, 1

EXPORTS = (
    "gvote_workspace_bytes", "gvote_workspace_queries", "gvote_fit", "gvote_fit_update", "gvote_fit_finish", "gvote_fit_static", "gvote_sample", "gvote_project", "gvote_vote", "gvote_select",
    "gvote_compact", "gvote_pack", "gvote_overlap", "gvote_compress", "gvote_compress_moments", "gvote_recompress", "gvote_cache_workspace_bytes", "gvote_store8", "gvote_prune8", "gvote_append8", "gvote_attend8",
    "gvote_accumulate", "gvote_evict", "gvote_attend_workspace_bytes", "gvote_page_tables", "gvote_page_write", "gvote_page_attend", "gvote_attend", "gvote_compress_host", "gvote_host_arena_release",
    "gvote_poll_status", "gvote_clear_status", "gvote_exact_heads", "gvote_profile_enable", "gvote_profile_report", "gvote_launch_count", "gvote_status_string", "gvote_last_cuda_error",
)


class GVoteParams(ctypes.Structure):
    """Mirror of `gvote_params` (same field order and C types)."""
    _fields_ = [
        ("d_h", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("d_k", ctypes.c_int32), ("rope_theta", ctypes.c_double), ("S", ctypes.c_int32),
        ("p_nuc", ctypes.c_float), ("n_f", ctypes.c_int32), ("n_s", ctypes.c_int32),
        ("sel_mode", ctypes.c_int32), ("include_c0", ctypes.c_int32), ("seed", ctypes.c_uint64),
        ("layer_id", ctypes.c_uint32), ("h_dtype", ctypes.c_int32),
    ]


class GVoteCache8(ctypes.Structure):
    """Mirror of `gvote_cache8`."""
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("cu_seqlens", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("tok_stride", ctypes.c_int64),
        ("head_stride", ctypes.c_int64), ("total_tokens", ctypes.c_int64), ("max_N", ctypes.c_int64),
        ("batch", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class Cache8:
    """An 8-bit cache: e4m3 codes K, V (uint8 [n_kv_heads, total_tokens, d_k]), one power-of-two scale per 64 rows
    of a head (float32 [n_kv_heads, cache8_row_blocks]), slab boundaries cu_seqlens (int32 [batch+1]), rows held
    kv_len (int32 [batch, n_kv_heads]) and geom = (batch, total_tokens, longest slab).  `alloc_cache8` makes one.
    The tensors are checked here, once; the entry points take the finished argument block."""
    __slots__ = ("K", "V", "k_scale", "v_scale", "cu_seqlens", "kv_len", "geom", "shape", "device", "args")

    def __init__(self, K, V, k_scale, v_scale, cu_seqlens, kv_len, geom):
        batch, total, max_N = geom
        H, _, d = K.shape
        blocks = cache8_row_blocks(total, batch)
        if K.stride() != V.stride():
            raise ValueError("K and V must share strides")
        dev = K.device
        self.args = GVoteCache8(
            _shaped(K, torch.uint8, (H, total, d), "K", dev, dense=False),
            _shaped(V, torch.uint8, (H, total, d), "V", dev, dense=False),
            _shaped(k_scale, torch.float32, (H, blocks), "k_scale", dev),
            _shaped(v_scale, torch.float32, (H, blocks), "v_scale", dev),
            _shaped(cu_seqlens, torch.int32, (batch + 1,), "cu_seqlens", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), K.stride(1), K.stride(0), total, max_N, batch, 0)
        self.K, self.V, self.k_scale, self.v_scale = K, V, k_scale, v_scale
        self.cu_seqlens, self.kv_len, self.geom = cu_seqlens, kv_len, (batch, total, max_N)
        self.shape, self.device = (H, d), dev

    def __setattr__(self, name, value):
        if hasattr(self, name):
            raise AttributeError(f"{name} of a Cache8 is fixed (its pointers are taken once): make another Cache8")
        object.__setattr__(self, name, value)


class GVotePages(ctypes.Structure):
    """Mirror of `gvote_pages`."""
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("tables", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
        ("free_pages", ctypes.c_void_p), ("n_free", ctypes.c_void_p), ("row_stride", ctypes.c_int64),
        ("page_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32), ("page_rows", ctypes.c_int32),
        ("max_pages", ctypes.c_int32), ("batch", ctypes.c_int32),
    ]


def _same_strides(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether a and b are laid out alike (the stride of a dimension of one may be anything)."""
    return a.stride() == b.stride() or all(n <= 1 or x == y for n, x, y in zip(a.shape, a.stride(), b.stride()))


class PageCache:
    """A paged cache: pages K, V (bfloat16 [n_pages, page_rows, d_k]), tables (int32 [batch, n_kv_heads, max_pages]), rows
    held kv_len (int32 [batch, n_kv_heads]) and the stack of unused pages free (int32 [n_pages]) of height n_free (int32 [1]).
    `alloc_pages` makes one.  The tensors are checked here, once; the entry points take the finished argument block."""
    __slots__ = ("K", "V", "tables", "kv_len", "free", "n_free", "shape", "device", "args")

    def __init__(self, K, V, tables, kv_len, free, n_free):
        n_pages, page_rows, d = K.shape
        batch, H, max_pages = tables.shape
        if not _same_strides(K, V):
            raise ValueError("K and V must share strides")
        dev = K.device
        self.args = GVotePages(
            _shaped(K, torch.bfloat16, (n_pages, page_rows, d), "K", dev, dense=False),
            _shaped(V, torch.bfloat16, (n_pages, page_rows, d), "V", dev, dense=False),
            _shaped(tables, torch.int32, (batch, H, max_pages), "tables", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), _shaped(free, torch.int32, (n_pages,), "free", dev),
            _shaped(n_free, torch.int32, (1,), "n_free", dev), K.stride(1), K.stride(0), n_pages, page_rows, max_pages, batch)
        self.K, self.V, self.tables, self.kv_len, self.free, self.n_free = K, V, tables, kv_len, free, n_free
        self.shape, self.device = (H, d), dev

    def __setattr__(self, name, value):
        if hasattr(self, name):
            raise AttributeError(f"{name} of a PageCache is fixed (its pointers are taken once): make another PageCache")
        object.__setattr__(self, name, value)


class GVoteError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = load()
        msg = lib.gvote_status_string(status).decode()
        cuda = lib.gvote_last_cuda_error().decode()
        super().__init__(f"{where}: {msg} ({status})" + (f": {cuda}" if status == -5 and cuda else ""))
        self.status = status


def load():
    """Load libgvote.so (built by `python -m paper_2509_03136_b200.build`).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2509_03136_b200.build` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    C8 = ctypes.POINTER(GVoteCache8)
    PG = ctypes.POINTER(GVotePages)
    P, vp, i32, i64, sz = ctypes.POINTER(GVoteParams), ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.gvote_workspace_bytes.restype = sz
    lib.gvote_workspace_bytes.argtypes = [P, i32, i64, i64]
    lib.gvote_workspace_queries.restype = sz
    lib.gvote_workspace_queries.argtypes = [P, i32, i64, i64]
    lib.gvote_fit.restype = i32
    lib.gvote_fit.argtypes = [P, vp, i64, vp, i32, i64, i64, vp, vp, vp, sz, vp]
    lib.gvote_fit_update.restype = i32
    lib.gvote_fit_update.argtypes = [P, vp, i64, vp, i32, i64, i64, vp, vp, sz, vp]
    lib.gvote_fit_finish.restype = i32
    lib.gvote_fit_finish.argtypes = [P, vp, i32, vp, vp, vp]
    lib.gvote_compress_moments.restype = i32
    lib.gvote_compress_moments.argtypes = [P, vp, vp, vp, vp, i64, vp, vp, vp, i64, i64, vp, i32, i64, i64, vp, vp, vp,
                                           vp, sz, vp]
    lib.gvote_recompress.restype = i32
    lib.gvote_recompress.argtypes = [P, vp, vp, vp, vp, i64, vp, vp, vp, i64, i64, vp, vp, vp, vp, i32, i64, i64, vp, vp,
                                     vp, vp, sz, vp]
    lib.gvote_fit_static.restype = i32
    lib.gvote_fit_static.argtypes = [P, vp, i64, vp, i32, i64, vp, vp, vp]
    lib.gvote_sample.restype = i32
    lib.gvote_sample.argtypes = [P, vp, vp, i32, vp, vp, vp]
    lib.gvote_project.restype = i32
    lib.gvote_project.argtypes = [P, vp, vp, vp, i64, vp, vp, i32, vp, vp, sz, vp]
    lib.gvote_vote.restype = i32
    lib.gvote_vote.argtypes = [P, vp, vp, i64, i64, vp, i32, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.gvote_select.restype = i32
    lib.gvote_select.argtypes = [P, vp, vp, vp, i64, vp, vp, i64, i64, vp, i32, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    lib.gvote_compact.restype = i32
    lib.gvote_compact.argtypes = [P, vp, vp, i64, i64, vp, vp, i32, i64, i64, vp, vp, sz, vp]
    lib.gvote_overlap.restype = i32
    lib.gvote_overlap.argtypes = [P, vp, vp, i64, i64, vp, vp, i32, i64, i64, vp, vp, sz, vp]
    lib.gvote_pack.restype = i32
    lib.gvote_pack.argtypes = [P, vp, vp, i64, i64, vp, vp, i32, i64, i64, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.gvote_compress.restype = i32
    lib.gvote_compress.argtypes = [P, vp, i64, vp, vp, i64, vp, vp, vp, i64, i64, vp, i32, i64, i64, vp, vp, vp,
                                   vp, sz, vp]
    lib.gvote_cache_workspace_bytes.restype = sz
    lib.gvote_cache_workspace_bytes.argtypes = [P, i32, i64, i64, i64, i64]
    lib.gvote_store8.restype = i32
    lib.gvote_store8.argtypes = [P, vp, vp, i64, i64, vp, vp, vp, i32, i64, i64, C8, vp, vp, vp, vp, vp, sz, vp]
    lib.gvote_prune8.restype = i32
    lib.gvote_prune8.argtypes = [P, C8, vp, C8, vp, vp, vp, vp, vp, sz, vp]
    lib.gvote_append8.restype = i32
    lib.gvote_append8.argtypes = [P, vp, vp, i64, i64, vp, i64, i64, C8, vp, vp, vp, vp, vp, sz, vp]
    lib.gvote_attend8.restype = i32
    lib.gvote_attend8.argtypes = [P, vp, i64, i64, vp, i64, i64, C8, vp, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.gvote_accumulate.restype = i32
    lib.gvote_accumulate.argtypes = [P, vp, i64, i64, vp, i64, i64, vp, i64, i64, vp, vp, i32, i64, i64, vp, vp, vp, vp,
                                     sz, vp]
    lib.gvote_evict.restype = i32
    lib.gvote_evict.argtypes = [P, vp, vp, vp, i32, i64, i64, vp, i32, vp, vp, vp, sz, vp]
    lib.gvote_attend_workspace_bytes.restype = sz
    lib.gvote_attend_workspace_bytes.argtypes = [P, i32, i64, i64]
    lib.gvote_page_tables.restype = i32
    lib.gvote_page_tables.argtypes = [P, PG, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.gvote_page_write.restype = i32
    lib.gvote_page_write.argtypes = [P, vp, vp, i64, i64, vp, i64, PG, vp, sz, vp]
    lib.gvote_page_attend.restype = i32
    lib.gvote_page_attend.argtypes = [P, vp, i64, i64, vp, i64, i64, PG, vp, i64, i64, vp, vp, sz, vp]
    lib.gvote_attend.restype = i32
    lib.gvote_attend.argtypes = [P, vp, i64, i64, vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i64, i64, vp, i64, i64, vp,
                                 vp, sz, vp]
    lib.gvote_compress_host.restype = i32
    lib.gvote_compress_host.argtypes = [P, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.gvote_host_arena_release.restype = None
    lib.gvote_host_arena_release.argtypes = []
    lib.gvote_poll_status.restype = i32
    lib.gvote_poll_status.argtypes = [vp, vp]
    lib.gvote_clear_status.restype = i32
    lib.gvote_clear_status.argtypes = [vp, vp]
    lib.gvote_exact_heads.restype = i64
    lib.gvote_exact_heads.argtypes = [vp, vp]
    lib.gvote_profile_enable.restype = None
    lib.gvote_profile_enable.argtypes = [i32]
    lib.gvote_profile_report.restype = sz
    lib.gvote_profile_report.argtypes = [ctypes.c_char_p, sz]
    lib.gvote_launch_count.restype = i64
    lib.gvote_launch_count.argtypes = []
    lib.gvote_status_string.restype = ctypes.c_char_p
    lib.gvote_status_string.argtypes = [i32]
    lib.gvote_last_cuda_error.restype = ctypes.c_char_p
    lib.gvote_last_cuda_error.argtypes = []
    _lib = lib
    return lib


# ----------------------------------------------------------------------------- helpers
def make_params(*, d_h: int, n_q_heads: int, n_kv_heads: int, d_k: int, rope_theta: float, S: int,
                p_nuc: float, n_f: int, n_s: int, seed: int, layer_id: int = 0, sel_mode: int = SEL_TOPK_C0,
                include_c0: bool = False, h_dtype: int = DTYPE_F32) -> GVoteParams:
    return GVoteParams(d_h, n_q_heads, n_kv_heads, d_k, float(rope_theta), S, float(p_nuc), n_f, n_s, sel_mode,
                       int(bool(include_c0)), int(seed) & 0xFFFFFFFFFFFFFFFF, int(layer_id) & 0xFFFFFFFF, h_dtype)


def params_from_config(cfg, layer_id: int = 0, **kw) -> GVoteParams:
    """Parameters for a `synth.GVoteConfig`."""
    return make_params(d_h=cfg.d_h, n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads, d_k=cfg.d_k,
                       rope_theta=cfg.rope_theta, S=cfg.S, p_nuc=cfg.p_nuc, n_f=cfg.n_f, n_s=cfg.n_s,
                       seed=cfg.seed, layer_id=layer_id, **kw)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _check(status: int, where: str) -> None:
    if status != GVOTE_OK:
        raise GVoteError(status, where)


def _dev(t: torch.Tensor, dtype, name: str, dense: bool = True) -> torch.Tensor:
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if dense and not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    if not dense and t.stride(-1) != 1:
        raise TypeError(f"{name} must be contiguous along its last dimension")
    return t


def mask_row_words(total_tokens: int, batch: int) -> int:
    return (total_tokens >> 5) + batch


def mask_word_offset(cu_r: int, r: int) -> int:
    return (cu_r >> 5) + r


def batch_geometry(cu_seqlens_host: Sequence[int]) -> Tuple[int, int, int]:
    """(batch, total_tokens, max_N) from host-side cumulative lengths."""
    cu = [int(x) for x in cu_seqlens_host]
    return len(cu) - 1, cu[-1], max((b - a for a, b in zip(cu[:-1], cu[1:])), default=0)


def gvote_workspace_bytes(p: GVoteParams, batch: int, total_tokens: int, max_N: int) -> int:
    return int(load().gvote_workspace_bytes(ctypes.byref(p), batch, total_tokens, max_N))


def workspace_queries(p: GVoteParams, ws: torch.Tensor, batch: int, total_tokens: int, max_N: int) -> torch.Tensor:
    """The rotated queries a whole-pass call left in `ws`: a bf16 view [batch, n_kv_heads, G*(S+1), d_k]."""
    off = int(load().gvote_workspace_queries(ctypes.byref(p), batch, total_tokens, max_N))
    if off == 0:
        raise GVoteError(-1, "gvote_workspace_queries")
    G = p.n_q_heads // p.n_kv_heads
    n = batch * p.n_kv_heads * G * (p.S + 1) * p.d_k
    return ws[off:off + 2 * n].view(torch.bfloat16).view(batch, p.n_kv_heads, G * (p.S + 1), p.d_k)


def alloc_workspace(p: GVoteParams, batch: int, total_tokens: int, max_N: int, device="cuda",
                    softmax_dump: bool = False) -> torch.Tensor:
    """A zero-filled workspace for these parameters.  softmax_dump=True sizes it for calls that ask
    gvote_vote / gvote_select for the softmax rows (dbg_probs): those keep the fp32 logits of every row,
    like the per-sample top-p mode, so the size is that mode's."""
    if softmax_dump and p.sel_mode != SEL_TOPP:
        q = GVoteParams.from_buffer_copy(p)
        q.sel_mode = SEL_TOPP
        p = q
    n = gvote_workspace_bytes(p, batch, total_tokens, max_N)
    if n == 0:
        raise GVoteError(-1, "gvote_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


CACHE8_BLOCK = 64
ATTEND8_MAX_Q = 32


def cache8_row_blocks(total_tokens: int, batch: int) -> int:
    return (total_tokens >> 6) + batch


def cache8_block_offset(cu_r: int, r: int) -> int:
    return (cu_r >> 6) + r


def alloc_cache8(p: GVoteParams, cu_seqlens_host: Sequence[int], device="cuda") -> Cache8:
    """An empty 8-bit cache with these slabs (zero-filled)."""
    batch, total, max_N = geom = batch_geometry(cu_seqlens_host)
    K, V = (torch.zeros(p.n_kv_heads, total, p.d_k, dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros(p.n_kv_heads, cache8_row_blocks(total, batch), device=device) for _ in range(2))
    cu = torch.tensor([int(x) for x in cu_seqlens_host], dtype=torch.int32, device=device)
    return Cache8(K, V, ks, vs, cu, torch.zeros(batch, p.n_kv_heads, dtype=torch.int32, device=device), geom)


def alloc_cache_workspace(p: GVoteParams, batch: int, total_tokens: int, max_N: int, total_q: int = 0, max_q: int = 0,
                          device="cuda") -> torch.Tensor:
    """A zero-filled workspace for the entry points of the 8-bit cache and the eviction: slabs of this geometry,
    total_q query tokens in all and at most max_q of one request."""
    n = int(load().gvote_cache_workspace_bytes(ctypes.byref(p), batch, total_tokens, max_N, total_q, max_q))
    if n == 0:
        raise GVoteError(-1, "gvote_cache_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


ATTEND_FEW_Q = 32


def alloc_pages(p: GVoteParams, batch: int, n_pages: int, page_rows: int, max_pages: int, device="cuda") -> PageCache:
    """An empty paged cache: every page unused, tables of max_pages pages per head, the first page on top of the stack."""
    K, V = (torch.zeros(n_pages, page_rows, p.d_k, dtype=torch.bfloat16, device=device) for _ in range(2))
    return PageCache(K, V, torch.zeros(batch, p.n_kv_heads, max_pages, dtype=torch.int32, device=device),
                     torch.zeros(batch, p.n_kv_heads, dtype=torch.int32, device=device),
                     torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                     torch.full((1,), n_pages, dtype=torch.int32, device=device))


def alloc_attend_workspace(p: GVoteParams, batch: int, total_q: int = 0, max_q: int = 0, device="cuda") -> torch.Tensor:
    """A zero-filled workspace for the entry points of the paged cache and for gvote_attend: total_q query tokens in all and at
    most max_q of one request.  It is for these entry points alone."""
    n = int(load().gvote_attend_workspace_bytes(ctypes.byref(p), batch, total_q, max_q))
    if n == 0:
        raise GVoteError(-1, "gvote_attend_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def _shaped(t: Optional[torch.Tensor], dtype, shape, name: str, dev: torch.device, dense: bool = True) -> Optional[int]:
    """The pointer of a tensor of this type and shape on `dev`; None stays None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.device == dev and dev.type == "cuda" and t.is_contiguous():
        return t.data_ptr() or None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != dev or not t.is_cuda:
        raise (TypeError if not t.is_cuda else ValueError)(f"{name} is on {t.device}, must be on {dev} (a CUDA device)")
    if not t.is_contiguous() and (dense or t.stride(-1) != 1):
        raise TypeError(f"{name} must be contiguous" + ("" if dense else " along its last dimension"))
    return t.data_ptr() or None


def _cache8(p, c: Cache8, name: str, dev: torch.device):
    if c.device != dev:
        raise ValueError(f"{name} is on {c.device}, must be on {dev}")
    if c.shape != (p.n_kv_heads, p.d_k):
        raise ValueError(f"{name} holds {c.shape[0]} heads of {c.shape[1]} values, the parameters say "
                         f"{p.n_kv_heads} of {p.d_k}")
    return ctypes.byref(c.args)


def _pages(p, c: PageCache, dev: torch.device):
    if c.device != dev:
        raise ValueError(f"pages are on {c.device}, must be on {dev}")
    if c.shape != (p.n_kv_heads, p.d_k):
        raise ValueError(f"pages hold {c.shape[0]} heads of {c.shape[1]} values, the parameters say {p.n_kv_heads} of {p.d_k}")
    return ctypes.byref(c.args)


# The current device and its stream's handle, by the calls that make no objects (1.5 us of a call's 14) where torch has them.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _launch(entry, dev: torch.device, p, *args, ws: torch.Tensor) -> None:
    """Calls a library entry point with its workspace on the current stream of the tensors' device."""
    n = ws.numel()
    wp = _shaped(ws, torch.uint8, (n,), "ws", dev)
    here = _current_device()
    if dev.index != here:
        raise ValueError(f"the tensors are on {dev}, the current device is cuda:{here}")
    status = entry(ctypes.byref(p), *args, wp, n, _raw_stream(here))
    if status:
        raise GVoteError(status, entry.__name__)


# ----------------------------------------------------------------------------- entry points
def gvote_fit(p, h, cu_seqlens, geom, mu, var, ws) -> None:
    batch, total, max_N = geom
    _dev(h, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h", dense=False)
    _dev(cu_seqlens, torch.int32, "cu_seqlens"); _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var")
    _check(load().gvote_fit(ctypes.byref(p), _ptr(h), h.stride(0), _ptr(cu_seqlens), batch, total, max_N,
                            _ptr(mu), _ptr(var), _ptr(ws), ws.numel(), _stream()), "gvote_fit")


def gvote_fit_update(p, h_block, cu_block, geom, state, ws) -> None:
    """Fold one block of hidden-state rows (requests packed by cu_block) into the running moments
    `state` [batch, 3, d_h] float64 (zero-filled before the first block)."""
    batch, total, max_rows = geom
    _dev(h_block, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h_block", dense=False)
    _dev(cu_block, torch.int32, "cu_block"); _dev(state, torch.float64, "state")
    _check(load().gvote_fit_update(ctypes.byref(p), _ptr(h_block), h_block.stride(0), _ptr(cu_block), batch, total,
                                   max_rows, _ptr(state), _ptr(ws), ws.numel(), _stream()), "gvote_fit_update")


def gvote_fit_finish(p, state, batch, mu, var) -> None:
    _dev(state, torch.float64, "state"); _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var")
    _check(load().gvote_fit_finish(ctypes.byref(p), _ptr(state), batch, _ptr(mu), _ptr(var), _stream()),
           "gvote_fit_finish")


def gvote_compress_moments(p, mu, var, h_last, W_q, b_q, K, V, cu_seqlens, geom, mask, budget, b_step, ws) -> None:
    batch, total, max_N = geom
    _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var")
    _dev(h_last, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h_last")
    _dev(W_q, torch.bfloat16, "W_q", dense=False); _dev(K, torch.bfloat16, "K", dense=False); _dev(V, torch.bfloat16, "V", dense=False)
    _dev(mask, torch.int32, "mask"); _dev(budget, torch.int32, "budget"); _dev(b_step, torch.int32, "b_step")
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    _check(load().gvote_compress_moments(ctypes.byref(p), _ptr(mu), _ptr(var), _ptr(h_last), _ptr(W_q), W_q.stride(0),
                                         _ptr(b_q), _ptr(K), _ptr(V), K.stride(1), K.stride(0), _ptr(cu_seqlens),
                                         batch, total, max_N, _ptr(mask), _ptr(budget), _ptr(b_step), _ptr(ws),
                                         ws.numel(), _stream()), "gvote_compress_moments")


def gvote_recompress(p, mu, var, h_last, W_q, b_q, K, V, cu_seqlens, kv_len, seq_len, token_pos, geom, mask, budget,
                     b_step, ws) -> None:
    """The pass on a cache pruned before: kv_len [batch, n_kv_heads] rows per head, seq_len [batch] tokens
    seen, token_pos [n_kv_heads, total] slot -> position map (or None), compacted with the rows."""
    batch, total, max_N = geom
    _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var")
    _dev(h_last, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h_last")
    _dev(W_q, torch.bfloat16, "W_q", dense=False); _dev(K, torch.bfloat16, "K", dense=False); _dev(V, torch.bfloat16, "V", dense=False)
    _dev(mask, torch.int32, "mask"); _dev(budget, torch.int32, "budget"); _dev(b_step, torch.int32, "b_step")
    for t, name in ((kv_len, "kv_len"), (seq_len, "seq_len"), (token_pos, "token_pos")):
        if t is not None:                      # a missing kv_len or seq_len is the library's to refuse
            _dev(t, torch.int32, name)
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    _check(load().gvote_recompress(ctypes.byref(p), _ptr(mu), _ptr(var), _ptr(h_last), _ptr(W_q), W_q.stride(0),
                                   _ptr(b_q), _ptr(K), _ptr(V), K.stride(1), K.stride(0), _ptr(cu_seqlens),
                                   _ptr(kv_len), _ptr(seq_len), _ptr(token_pos), batch, total, max_N, _ptr(mask),
                                   _ptr(budget), _ptr(b_step), _ptr(ws), ws.numel(), _stream()), "gvote_recompress")


FIT_STATIC_MAX_ENTRIES = 131072


def gvote_fit_static(p, h, cu_seqlens, batch: int, max_N: int, mu, var) -> None:
    """`gvote_fit` for callers that cannot ask for device memory where they stand (an allocator
    callback, a serving loop with a frozen pool): no workspace argument, the partial sums go to
    a fixed array inside the library.  Needs batch * d_h <= FIT_STATIC_MAX_ENTRIES; calls that
    could overlap on the GPU must be serialised by the caller, they share that array."""
    _dev(h, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h", dense=False)
    _dev(cu_seqlens, torch.int32, "cu_seqlens"); _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var")
    _check(load().gvote_fit_static(ctypes.byref(p), _ptr(h), h.stride(0), _ptr(cu_seqlens), batch, max_N,
                                   _ptr(mu), _ptr(var), _stream()), "gvote_fit_static")


def gvote_sample(p, mu, var, batch, H_tilde, raw=None) -> None:
    _dev(mu, torch.float32, "mu"); _dev(var, torch.float32, "var"); _dev(H_tilde, torch.float32, "H_tilde")
    if raw is not None:
        _dev(raw, torch.int32, "raw")
    _check(load().gvote_sample(ctypes.byref(p), _ptr(mu), _ptr(var), batch, _ptr(H_tilde), _ptr(raw), _stream()),
           "gvote_sample")


def gvote_project(p, H_tilde, h_last, W_q, b_q, cu_seqlens, batch, Q, ws) -> None:
    _dev(H_tilde, torch.float32, "H_tilde"); _dev(W_q, torch.bfloat16, "W_q", dense=False); _dev(Q, torch.bfloat16, "Q")
    _dev(h_last, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h_last")
    _check(load().gvote_project(ctypes.byref(p), _ptr(H_tilde), _ptr(h_last), _ptr(W_q), W_q.stride(0), _ptr(b_q),
                                _ptr(cu_seqlens), batch, _ptr(Q), _ptr(ws), ws.numel(), _stream()), "gvote_project")


def gvote_vote(p, Q, K, cu_seqlens, geom, mask, budget, b_step, ws, dbg_probs=None) -> None:
    batch, total, max_N = geom
    _dev(Q, torch.bfloat16, "Q"); _dev(K, torch.bfloat16, "K", dense=False); _dev(mask, torch.int32, "mask")
    _dev(budget, torch.int32, "budget"); _dev(b_step, torch.int32, "b_step")
    _check(load().gvote_vote(ctypes.byref(p), _ptr(Q), _ptr(K), K.stride(1), K.stride(0), _ptr(cu_seqlens), batch,
                             total, max_N, _ptr(mask), _ptr(budget), _ptr(b_step), _ptr(dbg_probs), _ptr(ws),
                             ws.numel(), _stream()), "gvote_vote")


def gvote_select(p, H_tilde, h_last, W_q, b_q, K, cu_seqlens, geom, mask, budget, b_step, ws, dbg_probs=None) -> None:
    batch, total, max_N = geom
    _dev(H_tilde, torch.float32, "H_tilde"); _dev(W_q, torch.bfloat16, "W_q", dense=False); _dev(K, torch.bfloat16, "K", dense=False)
    _check(load().gvote_select(ctypes.byref(p), _ptr(H_tilde), _ptr(h_last), _ptr(W_q), W_q.stride(0), _ptr(b_q),
                               _ptr(K), K.stride(1), K.stride(0), _ptr(cu_seqlens), batch, total, max_N, _ptr(mask),
                               _ptr(budget), _ptr(b_step), _ptr(dbg_probs), _ptr(ws), ws.numel(), _stream()),
           "gvote_select")


def gvote_compact(p, K, V, mask, cu_seqlens, geom, budget, ws) -> None:
    batch, total, max_N = geom
    _dev(K, torch.bfloat16, "K", dense=False); _dev(V, torch.bfloat16, "V", dense=False); _dev(mask, torch.int32, "mask")
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    _check(load().gvote_compact(ctypes.byref(p), _ptr(K), _ptr(V), K.stride(1), K.stride(0), _ptr(mask),
                                _ptr(cu_seqlens), batch, total, max_N, _ptr(budget), _ptr(ws), ws.numel(), _stream()),
           "gvote_compact")


def gvote_overlap(p, Q, K, mask, cu_seqlens, geom, overlap, ws) -> None:
    """Share of each query head's current-query attention that falls on the kept keys (Section 3.3)."""
    batch, total, max_N = geom
    _dev(Q, torch.bfloat16, "Q"); _dev(K, torch.bfloat16, "K", dense=False); _dev(mask, torch.int32, "mask")
    _dev(overlap, torch.float32, "overlap")
    _check(load().gvote_overlap(ctypes.byref(p), _ptr(Q), _ptr(K), K.stride(1), K.stride(0), _ptr(mask),
                                _ptr(cu_seqlens), batch, total, max_N, _ptr(overlap), _ptr(ws), ws.numel(), _stream()),
           "gvote_overlap")


def gvote_pack(p, K, V, mask, cu_seqlens, geom, K_packed, V_packed, cu_seqlens_k, budget, ws) -> None:
    batch, total, max_N = geom
    _dev(K, torch.bfloat16, "K", dense=False); _dev(V, torch.bfloat16, "V", dense=False); _dev(mask, torch.int32, "mask")
    _dev(K_packed, torch.bfloat16, "K_packed"); _dev(V_packed, torch.bfloat16, "V_packed")
    _dev(cu_seqlens_k, torch.int32, "cu_seqlens_k"); _dev(budget, torch.int32, "budget")
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    if K_packed.shape != V_packed.shape or K_packed.dim() != 2 or K_packed.shape[1] != p.d_k:
        raise ValueError("K_packed and V_packed must be [rows, d_k]")
    _check(load().gvote_pack(ctypes.byref(p), _ptr(K), _ptr(V), K.stride(1), K.stride(0), _ptr(mask), _ptr(cu_seqlens),
                             batch, total, max_N, _ptr(K_packed), _ptr(V_packed), K_packed.shape[0],
                             _ptr(cu_seqlens_k), _ptr(budget), _ptr(ws), ws.numel(), _stream()), "gvote_pack")


def gvote_compress(p, h, W_q, b_q, K, V, cu_seqlens, geom, mask, budget, b_step, ws, h_last=None) -> None:
    batch, total, max_N = geom
    _dev(h, torch.float32 if p.h_dtype == DTYPE_F32 else torch.bfloat16, "h", dense=False)
    _dev(W_q, torch.bfloat16, "W_q", dense=False); _dev(K, torch.bfloat16, "K", dense=False); _dev(V, torch.bfloat16, "V", dense=False)
    _dev(mask, torch.int32, "mask"); _dev(budget, torch.int32, "budget"); _dev(b_step, torch.int32, "b_step")
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    _check(load().gvote_compress(ctypes.byref(p), _ptr(h), h.stride(0), _ptr(h_last), _ptr(W_q), W_q.stride(0),
                                 _ptr(b_q), _ptr(K), _ptr(V), K.stride(1), K.stride(0), _ptr(cu_seqlens), batch,
                                 total, max_N, _ptr(mask), _ptr(budget), _ptr(b_step), _ptr(ws), ws.numel(),
                                 _stream()), "gvote_compress")


def gvote_store8(p, K, V, cu_seqlens, geom, cache: Cache8, ws, mask=None, kv_len=None, acc=None, acc_out=None,
                 token_pos=None, token_pos_out=None) -> None:
    """The kept rows of the bf16 slabs K, V into the 8-bit cache; acc and token_pos move with them."""
    batch, total, max_N = geom
    H, dst, dev = p.n_kv_heads, (p.n_kv_heads, cache.geom[1]), K.device
    if K.stride() != V.stride():
        raise ValueError("K and V must share strides")
    _launch(load().gvote_store8, dev, p, _shaped(K, torch.bfloat16, (H, total, p.d_k), "K", dev, dense=False),
            _shaped(V, torch.bfloat16, (H, total, p.d_k), "V", dev, dense=False), K.stride(1), K.stride(0),
            _shaped(mask, torch.int32, (H, mask_row_words(total, batch)), "mask", dev),
            _shaped(cu_seqlens, torch.int32, (batch + 1,), "cu_seqlens", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), batch, total, max_N, _cache8(p, cache, "cache", dev),
            _shaped(acc, torch.float32, (H, total), "acc", dev), _shaped(acc_out, torch.float32, dst, "acc_out", dev),
            _shaped(token_pos, torch.int32, (H, total), "token_pos", dev),
            _shaped(token_pos_out, torch.int32, dst, "token_pos_out", dev), ws=ws)


def gvote_prune8(p, cache: Cache8, mask, out: Cache8, ws, acc=None, acc_out=None, token_pos=None,
                 token_pos_out=None) -> None:
    """The kept rows of one 8-bit cache into another (mask=None keeps all)."""
    batch, total, _ = cache.geom
    H, dst, dev = p.n_kv_heads, (p.n_kv_heads, out.geom[1]), cache.device
    _launch(load().gvote_prune8, dev, p, _cache8(p, cache, "cache", dev),
            _shaped(mask, torch.int32, (H, mask_row_words(total, batch)), "mask", dev), _cache8(p, out, "out", dev),
            _shaped(acc, torch.float32, (H, total), "acc", dev), _shaped(acc_out, torch.float32, dst, "acc_out", dev),
            _shaped(token_pos, torch.int32, (H, total), "token_pos", dev),
            _shaped(token_pos_out, torch.int32, dst, "token_pos_out", dev), ws=ws)


def gvote_append8(p, K_new, V_new, cu_new, max_new: int, cache: Cache8, kv_len_out, ws, acc=None, token_pos=None,
                  pos_new=None) -> None:
    """New tokens' rows [n_kv_heads, total_new, d_k] behind the rows the cache holds; kv_len_out may be cache.kv_len."""
    batch, total, _ = cache.geom
    H, total_new, dev = p.n_kv_heads, K_new.shape[1], cache.device
    if total_new and K_new.stride() != V_new.stride():
        raise ValueError("K_new and V_new must share strides")
    _launch(load().gvote_append8, dev, p,
            _shaped(K_new, torch.bfloat16, (H, total_new, p.d_k), "K_new", dev, dense=False),
            _shaped(V_new, torch.bfloat16, (H, total_new, p.d_k), "V_new", dev, dense=False), K_new.stride(1),
            K_new.stride(0), _shaped(cu_new, torch.int32, (batch + 1,), "cu_new", dev), total_new, max_new,
            _cache8(p, cache, "cache", dev), _shaped(kv_len_out, torch.int32, (batch, H), "kv_len_out", dev),
            _shaped(acc, torch.float32, (H, total), "acc", dev),
            _shaped(token_pos, torch.int32, (H, total), "token_pos", dev),
            _shaped(pos_new, torch.int32, (total_new,), "pos_new", dev), ws=ws)


def gvote_attend8(p, Q, cu_q, max_q: int, cache: Cache8, out, ws, lse=None, acc=None, acc_out=None) -> None:
    """Attention of Q [total_q, n_q_heads, d_k] (a request's tokens are the last rows of its cache) over the 8-bit
    cache into out; the softmax weights are added to acc_out when it is given."""
    batch, total, _ = cache.geom
    H, total_q, dev = p.n_kv_heads, Q.shape[0], cache.device
    shape = (total_q, p.n_q_heads, p.d_k)
    _launch(load().gvote_attend8, dev, p, _shaped(Q, torch.bfloat16, shape, "Q", dev, dense=False), Q.stride(0),
            Q.stride(1), _shaped(cu_q, torch.int32, (batch + 1,), "cu_q", dev), total_q, max_q,
            _cache8(p, cache, "cache", dev), _shaped(out, torch.bfloat16, shape, "out", dev, dense=False), out.stride(0),
            out.stride(1), _shaped(lse, torch.float32, (total_q, p.n_q_heads), "lse", dev),
            _shaped(acc, torch.float32, (H, total), "acc", dev), _shaped(acc_out, torch.float32, (H, total), "acc_out", dev),
            ws=ws)


def gvote_accumulate(p, Q, cu_q, max_q: int, K, cu_seqlens, geom, acc_out, ws, acc=None, lse=None, kv_len=None) -> None:
    """acc_out = acc (or 0) + the softmax weights the prompt's queries Q [total_q, n_q_heads, d_k] give to the keys."""
    batch, total, max_N = geom
    H, total_q, dev = p.n_kv_heads, Q.shape[0], K.device
    _launch(load().gvote_accumulate, dev, p,
            _shaped(Q, torch.bfloat16, (total_q, p.n_q_heads, p.d_k), "Q", dev, dense=False), Q.stride(0), Q.stride(1),
            _shaped(cu_q, torch.int32, (batch + 1,), "cu_q", dev), total_q, max_q,
            _shaped(K, torch.bfloat16, (H, total, p.d_k), "K", dev, dense=False), K.stride(1), K.stride(0),
            _shaped(cu_seqlens, torch.int32, (batch + 1,), "cu_seqlens", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), batch, total, max_N,
            _shaped(lse, torch.float32, (total_q, p.n_q_heads), "lse", dev),
            _shaped(acc, torch.float32, (H, total), "acc", dev), _shaped(acc_out, torch.float32, (H, total), "acc_out", dev),
            ws=ws)


def gvote_evict(p, acc, cu_seqlens, geom, keep, n_recent: int, mask, budget, ws, kv_len=None) -> None:
    """Keep-mask of the n_recent last rows, the p.n_s first and the rows of largest acc, keep [batch, n_kv_heads] in all."""
    batch, total, max_N = geom
    H, dev = p.n_kv_heads, acc.device
    _launch(load().gvote_evict, dev, p, _shaped(acc, torch.float32, (H, total), "acc", dev),
            _shaped(cu_seqlens, torch.int32, (batch + 1,), "cu_seqlens", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), batch, total, max_N,
            _shaped(keep, torch.int32, (batch, H), "keep", dev), n_recent,
            _shaped(mask, torch.int32, (H, mask_row_words(total, batch)), "mask", dev),
            _shaped(budget, torch.int32, (batch, H), "budget", dev), ws=ws)


def gvote_page_tables(p, pages: PageCache, ws, keep=None, cu_new=None, max_new: int = 0, slots=None, mask=None) -> None:
    """Cuts every head to keep [batch, n_kv_heads] rows, then grows it by the request's new tokens (packed by cu_new, at most
    max_new of one request), or by those that mask keeps; slots [n_kv_heads, total_new] says where each new row goes."""
    H, dev, batch = p.n_kv_heads, pages.device, pages.tables.shape[0]
    if cu_new is not None and slots is None:
        raise ValueError("cu_new needs slots")
    total_new = 0 if slots is None else slots.shape[1]
    _launch(load().gvote_page_tables, dev, p, _pages(p, pages, dev), _shaped(keep, torch.int32, (batch, H), "keep", dev),
            _shaped(cu_new, torch.int32, (batch + 1,), "cu_new", dev), total_new, max_new,
            _shaped(mask, torch.int32, (H, mask_row_words(total_new, batch)), "mask", dev),
            _shaped(slots, torch.int32, (H, total_new), "slots", dev), ws=ws)


def gvote_page_write(p, K_new, V_new, slots, pages: PageCache, ws) -> None:
    """Rows of K_new, V_new [n_kv_heads, total_new, d_k] to the places slots [n_kv_heads, total_new] names (negative: dropped).
    Slots that are not negative are to differ."""
    H, total_new, dev = p.n_kv_heads, K_new.shape[1], pages.device
    if total_new and not _same_strides(K_new, V_new):
        raise ValueError("K_new and V_new must share strides")
    _launch(load().gvote_page_write, dev, p, _shaped(K_new, torch.bfloat16, (H, total_new, p.d_k), "K_new", dev, dense=False),
            _shaped(V_new, torch.bfloat16, (H, total_new, p.d_k), "V_new", dev, dense=False), K_new.stride(1), K_new.stride(0),
            _shaped(slots, torch.int32, (H, total_new), "slots", dev), total_new, _pages(p, pages, dev), ws=ws)


def gvote_page_attend(p, Q, cu_q, max_q: int, pages: PageCache, out, ws, lse=None) -> None:
    """Attention of Q [total_q, n_q_heads, d_k] (a request's tokens are the last rows of its cache) over the pages into out."""
    total_q, dev = Q.shape[0], pages.device
    shape = (total_q, p.n_q_heads, p.d_k)
    _launch(load().gvote_page_attend, dev, p, _shaped(Q, torch.bfloat16, shape, "Q", dev, dense=False), Q.stride(0), Q.stride(1),
            _shaped(cu_q, torch.int32, (pages.tables.shape[0] + 1,), "cu_q", dev), total_q, max_q, _pages(p, pages, dev),
            _shaped(out, torch.bfloat16, shape, "out", dev, dense=False), out.stride(0), out.stride(1),
            _shaped(lse, torch.float32, (total_q, p.n_q_heads), "lse", dev), ws=ws)


def gvote_attend(p, Q, cu_q, max_q: int, K, V, cu_seqlens, geom, out, ws, lse=None, kv_len=None) -> None:
    """Attention of Q [total_q, n_q_heads, d_k] (a request's tokens are the last of its rows) over the bf16 slabs K, V: a
    prompt's causal attention, or tokens over a cache compacted in place (kv_len)."""
    batch, total, max_N = geom
    H, total_q, dev = p.n_kv_heads, Q.shape[0], K.device
    shape = (total_q, p.n_q_heads, p.d_k)
    if total and not _same_strides(K, V):
        raise ValueError("K and V must share strides")
    _launch(load().gvote_attend, dev, p, _shaped(Q, torch.bfloat16, shape, "Q", dev, dense=False), Q.stride(0), Q.stride(1),
            _shaped(cu_q, torch.int32, (batch + 1,), "cu_q", dev), total_q, max_q,
            _shaped(K, torch.bfloat16, (H, total, p.d_k), "K", dev, dense=False),
            _shaped(V, torch.bfloat16, (H, total, p.d_k), "V", dev, dense=False), K.stride(1), K.stride(0),
            _shaped(cu_seqlens, torch.int32, (batch + 1,), "cu_seqlens", dev),
            _shaped(kv_len, torch.int32, (batch, H), "kv_len", dev), batch, total, max_N,
            _shaped(out, torch.bfloat16, shape, "out", dev, dense=False), out.stride(0), out.stride(1),
            _shaped(lse, torch.float32, (total_q, p.n_q_heads), "lse", dev), ws=ws)


def gvote_compress_host(p, h, W_q, b_q, K, V, cu_seqlens, mask, budget, b_step) -> None:
    """Host-memory variant: every tensor is a CPU tensor (pinned for full copy speed); K and V are
    compacted in place in host memory; returns after the device work has completed."""
    for name, t in (("h", h), ("W_q", W_q), ("K", K), ("V", V), ("cu_seqlens", cu_seqlens), ("mask", mask),
                    ("budget", budget), ("b_step", b_step)):
        if t.is_cuda or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous CPU tensor")
    batch = cu_seqlens.numel() - 1
    _check(load().gvote_compress_host(ctypes.byref(p), _ptr(h), _ptr(W_q), _ptr(b_q), _ptr(K), _ptr(V),
                                      _ptr(cu_seqlens), batch, _ptr(mask), _ptr(budget), _ptr(b_step)),
           "gvote_compress_host")


def gvote_host_arena_release() -> None:
    load().gvote_host_arena_release()


def gvote_poll_status(ws) -> int:
    return int(load().gvote_poll_status(_ptr(ws), _stream()))


def gvote_clear_status(ws) -> None:
    _check(load().gvote_clear_status(_ptr(ws), _stream()), "gvote_clear_status")


def gvote_exact_heads(ws) -> int:
    """(request, KV head) pairs the default mode had to select again by the exact route since the
    status block was last cleared."""
    return int(load().gvote_exact_heads(_ptr(ws), _stream()))


def gvote_profile_enable(on: bool) -> None:
    load().gvote_profile_enable(1 if on else 0)


def gvote_profile_report() -> dict:
    """{kernel name: (launches, total milliseconds)} since profiling was enabled."""
    lib = load()
    cap = 1 << 16
    buf = ctypes.create_string_buffer(cap)
    lib.gvote_profile_report(buf, cap)
    out = {}
    for line in buf.value.decode().splitlines():
        name, n, ms = line.split()
        out[name] = (int(n), float(ms))
    return out


def gvote_launch_count() -> int:
    return int(load().gvote_launch_count())


def gvote_status_string(status: int) -> str:
    return load().gvote_status_string(status).decode()


# ----------------------------------------------------------------------------- tensor plumbing
def bf16_from_bits(bits: np.ndarray, device="cuda", pin: bool = False) -> torch.Tensor:
    """uint16 bit patterns -> torch.bfloat16 tensor (no value change)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    if device == "cpu":
        return t.pin_memory() if pin else t
    return t.to(device)


def bits_from_bf16(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def unpack_mask(mask_row: np.ndarray, word_offset: int, N: int) -> np.ndarray:
    """Bits of one request in one head's mask row -> bool [N]."""
    words = np.ascontiguousarray(mask_row[word_offset:word_offset + (N + 31) // 32]).view(np.uint32)
    bits = np.unpackbits(words.view(np.uint8), bitorder="little")
    return bits[:N].astype(bool)
