"""Python entry points of the C-ABI library, same names as in ``include/ht.h``.

Argument marshalling only: tensors are torch CUDA tensors whose ``data_ptr()`` goes
straight to the library, outputs are allocated with torch, work is enqueued on torch's
current stream.  Every step of the path runs in the library's kernels; there is no
fallback, and a missing ``libht.so`` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libht.so")

HT_F32, HT_F16, HT_BF16 = 0, 1, 2
HT_OK = 0
HT_ERR_INVALID_ARG, HT_ERR_UNSUPPORTED, HT_ERR_BAD_TREE, HT_ERR_WORKSPACE, HT_ERR_CUDA, HT_ERR_TIMEOUT = range(1, 7)
HT_STATUS_OK, HT_STATUS_BAD_TREE, HT_STATUS_BAD_LEN, HT_STATUS_BAD_PATH, HT_STATUS_PATH_TOO_LONG = range(5)
HT_ATTN_FORCE_SIMT = 1
HT_ATTN_WORKSPACE_CLEAN = 2
HT_ATTN_CONTEXT_FINAL = 4
HT_ATTN_TEST_SHORT_WAITS = 0x80000000
HT_STATUS_BAD_PAGE, HT_STATUS_TIMEOUT, HT_STATUS_BAD_PARAM = 5, 6, 7
HT_HEAD_NORM_Q, HT_HEAD_NORM_K = 1, 2
HT_ROPE_PLAIN, HT_ROPE_LINEAR, HT_ROPE_BY_PARTS = range(3)

EXPORTS = ("ht_version", "ht_last_error_string", "ht_transfer", "ht_tree_attention_workspace",
           "ht_tree_attention", "ht_verify_greedy", "ht_kv_compact", "ht_draft_tree", "ht_rope_kv_append", "ht_tree_attention_static",
           "ht_tree_attention_paged", "ht_rope_kv_append_paged", "ht_kv_compact_paged", "ht_tree_attention_launches",
           "ht_verify_greedy_compact", "ht_norm_rope_kv_append", "ht_norm_rope_kv_append_paged", "ht_sample", "ht_verify_sampled",
           "ht_tree_attention_scored", "ht_tree_attention_scored_paged", "ht_norm_rope_kv_append_q8", "ht_norm_rope_kv_append_q8_paged",
           "ht_tree_attention_q8_workspace", "ht_tree_attention_q8", "ht_tree_attention_q8_paged", "ht_kv_compact_q8", "ht_kv_compact_q8_paged",
           "ht_shape_logits", "ht_count_tokens")
HT_STATIC_SCRATCH_BYTES = 16 << 20

class _Dtypes(dict):
    def __missing__(self, dtype):
        raise ValueError("%s is not supported: float32, float16 or bfloat16" % (dtype,))


_DTYPES = _Dtypes({torch.float32: HT_F32, torch.float16: HT_F16, torch.bfloat16: HT_BF16})


class AttnDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("cap", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64),
                ("num_splits", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class PagedDesc(ctypes.Structure):
    _fields_ = [("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("B", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("cap", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("N", ctypes.c_int32), ("stride_layer", ctypes.c_int64),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class ScoreDesc(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("pos", ctypes.c_void_p)]


class HeadDesc(ctypes.Structure):
    _fields_ = [("norm", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float),
                ("rope_base", ctypes.c_float), ("factor", ctypes.c_float), ("low", ctypes.c_float), ("high", ctypes.c_float),
                ("orig_len", ctypes.c_float), ("magnitude", ctypes.c_float), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class Q8Scales(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("stride_layer", ctypes.c_int64), ("stride_b", ctypes.c_int64),
                ("stride_h", ctypes.c_int64)]


class WindowDesc(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


class HtError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("libht error %d: %s" % (code, message))
        self.code = code


_lib = None


def load() -> ctypes.CDLL:
    """Load ``libht.so`` (built in-tree by ``paper_2404_12022_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libht.so is missing at %s: build it with `python -m paper_2404_12022_b200.build`; "
                "there is no fallback path" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        lib.ht_version.restype = i32
        lib.ht_last_error_string.restype = ctypes.c_char_p
        lib.ht_transfer.restype = i32
        lib.ht_transfer.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp]
        lib.ht_tree_attention_workspace.restype = sz
        lib.ht_tree_attention_workspace.argtypes = [ctypes.POINTER(AttnDesc)]
        lib.ht_tree_attention_launches.restype = i32
        lib.ht_tree_attention_launches.argtypes = [ctypes.POINTER(AttnDesc)]
        lib.ht_tree_attention.restype = i32
        lib.ht_tree_attention.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
        lib.ht_tree_attention_static.restype = i32
        lib.ht_tree_attention_static.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, vp, vp, vp, vp, vp]
        lib.ht_tree_attention_paged.restype = i32
        lib.ht_tree_attention_paged.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(PagedDesc), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
        lib.ht_rope_kv_append_paged.restype = i32
        lib.ht_rope_kv_append_paged.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(PagedDesc), vp, vp, vp, vp, vp, vp,
                                                ctypes.c_float, vp, vp, vp, vp, vp]
        lib.ht_kv_compact_paged.restype = i32
        lib.ht_kv_compact_paged.argtypes = [vp, vp, ctypes.POINTER(CacheDesc), ctypes.POINTER(PagedDesc), vp, vp, vp, vp, i32,
                                            vp, vp, vp]
        lib.ht_verify_greedy.restype = i32
        lib.ht_verify_greedy.argtypes = [vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        lib.ht_verify_greedy_compact.restype = i32
        lib.ht_verify_greedy_compact.argtypes = [vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                                 vp, vp, ctypes.POINTER(CacheDesc), vp, vp, vp, vp]
        lib.ht_kv_compact.restype = i32
        lib.ht_kv_compact.argtypes = [vp, vp, ctypes.POINTER(CacheDesc), vp, vp, vp, i32, vp, vp, vp]
        lib.ht_draft_tree.restype = i32
        lib.ht_draft_tree.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.ht_rope_kv_append.restype = i32
        lib.ht_rope_kv_append.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
        lib.ht_tree_attention_scored.restype = i32
        lib.ht_tree_attention_scored.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(ScoreDesc), *lib.ht_tree_attention.argtypes[1:]]
        lib.ht_tree_attention_scored_paged.restype = i32
        lib.ht_tree_attention_scored_paged.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(PagedDesc), ctypes.POINTER(ScoreDesc),
                                                       *lib.ht_tree_attention_paged.argtypes[2:]]
        place = [vp] * 10
        lib.ht_norm_rope_kv_append.restype = i32
        lib.ht_norm_rope_kv_append.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(HeadDesc), *place, vp, vp]
        lib.ht_norm_rope_kv_append_paged.restype = i32
        lib.ht_norm_rope_kv_append_paged.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(HeadDesc), ctypes.POINTER(PagedDesc),
                                                     *place, vp, vp, vp]
        lib.ht_sample.restype = i32
        lib.ht_sample.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.ht_verify_sampled.restype = i32
        lib.ht_verify_sampled.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        attn, head, paged, scales, cache = (ctypes.POINTER(t) for t in (AttnDesc, HeadDesc, PagedDesc, Q8Scales, CacheDesc))
        window = ctypes.POINTER(WindowDesc)
        lib.ht_norm_rope_kv_append_q8.restype = i32
        lib.ht_norm_rope_kv_append_q8.argtypes = [attn, head, scales, *place, vp, vp]
        lib.ht_norm_rope_kv_append_q8_paged.restype = i32
        lib.ht_norm_rope_kv_append_q8_paged.argtypes = [attn, head, paged, scales, *place, vp, vp, vp]
        lib.ht_tree_attention_q8_workspace.restype = sz
        lib.ht_tree_attention_q8_workspace.argtypes = [attn]
        lib.ht_tree_attention_q8.restype = i32
        lib.ht_tree_attention_q8.argtypes = [attn, window, scales, *lib.ht_tree_attention.argtypes[1:]]
        lib.ht_tree_attention_q8_paged.restype = i32
        lib.ht_tree_attention_q8_paged.argtypes = [attn, paged, window, scales, *lib.ht_tree_attention_paged.argtypes[2:]]
        lib.ht_kv_compact_q8.restype = i32
        lib.ht_kv_compact_q8.argtypes = [vp, vp, scales, cache, vp, vp, vp, i32, vp, vp, vp]
        lib.ht_kv_compact_q8_paged.restype = i32
        lib.ht_kv_compact_q8_paged.argtypes = [vp, vp, scales, cache, paged, vp, vp, vp, vp, i32, vp, vp, vp]
        lib.ht_shape_logits.restype = i32
        lib.ht_shape_logits.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
        lib.ht_count_tokens.restype = i32
        lib.ht_count_tokens.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != HT_OK:
        raise HtError(rc, load().ht_last_error_string().decode())


try:                                       # the same number without the stream object around it (3 us of a call's 20)
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    _raw_stream = None


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, dtype=None, name="tensor"):
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (this library has no CPU path)" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s" % (name, dtype))


def transfer(h_src: torch.Tensor, W: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """h_src [B, d], W [k, d, d] -> out [B, k, d] (same dtype)."""
    _need(h_src, name="h_src")
    _need(W, h_src.dtype, "W")
    B, d = h_src.shape
    k = W.shape[0]
    if tuple(W.shape) != (k, d, d):
        raise ValueError("W must be [k, d, d]")
    if out is None:
        out = torch.empty((B, k, d), dtype=h_src.dtype, device=h_src.device)
    _need(out, h_src.dtype, "out")
    _check(load().ht_transfer(_ptr(h_src), _ptr(W), _ptr(out), B, k, d, _DTYPES[h_src.dtype], _stream()))
    return out


def make_attn_desc(q: torch.Tensor, k_cache: torch.Tensor, scale: float = 0.0, num_splits: int = 0,
                   flags: int = 0) -> AttnDesc:
    B, N, Hq, D = q.shape
    Bc, Hkv, cap, Dc = k_cache.shape
    if (Bc, Dc) != (B, D):
        raise ValueError("cache shape does not match q")
    if k_cache.stride(3) != 1 or k_cache.stride(2) != D:
        raise ValueError("cache rows must be contiguous and D apart")
    return AttnDesc(B, N, Hq, Hkv, D, cap, _DTYPES[q.dtype], float(scale), k_cache.stride(0),
                    k_cache.stride(1), num_splits, flags)


def tree_attention_launches(desc: AttnDesc) -> int:
    """Kernels of this library that one ``tree_attention`` call with this descriptor enqueues."""
    return int(load().ht_tree_attention_launches(ctypes.byref(desc)))


def tree_attention_workspace(desc: AttnDesc) -> int:
    return int(load().ht_tree_attention_workspace(ctypes.byref(desc)))


def tree_attention(q, k_cache, v_cache, kv_len, parent, out=None, workspace=None, status=None,
                   scale: float = 0.0, num_splits: int = 0, flags: int = 0):
    """q [B, N, Hq, D]; caches [B, Hkv, cap, D] (may be strided views over b / head);
    kv_len [B] int32; parent [B, N] int32.  Returns (out, status)."""
    _need(q, name="q")
    _need(kv_len, torch.int32, "kv_len")
    _need(parent, torch.int32, "parent")
    if not (k_cache.is_cuda and v_cache.is_cuda) or k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise ValueError("caches must be CUDA tensors of q's dtype")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must share shape and strides")
    desc = make_attn_desc(q, k_cache, scale, num_splits, flags)
    B, N = desc.B, desc.N
    if tuple(parent.shape) != (B, N) or tuple(kv_len.shape) != (B,):
        raise ValueError("parent must be [B, N] and kv_len [B]")
    if out is None:
        out = torch.empty_like(q)
    _need(out, q.dtype, "out")
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=q.device)
    need = tree_attention_workspace(desc)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().ht_tree_attention(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                    _ptr(parent), _ptr(out), _ptr(workspace), ws_bytes, _ptr(status), _stream()))
    return out, status


def tree_attention_paged(q, k_pages, v_pages, block_table, kv_len, parent, out=None, workspace=None, status=None,
                         scale: float = 0.0, flags: int = 0):
    """q [B, N, Hq, D]; page pools [n_pages, Hkv, page_size, D] (may be strided over page / head);
    block_table [B, max_pages] int32; kv_len [B] int32; parent [B, N] int32.  Returns (out, status)."""
    _need(q, name="q")
    _need(block_table, torch.int32, "block_table")
    _need(kv_len, torch.int32, "kv_len")
    _need(parent, torch.int32, "parent")
    if not (k_pages.is_cuda and v_pages.is_cuda) or k_pages.dtype != q.dtype or v_pages.dtype != q.dtype:
        raise ValueError("page pools must be CUDA tensors of q's dtype")
    if k_pages.stride() != v_pages.stride() or k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages must share shape and strides")
    B, N, Hq, D = q.shape
    n_pages, Hkv, page_size, Dp = k_pages.shape
    if Dp != D or k_pages.stride(3) != 1 or k_pages.stride(2) != D:
        raise ValueError("page rows must be contiguous and D apart")
    if block_table.dim() != 2 or block_table.shape[0] != B or tuple(parent.shape) != (B, N) or tuple(kv_len.shape) != (B,):
        raise ValueError("block_table must be [B, max_pages], parent [B, N], kv_len [B]")
    max_pages = block_table.shape[1]
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q.dtype], scale, 0, 0, 0, flags)
    pages = PagedDesc(page_size, max_pages, n_pages, k_pages.stride(0), k_pages.stride(1))
    if out is None:
        out = torch.empty_like(q)
    _need(out, q.dtype, "out")
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=q.device)
    need = tree_attention_workspace(desc)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().ht_tree_attention_paged(ctypes.byref(desc), ctypes.byref(pages), _ptr(q), _ptr(k_pages), _ptr(v_pages),
                                          _ptr(block_table), _ptr(kv_len), _ptr(parent), _ptr(out), _ptr(workspace),
                                          ws_bytes, _ptr(status), _stream()))
    return out, status


def tree_attention_static(q, k_cache, v_cache, kv_len, parent, out=None, status=None, scale: float = 0.0,
                          num_splits: int = 0):
    """Tree attention for callers that cannot allocate scratch: same results as
    ``tree_attention``, with the split partials in the library's built-in array (at most
    ``HT_STATIC_SCRATCH_BYTES``; larger problems raise).  Calls must not overlap on the GPU.
    ``out`` and ``status`` may be passed in so that the call itself allocates nothing."""
    _need(q, name="q")
    _need(kv_len, torch.int32, "kv_len")
    _need(parent, torch.int32, "parent")
    desc = make_attn_desc(q, k_cache, scale, num_splits, 0)
    if out is None:
        out = torch.empty_like(q)
    if status is None:
        status = torch.empty(desc.B, dtype=torch.int32, device=q.device)
    _check(load().ht_tree_attention_static(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_len),
                                           _ptr(parent), _ptr(out), _ptr(status), _stream()))
    return out, status


def verify_greedy(logits, tokens, parent, root_pred=None, max_path: int = 8, accept_len=None):
    """logits [B, N, V]; tokens [B, T] int32; parent [B, N] int32; root_pred [B] int32 or None.
    ``accept_len`` [B] int32, if given, must hold zeros or what an earlier call left in it (the kernel counts
    arrivals in its upper bits); by default a zeroed tensor is made.
    Returns (pred [B, N], accept_len [B], accept_path [B, max_path], next_token [B], status [B])."""
    _need(logits, name="logits")
    _need(tokens, torch.int32, "tokens")
    _need(parent, torch.int32, "parent")
    B, N, V = logits.shape
    T = tokens.shape[1]
    if tuple(parent.shape) != (B, N) or tokens.shape[0] != B:
        raise ValueError("parent must be [B, N] and tokens [B, T]")
    if root_pred is not None:
        _need(root_pred, torch.int32, "root_pred")
    dev = logits.device
    pred = torch.empty((B, N), dtype=torch.int32, device=dev)
    if accept_len is None:
        accept_len = torch.zeros(B, dtype=torch.int32, device=dev)
    else:
        _need(accept_len, torch.int32, "accept_len")
    accept_path = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    next_token = torch.empty(B, dtype=torch.int32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    _check(load().ht_verify_greedy(_ptr(logits), _DTYPES[logits.dtype], _ptr(tokens), _ptr(parent),
                                   _ptr(root_pred), B, N, T, V, max_path, _ptr(pred), _ptr(accept_len),
                                   _ptr(accept_path), _ptr(next_token), _ptr(status), _stream()))
    return pred, accept_len, accept_path, next_token, status


def verify_greedy_compact(logits, tokens, parent, root_pred, k_cache, v_cache, kv_len, max_path: int = 8, rows: int = 0,
                          accept_len=None):
    """Verification and compaction in one launch: ``verify_greedy`` followed by ``kv_compact`` on caches
    [layers, B, Hkv, cap, D].  ``rows``: logits rows per sequence whose argmax is taken (0 = the T tree rows).
    Returns (pred, accept_len, accept_path, next_token, status, new_kv_len, compact_status)."""
    _need(logits, name="logits")
    _need(tokens, torch.int32, "tokens")
    _need(parent, torch.int32, "parent")
    _need(kv_len, torch.int32, "kv_len")
    B, N, V = logits.shape
    T = tokens.shape[1]
    if tuple(parent.shape) != (B, N) or tokens.shape[0] != B:
        raise ValueError("parent must be [B, N] and tokens [B, T]")
    if root_pred is not None:
        _need(root_pred, torch.int32, "root_pred")
    if not (k_cache.is_cuda and v_cache.is_cuda) or k_cache.dtype != v_cache.dtype:
        raise ValueError("caches must be CUDA tensors of one dtype")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must share shape and strides")
    layers, Bc, Hkv, cap, D = k_cache.shape
    if k_cache.stride(4) != 1 or k_cache.stride(3) != D or Bc != B:
        raise ValueError("cache rows must be contiguous and D apart, and the caches must hold B sequences")
    desc = CacheDesc(layers, B, Hkv, cap, D, _DTYPES[k_cache.dtype], N, k_cache.stride(0), k_cache.stride(1), k_cache.stride(2))
    dev = logits.device
    pred = torch.full((B, N), -1, dtype=torch.int32, device=dev)
    if accept_len is None:
        accept_len = torch.zeros(B, dtype=torch.int32, device=dev)
    else:
        _need(accept_len, torch.int32, "accept_len")
    accept_path = torch.empty((B, max_path), dtype=torch.int32, device=dev)
    next_token = torch.empty(B, dtype=torch.int32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    new_kv_len = torch.empty(B, dtype=torch.int32, device=dev)
    compact_status = torch.empty(B, dtype=torch.int32, device=dev)
    _check(load().ht_verify_greedy_compact(_ptr(logits), _DTYPES[logits.dtype], _ptr(tokens), _ptr(parent), _ptr(root_pred),
                                           B, N, T, V, max_path, rows, _ptr(pred), _ptr(accept_len), _ptr(accept_path),
                                           _ptr(next_token), _ptr(status), _ptr(k_cache), _ptr(v_cache), ctypes.byref(desc),
                                           _ptr(kv_len), _ptr(new_kv_len), _ptr(compact_status), _stream()))
    return pred, accept_len, accept_path, next_token, status, new_kv_len, compact_status


def kv_compact(k_cache, v_cache, n_rows: int, kv_len, accept_len, accept_path, new_kv_len=None,
               status=None):
    """In-place compaction of caches [layers, B, Hkv, cap, D].  Returns (new_kv_len, status)."""
    if not (k_cache.is_cuda and v_cache.is_cuda) or k_cache.dtype != v_cache.dtype:
        raise ValueError("caches must be CUDA tensors of one dtype")
    if k_cache.stride() != v_cache.stride() or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must share shape and strides")
    layers, B, Hkv, cap, D = k_cache.shape
    if k_cache.stride(4) != 1 or k_cache.stride(3) != D:
        raise ValueError("cache rows must be contiguous and D apart")
    _need(kv_len, torch.int32, "kv_len")
    _need(accept_len, torch.int32, "accept_len")
    _need(accept_path, torch.int32, "accept_path")
    max_path = accept_path.shape[1]
    desc = CacheDesc(layers, B, Hkv, cap, D, _DTYPES[k_cache.dtype], int(n_rows), k_cache.stride(0),
                     k_cache.stride(1), k_cache.stride(2))
    dev = k_cache.device
    if new_kv_len is None:
        new_kv_len = torch.empty(B, dtype=torch.int32, device=dev)
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=dev)
    _check(load().ht_kv_compact(_ptr(k_cache), _ptr(v_cache), ctypes.byref(desc), _ptr(kv_len),
                                _ptr(accept_len), _ptr(accept_path), max_path, _ptr(new_kv_len),
                                _ptr(status), _stream()))
    return new_kv_len, status


def draft_tree(logits, first_row: int, P: int, K: int, tmpl_parent, tmpl_rank, root_token, base_pos):
    """logits [B, rows, V]; pseudo position i (1..P) is row first_row + i - 1; tmpl_parent, tmpl_rank
    [T] int32; root_token [B] int32 or None; base_pos [B] int32.
    Returns (topk [B, P, K], tokens [B, T], pos [B, T], status [B])."""
    _need(logits, name="logits")
    _need(tmpl_parent, torch.int32, "tmpl_parent")
    _need(tmpl_rank, torch.int32, "tmpl_rank")
    _need(base_pos, torch.int32, "base_pos")
    if root_token is not None:
        _need(root_token, torch.int32, "root_token")
    B, rows, V = logits.shape
    T = tmpl_parent.shape[0]
    dev = logits.device
    topk = torch.empty((B, P, K), dtype=torch.int32, device=dev)
    tokens = torch.empty((B, T), dtype=torch.int32, device=dev)
    pos = torch.empty((B, T), dtype=torch.int32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    _check(load().ht_draft_tree(_ptr(logits), _DTYPES[logits.dtype], B, rows, V, first_row, P, K, _ptr(tmpl_parent),
                                _ptr(tmpl_rank), T, _ptr(root_token), _ptr(base_pos), _ptr(topk), _ptr(tokens),
                                _ptr(pos), _ptr(status), _stream()))
    return topk, tokens, pos, status


def rope_kv_append(q_in, k_in, v_in, pos, kv_len, k_cache, v_cache, rope_base: float = 10000.0, q_out=None):
    """q_in [B, N, Hq, D]; k_in, v_in [B, N, Hkv, D]; pos [B, N] int32; kv_len [B] int32; caches
    [B, Hkv, cap, D] (written in place at rows kv_len[b] + r).  Returns (q_out, status)."""
    _need(q_in, name="q_in")
    _need(k_in, q_in.dtype, "k_in")
    _need(v_in, q_in.dtype, "v_in")
    _need(pos, torch.int32, "pos")
    _need(kv_len, torch.int32, "kv_len")
    desc = make_attn_desc(q_in, k_cache)
    if q_out is None:
        q_out = torch.empty_like(q_in)
    status = torch.empty(desc.B, dtype=torch.int32, device=q_in.device)
    _check(load().ht_rope_kv_append(ctypes.byref(desc), _ptr(q_in), _ptr(k_in), _ptr(v_in), _ptr(pos), _ptr(kv_len),
                                    float(rope_base), _ptr(q_out), _ptr(k_cache), _ptr(v_cache), _ptr(status), _stream()))
    return q_out, status


def rope_kv_append_paged(q_in, k_in, v_in, pos, kv_len, block_table, k_pages, v_pages, rope_base: float = 10000.0,
                         q_out=None):
    """As ``rope_kv_append`` with the caches as page pools [n_pages, Hkv, page_size, D] (written in place at the
    logical rows kv_len[b] + r through block_table [B, max_pages]).  Returns (q_out, status)."""
    _need(q_in, name="q_in")
    _need(k_in, q_in.dtype, "k_in")
    _need(v_in, q_in.dtype, "v_in")
    _need(pos, torch.int32, "pos")
    _need(kv_len, torch.int32, "kv_len")
    _need(block_table, torch.int32, "block_table")
    B, N, Hq, D = q_in.shape
    n_pages, Hkv, page_size, Dp = k_pages.shape
    if Dp != D or k_pages.stride(3) != 1 or k_pages.stride(2) != D or k_pages.stride() != v_pages.stride():
        raise ValueError("page rows must be contiguous and D apart, K and V pools alike")
    max_pages = block_table.shape[1]
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q_in.dtype], 0.0, 0, 0, 0, 0)
    pages = PagedDesc(page_size, max_pages, n_pages, k_pages.stride(0), k_pages.stride(1))
    if q_out is None:
        q_out = torch.empty_like(q_in)
    status = torch.empty(B, dtype=torch.int32, device=q_in.device)
    _check(load().ht_rope_kv_append_paged(ctypes.byref(desc), ctypes.byref(pages), _ptr(q_in), _ptr(k_in), _ptr(v_in),
                                          _ptr(pos), _ptr(kv_len), _ptr(block_table), float(rope_base), _ptr(q_out),
                                          _ptr(k_pages), _ptr(v_pages), _ptr(status), _stream()))
    return q_out, status


def kv_compact_paged(k_pages, v_pages, block_table, n_rows: int, kv_len, accept_len, accept_path, new_kv_len=None,
                     status=None):
    """In-place compaction of page pools [layers, n_pages, Hkv, page_size, D] that share block_table
    [B, max_pages].  Returns (new_kv_len, status)."""
    if not (k_pages.is_cuda and v_pages.is_cuda) or k_pages.dtype != v_pages.dtype:
        raise ValueError("pools must be CUDA tensors of one dtype")
    if k_pages.stride() != v_pages.stride() or k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages must share shape and strides")
    layers, n_pages, Hkv, page_size, D = k_pages.shape
    if k_pages.stride(4) != 1 or k_pages.stride(3) != D:
        raise ValueError("page rows must be contiguous and D apart")
    _need(block_table, torch.int32, "block_table")
    _need(kv_len, torch.int32, "kv_len")
    _need(accept_len, torch.int32, "accept_len")
    _need(accept_path, torch.int32, "accept_path")
    B, max_pages = block_table.shape
    max_path = accept_path.shape[1]
    desc = CacheDesc(layers, B, Hkv, max_pages * page_size, D, _DTYPES[k_pages.dtype], int(n_rows), k_pages.stride(0), 0, 0)
    pages = PagedDesc(page_size, max_pages, n_pages, k_pages.stride(1), k_pages.stride(2))
    dev = k_pages.device
    if new_kv_len is None:
        new_kv_len = torch.empty(B, dtype=torch.int32, device=dev)
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=dev)
    _check(load().ht_kv_compact_paged(_ptr(k_pages), _ptr(v_pages), ctypes.byref(desc), ctypes.byref(pages),
                                      _ptr(block_table), _ptr(kv_len), _ptr(accept_len), _ptr(accept_path), max_path,
                                      _ptr(new_kv_len), _ptr(status), _stream()))
    return new_kv_len, status


def make_head_desc(D: int, norm: int = HT_HEAD_NORM_Q | HT_HEAD_NORM_K, eps: float = 1e-6, weight_offset: float = 0.0,
                   rot_dim: Optional[int] = None, interleaved: bool = False, rope_base: float = 10000.0,
                   scaling: int = HT_ROPE_PLAIN, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                   orig_len: float = 0.0, magnitude: float = 1.0) -> HeadDesc:
    """What ``norm_rope_kv_append`` does to each head of ``D`` features (``rot_dim`` None: all of them are rotated).
    The calls fill in the row strides of their tensors."""
    return HeadDesc(norm, D if rot_dim is None else rot_dim, int(interleaved), scaling, eps, weight_offset, rope_base, factor, low,
                    high, orig_len, magnitude, 0, 0, 0)


def _device_of(t: torch.Tensor, name: str) -> int:
    """The index of t's device, which must be the current one: the work goes to its current stream."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("%s must be a CUDA tensor (this library has no CPU path)" % name)
    if dev != torch.cuda.current_device():
        raise ValueError("%s lives on device %d, which is not the current one" % (name, dev))
    return dev


def _dense(t: torch.Tensor, dev: int, dtype, shape, name: str):
    """t must be a contiguous tensor of this device, dtype and shape."""
    if t.get_device() != dev or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor of device %d, %s, shape %s; it is %s on %s, shape %s%s" % (
            name, dev, dtype, tuple(shape), t.dtype, t.device, tuple(t.shape), "" if t.is_contiguous() else ", strided"))


def _rows(t: torch.Tensor, dev: int, dtype, B: int, N: int, D: int, name: str):
    """(heads, elements between rows) of t [B, N, H, D], whose heads must be dense and whose rows evenly spaced."""
    shape, (sb, sn, sh, sd) = t.shape, t.stride() if t.dim() == 4 else (0, 0, 0, 0)
    if t.get_device() != dev or t.dtype != dtype or len(shape) != 4 or shape[0] != B or shape[1] != N or shape[3] != D:
        raise ValueError("%s must be a CUDA tensor of device %d, %s, shape [%d, %d, heads, %d]" % (name, dev, dtype, B, N, D))
    H = shape[2]
    if sd != 1 or (sh != D and H > 1) or (B > 1 and N > 1 and sb != N * sn):
        raise ValueError("%s: heads must be contiguous and D apart, rows evenly spaced over [B, N]" % name)
    row = sn if N > 1 else (sb if B > 1 else H * D)
    if row < H * D:                                      # (a broadcast tensor's 0 would read as "dense")
        raise ValueError("%s: rows must not overlap; they are %d elements apart" % (name, row))
    return H, row


def _pair(k: torch.Tensor, v: torch.Tensor, dev: int, dtype, name: str):
    """Shape and strides of a K and a V cache, which must agree."""
    shape, strides = k.shape, k.stride()
    if k.get_device() != dev or v.get_device() != dev or k.dtype != dtype or v.dtype != dtype:
        raise ValueError("%s must be CUDA tensors of device %d, %s" % (name, dev, dtype))
    if v.shape != shape or v.stride() != strides or len(shape) != 4:
        raise ValueError("%s must share a 4-dimensional shape and strides" % name)
    if strides[3] != 1 or strides[2] != shape[3]:
        raise ValueError("%s: rows must be contiguous and D apart" % name)
    if (strides[0] == 0 and shape[0] > 1) or (strides[1] == 0 and shape[1] > 1):         # (0 would read as "dense")
        raise ValueError("%s must not be broadcast" % name)
    return shape, strides


def _new_status(B: int, N: int, device) -> torch.Tensor:
    """Status words for a call of N rows per sequence; one without rows writes none, and leaves nothing to report."""
    return (torch.empty if N else torch.zeros)(B, dtype=torch.int32, device=device)


def _place_args(q_in, k_in, v_in, pos, kv_len, head, q_weight, k_weight, q_out):
    B, N, Hq, D = q_in.shape
    dtype, dev = q_in.dtype, _device_of(q_in, "q_in")
    head = HeadDesc.from_buffer_copy(head)               # the caller's is left as it is
    _, head.q_stride = _rows(q_in, dev, dtype, B, N, D, "q_in")
    Hkv, head.k_stride = _rows(k_in, dev, dtype, B, N, D, "k_in")
    Hv, head.v_stride = _rows(v_in, dev, dtype, B, N, D, "v_in")
    if Hkv != Hv:
        raise ValueError("k_in and v_in must have the same heads")
    _dense(pos, dev, torch.int32, (B, N), "pos")
    _dense(kv_len, dev, torch.int32, (B,), "kv_len")
    if q_weight is not None:
        _dense(q_weight, dev, dtype, (D,), "q_weight")
    if k_weight is not None:
        _dense(k_weight, dev, dtype, (D,), "k_weight")
    if q_out is None:
        q_out = torch.empty((B, N, Hq, D), dtype=dtype, device=q_in.device)
    _dense(q_out, dev, dtype, (B, N, Hq, D), "q_out")
    return head, q_out, (torch.empty_like if N else torch.zeros_like)(kv_len), Hkv, dev          # (status: a word per sequence)


def norm_rope_kv_append(q_in, k_in, v_in, pos, kv_len, k_cache, v_cache, head: HeadDesc, q_weight=None, k_weight=None, q_out=None):
    """Norm and rotation of the query and key heads as ``head`` (``make_head_desc``) says, K and V into the caches.
    q_in [B, N, Hq, D], k_in, v_in [B, N, Hkv, D] (rows may be strided: slices of a fused projection); pos [B, N] int32;
    kv_len [B] int32; caches [B, Hkv, cap, D] (written in place at rows kv_len[b] + r).  Returns (q_out, status)."""
    head, q_out, status, Hkv, dev = _place_args(q_in, k_in, v_in, pos, kv_len, head, q_weight, k_weight, q_out)
    (Bc, Hc, cap, Dc), strides = _pair(k_cache, v_cache, dev, q_in.dtype, "caches")
    B, N, Hq, D = q_in.shape
    if Bc != B or Hc != Hkv or Dc != D:
        raise ValueError("the caches must be [B, Hkv, cap, D]")
    desc = AttnDesc(B, N, Hq, Hkv, D, cap, _DTYPES[q_in.dtype], 0.0, strides[0], strides[1], 0, 0)
    _check(load().ht_norm_rope_kv_append(ctypes.byref(desc), ctypes.byref(head), q_in.data_ptr(), k_in.data_ptr(), v_in.data_ptr(),
                                         _ptr(q_weight), _ptr(k_weight), pos.data_ptr(), kv_len.data_ptr(), q_out.data_ptr(),
                                         k_cache.data_ptr(), v_cache.data_ptr(), status.data_ptr(), _stream()))
    return q_out, status


def norm_rope_kv_append_paged(q_in, k_in, v_in, pos, kv_len, block_table, k_pages, v_pages, head: HeadDesc, q_weight=None,
                              k_weight=None, q_out=None):
    """As ``norm_rope_kv_append`` with the caches as page pools [n_pages, Hkv, page_size, D] (written in place at the
    logical rows kv_len[b] + r through block_table [B, max_pages]).  Returns (q_out, status)."""
    head, q_out, status, Hkv, dev = _place_args(q_in, k_in, v_in, pos, kv_len, head, q_weight, k_weight, q_out)
    (n_pages, Hp, page_size, Dp), strides = _pair(k_pages, v_pages, dev, q_in.dtype, "page pools")
    B, N, Hq, D = q_in.shape
    if Hp != Hkv or Dp != D:
        raise ValueError("the pools must be [n_pages, Hkv, page_size, D]")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _dense(block_table, dev, torch.int32, (B, max_pages), "block_table")
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q_in.dtype], 0.0, 0, 0, 0, 0)
    pages = PagedDesc(page_size, max_pages, n_pages, strides[0], strides[1])
    _check(load().ht_norm_rope_kv_append_paged(ctypes.byref(desc), ctypes.byref(head), ctypes.byref(pages), q_in.data_ptr(),
                                               k_in.data_ptr(), v_in.data_ptr(), _ptr(q_weight), _ptr(k_weight), pos.data_ptr(),
                                               kv_len.data_ptr(), block_table.data_ptr(), q_out.data_ptr(), k_pages.data_ptr(),
                                               v_pages.data_ptr(), status.data_ptr(), _stream()))
    return q_out, status


def _sample_args(logits, uniform, temperature, top_k, top_p, min_p):
    B, N, V = logits.shape
    dev = _device_of(logits, "logits")
    if not logits.is_contiguous():
        raise ValueError("logits must be contiguous")
    _dense(uniform, dev, torch.float32, (B, N), "uniform")
    if temperature is not None:
        _dense(temperature, dev, torch.float32, (B,), "temperature")
    if top_k is not None:
        _dense(top_k, dev, torch.int32, (B,), "top_k")
    if top_p is not None:
        _dense(top_p, dev, torch.float32, (B,), "top_p")
    if min_p is not None:
        _dense(min_p, dev, torch.float32, (B,), "min_p")
    return B, N, V, dev


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, token=None):
    """Tokens drawn from the filtered distributions of logits [B, N, V] with uniform [B, N] float32 numbers in [0, 1];
    temperature, top_p, min_p [B] float32 and top_k [B] int32, or None.  Returns (token [B, N], status [B])."""
    B, N, V, dev = _sample_args(logits, uniform, temperature, top_k, top_p, min_p)
    device = logits.device
    if token is None:
        token = torch.empty((B, N), dtype=torch.int32, device=device)
    else:
        _dense(token, dev, torch.int32, (B, N), "token")
    status = _new_status(B, N, device)
    _check(load().ht_sample(logits.data_ptr(), _DTYPES[logits.dtype], B, N, V, uniform.data_ptr(), _ptr(temperature), _ptr(top_k),
                            _ptr(top_p), _ptr(min_p), token.data_ptr(), status.data_ptr(), _stream()))
    return token, status


def verify_sampled(logits, uniform, tokens, parent, root_pred=None, temperature=None, top_k=None, top_p=None, min_p=None,
                   max_path: int = 8, accept_len=None):
    """``verify_greedy`` with the tree rows' tokens drawn as ``sample`` draws them.  logits [B, N, V], uniform [B, N];
    tokens [B, T], parent [B, N] int32, root_pred [B] int32 or None; ``accept_len`` as in ``verify_greedy``.
    Returns (pred [B, N], accept_len [B], accept_path [B, max_path], next_token [B], status [B])."""
    B, N, V, dev = _sample_args(logits, uniform, temperature, top_k, top_p, min_p)
    if tokens.dim() != 2:
        raise ValueError("tokens must be [B, T]")
    T = tokens.shape[1]
    _dense(tokens, dev, torch.int32, (B, T), "tokens")
    _dense(parent, dev, torch.int32, (B, N), "parent")
    if root_pred is not None:
        _dense(root_pred, dev, torch.int32, (B,), "root_pred")
    device = logits.device
    if accept_len is None:
        accept_len = torch.zeros(B, dtype=torch.int32, device=device)
    else:
        _dense(accept_len, dev, torch.int32, (B,), "accept_len")
    pred = torch.empty((B, N), dtype=torch.int32, device=device)
    accept_path = torch.empty((B, max_path), dtype=torch.int32, device=device)
    next_token = torch.empty(B, dtype=torch.int32, device=device)
    status = torch.empty(B, dtype=torch.int32, device=device)
    _check(load().ht_verify_sampled(logits.data_ptr(), _DTYPES[logits.dtype], uniform.data_ptr(), _ptr(temperature), _ptr(top_k),
                                    _ptr(top_p), _ptr(min_p), tokens.data_ptr(), parent.data_ptr(), _ptr(root_pred), B, N, T, V,
                                    max_path, pred.data_ptr(), accept_len.data_ptr(), accept_path.data_ptr(), next_token.data_ptr(),
                                    status.data_ptr(), _stream()))
    return pred, accept_len, accept_path, next_token, status


def _scored_args(q, kv_len, parent, cap, slopes, pos):
    if q.dim() != 4:
        raise ValueError("q must be [B, N, Hq, D]")
    B, N, Hq, D = q.shape
    dev = _device_of(q, "q")
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    _dense(kv_len, dev, torch.int32, (B,), "kv_len")
    _dense(parent, dev, torch.int32, (B, N), "parent")
    if slopes is None:
        return B, N, Hq, D, dev, ScoreDesc(cap, None, None)
    _dense(slopes, dev, torch.float32, (Hq,), "slopes")
    if pos is None:
        raise ValueError("slopes need pos")
    _dense(pos, dev, torch.int32, (B, N), "pos")
    return B, N, Hq, D, dev, ScoreDesc(cap, slopes.data_ptr(), pos.data_ptr())


def _attn_buffers(q, dev, desc, out, workspace, status, bytes_of=tree_attention_workspace):
    """The call's outputs and workspace, those that were not passed allocated."""
    if out is None:
        out = torch.empty_like(q)
    else:
        _dense(out, dev, q.dtype, q.shape, "out")
    if workspace is None:
        need = bytes_of(desc)
        ws, ws_bytes = (None, 0) if need == 0 else (torch.empty(need, dtype=torch.uint8, device=q.device), need)
    else:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous CUDA tensor of device %d" % dev)
        ws, ws_bytes = workspace, workspace.numel() * workspace.element_size()
    if status is None:
        status = _new_status(q.shape[0], q.shape[1], q.device)
    else:
        _dense(status, dev, torch.int32, q.shape[:1], "status")
    return out, ws, ws_bytes, status


def tree_attention_scored(q, k_cache, v_cache, kv_len, parent, cap: float = 0.0, slopes=None, pos=None, out=None, workspace=None,
                          status=None, scale: float = 0.0, num_splits: int = 0, flags: int = 0):
    """``tree_attention`` with the scores capped (cap * tanh(s / cap), 0: not) and biased by distance (slopes [Hq] float32
    with pos [B, N] int32, or None).  Returns (out, status)."""
    B, N, Hq, D, dev, score = _scored_args(q, kv_len, parent, cap, slopes, pos)
    (Bc, Hkv, rows, Dc), strides = _pair(k_cache, v_cache, dev, q.dtype, "caches")
    if Bc != B or Dc != D:
        raise ValueError("the caches must be [B, Hkv, cap, D]")
    desc = AttnDesc(B, N, Hq, Hkv, D, rows, _DTYPES[q.dtype], scale, strides[0], strides[1], num_splits, flags)
    out, ws, ws_bytes, status = _attn_buffers(q, dev, desc, out, workspace, status)
    _check(load().ht_tree_attention_scored(ctypes.byref(desc), ctypes.byref(score), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                           kv_len.data_ptr(), parent.data_ptr(), out.data_ptr(), _ptr(ws), ws_bytes, status.data_ptr(),
                                           _stream()))
    return out, status


def tree_attention_scored_paged(q, k_pages, v_pages, block_table, kv_len, parent, cap: float = 0.0, slopes=None, pos=None, out=None,
                                workspace=None, status=None, scale: float = 0.0, flags: int = 0):
    """``tree_attention_paged`` with the scores shaped as in ``tree_attention_scored``.  Returns (out, status)."""
    B, N, Hq, D, dev, score = _scored_args(q, kv_len, parent, cap, slopes, pos)
    (n_pages, Hkv, page_size, Dp), strides = _pair(k_pages, v_pages, dev, q.dtype, "page pools")
    if Dp != D:
        raise ValueError("the pools must be [n_pages, Hkv, page_size, D]")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _dense(block_table, dev, torch.int32, (B, max_pages), "block_table")
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q.dtype], scale, 0, 0, 0, flags)
    pages = PagedDesc(page_size, max_pages, n_pages, strides[0], strides[1])
    out, ws, ws_bytes, status = _attn_buffers(q, dev, desc, out, workspace, status)
    _check(load().ht_tree_attention_scored_paged(ctypes.byref(desc), ctypes.byref(pages), ctypes.byref(score), q.data_ptr(),
                                                 k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), kv_len.data_ptr(),
                                                 parent.data_ptr(), out.data_ptr(), _ptr(ws), ws_bytes, status.data_ptr(), _stream()))
    return out, status


_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _q8_cache(k, v, k_scale, v_scale, dev: int, dims: int, name: str):
    """Shape and strides of an 8-bit cache's codes [..., H, rows, D] and the descriptor of its scales [..., H, rows]."""
    if not (k.dtype is v.dtype is _E4M3 and k_scale.dtype is v_scale.dtype is _E8M0 and
            k.get_device() == v.get_device() == k_scale.get_device() == v_scale.get_device() == dev):
        raise ValueError("%s must be CUDA tensors of device %d, codes float8_e4m3fn and scales float8_e8m0fnu" % (name, dev))
    shape, strides, own = tuple(k.shape), k.stride(), k_scale.stride()
    if v.shape != shape or v.stride() != strides or len(shape) != dims:
        raise ValueError("%s: codes must share a %d-dimensional shape and strides" % (name, dims))
    rows = shape[:-1]
    if k_scale.shape != rows or v_scale.shape != rows or own != v_scale.stride():
        raise ValueError("%s: scales must be shaped as the codes without their last dimension, and share strides" % name)
    if strides[-1] != 1 or strides[-2] != shape[-1] or own[-1] != 1:
        raise ValueError("%s: rows must be contiguous and D apart, scales one apart" % name)
    if (0 in strides or 0 in own) and any((a == 0 or b == 0) and n > 1 for a, b, n in zip(strides, own, shape)):   # (0 would read as "dense")
        raise ValueError("%s must not be broadcast" % name)
    return shape, strides, Q8Scales(k_scale.data_ptr(), v_scale.data_ptr(), own[0] if dims == 5 else 0, own[-3], own[-2])


def norm_rope_kv_append_q8(q_in, k_in, v_in, pos, kv_len, k_cache, v_cache, k_scale, v_scale, head: HeadDesc, q_weight=None, k_weight=None,
                           q_out=None):
    """``norm_rope_kv_append`` into an 8-bit cache: codes [B, Hkv, cap, D] float8_e4m3fn, scales [B, Hkv, cap] float8_e8m0fnu (a
    row stands for codes * scale; cap a multiple of 16), written in place at rows kv_len[b] + r.  Returns (q_out, status)."""
    head, q_out, status, Hkv, dev = _place_args(q_in, k_in, v_in, pos, kv_len, head, q_weight, k_weight, q_out)
    (Bc, Hc, cap, Dc), strides, scales = _q8_cache(k_cache, v_cache, k_scale, v_scale, dev, 4, "caches")
    B, N, Hq, D = q_in.shape
    if Bc != B or Hc != Hkv or Dc != D:
        raise ValueError("the caches must be [B, Hkv, cap, D]")
    desc = AttnDesc(B, N, Hq, Hkv, D, cap, _DTYPES[q_in.dtype], 0.0, strides[0], strides[1], 0, 0)
    _check(load().ht_norm_rope_kv_append_q8(ctypes.byref(desc), ctypes.byref(head), ctypes.byref(scales), q_in.data_ptr(), k_in.data_ptr(),
                                            v_in.data_ptr(), _ptr(q_weight), _ptr(k_weight), pos.data_ptr(), kv_len.data_ptr(),
                                            q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), status.data_ptr(), _stream()))
    return q_out, status


def norm_rope_kv_append_q8_paged(q_in, k_in, v_in, pos, kv_len, block_table, k_pages, v_pages, k_scale, v_scale, head: HeadDesc,
                                 q_weight=None, k_weight=None, q_out=None):
    """As ``norm_rope_kv_append_q8`` with the cache as page pools [n_pages, Hkv, page_size, D] and [n_pages, Hkv, page_size] (written
    in place at the logical rows kv_len[b] + r through block_table [B, max_pages]).  Returns (q_out, status)."""
    head, q_out, status, Hkv, dev = _place_args(q_in, k_in, v_in, pos, kv_len, head, q_weight, k_weight, q_out)
    (n_pages, Hp, page_size, Dp), strides, scales = _q8_cache(k_pages, v_pages, k_scale, v_scale, dev, 4, "page pools")
    B, N, Hq, D = q_in.shape
    if Hp != Hkv or Dp != D:
        raise ValueError("the pools must be [n_pages, Hkv, page_size, D]")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _dense(block_table, dev, torch.int32, (B, max_pages), "block_table")
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q_in.dtype], 0.0, 0, 0, 0, 0)
    pages = PagedDesc(page_size, max_pages, n_pages, strides[0], strides[1])
    _check(load().ht_norm_rope_kv_append_q8_paged(ctypes.byref(desc), ctypes.byref(head), ctypes.byref(pages), ctypes.byref(scales),
                                                  q_in.data_ptr(), k_in.data_ptr(), v_in.data_ptr(), _ptr(q_weight), _ptr(k_weight),
                                                  pos.data_ptr(), kv_len.data_ptr(), block_table.data_ptr(), q_out.data_ptr(),
                                                  k_pages.data_ptr(), v_pages.data_ptr(), status.data_ptr(), _stream()))
    return q_out, status


def tree_attention_q8_workspace(desc: AttnDesc) -> int:
    return int(load().ht_tree_attention_q8_workspace(ctypes.byref(desc)))


def _q8_attn_args(q, kv_len, parent, window, sinks):
    if q.dim() != 4:
        raise ValueError("q must be [B, N, Hq, D]")
    B, N, Hq, D = q.shape
    dev = _device_of(q, "q")
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    _dense(kv_len, dev, torch.int32, (B,), "kv_len")
    _dense(parent, dev, torch.int32, (B, N), "parent")
    if not all(-1 << 31 <= x < 1 << 31 for x in (window, sinks)):   # (ctypes would take what is left of them in 32 bits)
        raise ValueError("window and sinks must be 32-bit integers")
    return B, N, Hq, D, dev, WindowDesc(window, sinks)


def tree_attention_q8(q, k_cache, v_cache, k_scale, v_scale, kv_len, parent, window: int = 0, sinks: int = 0, out=None, workspace=None,
                      status=None, scale: float = 0.0, num_splits: int = 0, flags: int = 0):
    """``tree_attention`` over an 8-bit cache (as ``norm_rope_kv_append_q8`` writes it); with ``window`` a row sees the keys at most
    window - 1 positions ahead of it and those at the first ``sinks`` positions.  Returns (out, status)."""
    B, N, Hq, D, dev, win = _q8_attn_args(q, kv_len, parent, window, sinks)
    (Bc, Hkv, cap, Dc), strides, scales = _q8_cache(k_cache, v_cache, k_scale, v_scale, dev, 4, "caches")
    if Bc != B or Dc != D:
        raise ValueError("the caches must be [B, Hkv, cap, D]")
    desc = AttnDesc(B, N, Hq, Hkv, D, cap, _DTYPES[q.dtype], scale, strides[0], strides[1], num_splits, flags)
    out, ws, ws_bytes, status = _attn_buffers(q, dev, desc, out, workspace, status, tree_attention_q8_workspace)
    _check(load().ht_tree_attention_q8(ctypes.byref(desc), ctypes.byref(win), ctypes.byref(scales), q.data_ptr(), k_cache.data_ptr(),
                                       v_cache.data_ptr(), kv_len.data_ptr(), parent.data_ptr(), out.data_ptr(), _ptr(ws), ws_bytes,
                                       status.data_ptr(), _stream()))
    return out, status


def tree_attention_q8_paged(q, k_pages, v_pages, k_scale, v_scale, block_table, kv_len, parent, window: int = 0, sinks: int = 0, out=None,
                            workspace=None, status=None, scale: float = 0.0, num_splits: int = 0, flags: int = 0):
    """``tree_attention_q8`` with the cache as page pools [n_pages, Hkv, page_size, D] and [n_pages, Hkv, page_size].
    Returns (out, status)."""
    B, N, Hq, D, dev, win = _q8_attn_args(q, kv_len, parent, window, sinks)
    (n_pages, Hkv, page_size, Dp), strides, scales = _q8_cache(k_pages, v_pages, k_scale, v_scale, dev, 4, "page pools")
    if Dp != D:
        raise ValueError("the pools must be [n_pages, Hkv, page_size, D]")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _dense(block_table, dev, torch.int32, (B, max_pages), "block_table")
    desc = AttnDesc(B, N, Hq, Hkv, D, max_pages * page_size, _DTYPES[q.dtype], scale, 0, 0, num_splits, flags)
    pages = PagedDesc(page_size, max_pages, n_pages, strides[0], strides[1])
    out, ws, ws_bytes, status = _attn_buffers(q, dev, desc, out, workspace, status, tree_attention_q8_workspace)
    _check(load().ht_tree_attention_q8_paged(ctypes.byref(desc), ctypes.byref(pages), ctypes.byref(win), ctypes.byref(scales), q.data_ptr(),
                                             k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(), kv_len.data_ptr(),
                                             parent.data_ptr(), out.data_ptr(), _ptr(ws), ws_bytes, status.data_ptr(), _stream()))
    return out, status


def _q8_compact_args(B, dev, kv_len, accept_len, accept_path, new_kv_len, status):
    if accept_path.dim() != 2:
        raise ValueError("accept_path must be [B, max_path]")
    _dense(kv_len, dev, torch.int32, (B,), "kv_len")
    _dense(accept_len, dev, torch.int32, (B,), "accept_len")
    _dense(accept_path, dev, torch.int32, (B, accept_path.shape[1]), "accept_path")
    if new_kv_len is None:
        new_kv_len = torch.empty_like(kv_len)
    else:
        _dense(new_kv_len, dev, torch.int32, (B,), "new_kv_len")
    if status is None:
        status = torch.empty_like(kv_len)
    else:
        _dense(status, dev, torch.int32, (B,), "status")
    return accept_path.shape[1], new_kv_len, status


def kv_compact_q8(k_cache, v_cache, k_scale, v_scale, n_rows: int, kv_len, accept_len, accept_path, new_kv_len=None, status=None):
    """In-place compaction of 8-bit caches [layers, B, Hkv, cap, D] with scales [layers, B, Hkv, cap].  Returns (new_kv_len, status)."""
    dev = _device_of(k_cache, "k_cache")
    (layers, B, Hkv, cap, D), strides, scales = _q8_cache(k_cache, v_cache, k_scale, v_scale, dev, 5, "caches")
    max_path, new_kv_len, status = _q8_compact_args(B, dev, kv_len, accept_len, accept_path, new_kv_len, status)
    desc = CacheDesc(layers, B, Hkv, cap, D, HT_F32, int(n_rows), strides[0], strides[1], strides[2])
    _check(load().ht_kv_compact_q8(k_cache.data_ptr(), v_cache.data_ptr(), ctypes.byref(scales), ctypes.byref(desc), kv_len.data_ptr(),
                                   accept_len.data_ptr(), accept_path.data_ptr(), max_path, new_kv_len.data_ptr(), status.data_ptr(), _stream()))
    return new_kv_len, status


def kv_compact_q8_paged(k_pages, v_pages, k_scale, v_scale, block_table, n_rows: int, kv_len, accept_len, accept_path, new_kv_len=None,
                        status=None):
    """In-place compaction of 8-bit page pools [layers, n_pages, Hkv, page_size, D] with scales [layers, n_pages, Hkv, page_size]
    that share block_table [B, max_pages].  Returns (new_kv_len, status)."""
    dev = _device_of(k_pages, "k_pages")
    (layers, n_pages, Hkv, page_size, D), strides, scales = _q8_cache(k_pages, v_pages, k_scale, v_scale, dev, 5, "page pools")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    B, max_pages = block_table.shape
    _dense(block_table, dev, torch.int32, (B, max_pages), "block_table")
    max_path, new_kv_len, status = _q8_compact_args(B, dev, kv_len, accept_len, accept_path, new_kv_len, status)
    desc = CacheDesc(layers, B, Hkv, max_pages * page_size, D, HT_F32, int(n_rows), strides[0], 0, 0)
    pages = PagedDesc(page_size, max_pages, n_pages, strides[1], strides[2])
    _check(load().ht_kv_compact_q8_paged(k_pages.data_ptr(), v_pages.data_ptr(), ctypes.byref(scales), ctypes.byref(desc), ctypes.byref(pages),
                                         block_table.data_ptr(), kv_len.data_ptr(), accept_len.data_ptr(), accept_path.data_ptr(), max_path,
                                         new_kv_len.data_ptr(), status.data_ptr(), _stream()))
    return new_kv_len, status


def shape_logits(logits, counts=None, tokens=None, parent=None, repetition=None, frequency=None, presence=None, bias_id=None, bias=None,
                 allowed=None, out=None):
    """Penalties, biases and masks on logits [B, N, V] ahead of ``sample`` and the verifications.  counts [B, V] int32 as
    ``count_tokens`` keeps them; tokens [B, T] and parent [B, N] int32: the draft tree, whose tokens count for the rows behind
    them; repetition, frequency, presence [B] float32; bias_id [B, n] int32 with bias [B, n] float32; allowed
    [B, N, ceil(V / 32)] int32, a bit per token.  All may be None; ``out`` may be ``logits``.  Returns (out, status [B])."""
    if logits.dim() != 3:
        raise ValueError("logits must be [B, N, V]")
    B, N, V = logits.shape
    dev = _device_of(logits, "logits")
    dtype = _DTYPES[logits.dtype]
    if not logits.is_contiguous():
        raise ValueError("logits must be contiguous")
    if counts is not None:
        _dense(counts, dev, torch.int32, (B, V), "counts")
    if (tokens is None) != (parent is None):
        raise ValueError("tokens and parent are given together")
    T = 0
    if tokens is not None:
        if tokens.dim() != 2:
            raise ValueError("tokens must be [B, T]")
        T = tokens.shape[1]
        _dense(tokens, dev, torch.int32, (B, T), "tokens")
        _dense(parent, dev, torch.int32, (B, N), "parent")
    for t, name in ((repetition, "repetition"), (frequency, "frequency"), (presence, "presence")):
        if t is not None:
            _dense(t, dev, torch.float32, (B,), name)
    if (bias_id is None) != (bias is None):
        raise ValueError("bias_id and bias are given together")
    n_bias = 0
    if bias_id is not None:
        if bias_id.dim() != 2:
            raise ValueError("bias_id must be [B, n]")
        n_bias = bias_id.shape[1]
        _dense(bias_id, dev, torch.int32, (B, n_bias), "bias_id")
        _dense(bias, dev, torch.float32, (B, n_bias), "bias")
    if allowed is not None:
        _dense(allowed, dev, torch.int32, (B, N, (V + 31) // 32), "allowed")
    if out is None:
        out = torch.empty_like(logits)
    else:
        _dense(out, dev, logits.dtype, logits.shape, "out")
    status = _new_status(B, N, logits.device)
    _check(load().ht_shape_logits(logits.data_ptr(), dtype, B, N, V, _ptr(counts), _ptr(tokens), _ptr(parent), T, _ptr(repetition),
                                  _ptr(frequency), _ptr(presence), _ptr(bias_id), _ptr(bias), n_bias, _ptr(allowed), out.data_ptr(),
                                  status.data_ptr(), _stream()))
    return out, status


def count_tokens(tokens, counts, length=None, index=None, prompt: bool = False, reset: bool = False):
    """Adds tokens [B, n] int32 to counts [B, V] int32 (in place): twice for each time a token was generated, and one where the
    prompt (``prompt``) holds it; ``reset`` begins anew.  length [B] int32: how many of them; index [B, m] int32: their places
    (``accept_path`` with ``accept_len`` as length).  Returns status [B]."""
    dev = _device_of(counts, "counts")
    if counts.dim() != 2 or tokens.dim() != 2:
        raise ValueError("counts must be [B, V] and tokens [B, n]")
    B, V = counts.shape
    n = n_tokens = tokens.shape[1]
    _dense(counts, dev, torch.int32, (B, V), "counts")
    _dense(tokens, dev, torch.int32, (B, n_tokens), "tokens")
    if index is not None:
        if index.dim() != 2:
            raise ValueError("index must be [B, m]")
        n = index.shape[1]
        _dense(index, dev, torch.int32, (B, n), "index")
    if length is not None:
        _dense(length, dev, torch.int32, (B,), "length")
    status = torch.empty(B, dtype=torch.int32, device=counts.device)
    _check(load().ht_count_tokens(tokens.data_ptr(), _ptr(index), _ptr(length), B, n_tokens, n, V, int(prompt), int(reset), counts.data_ptr(),
                                  status.data_ptr(), _stream()))
    return status
