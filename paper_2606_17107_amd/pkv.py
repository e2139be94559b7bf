"""Thin ctypes binding of libpkv (include/pkv.h), with the same names.

Only argument marshalling happens here: torch tensors contribute their device
pointers and strides, the caller's current HIP stream is passed through, and
every step of the computation runs in the HIP kernels of libpkv.so.  If the
library has not been built this module raises on first use; there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpkv.so")

PKV_OK = 0
PKV_ERR_NULL = 1
PKV_ERR_SHAPE = 2
PKV_ERR_ALIGN = 3
PKV_ERR_ALIAS = 4
PKV_ERR_UNSUPPORTED = 5
PKV_ERR_DEVICE = 6
STATUS_NAMES = {0: "PKV_OK", 1: "PKV_ERR_NULL", 2: "PKV_ERR_SHAPE", 3: "PKV_ERR_ALIGN",
                4: "PKV_ERR_ALIAS", 5: "PKV_ERR_UNSUPPORTED", 6: "PKV_ERR_DEVICE"}

PKV_BF16 = 0
PKV_F32 = 1
PKV_ROPE_HALF = 0
PKV_ROPE_INTERLEAVED = 1
PKV_ATTN_GQA = 0
PKV_ATTN_MLA = 1

_i64x3 = ctypes.c_int64 * 3
_i64x4 = ctypes.c_int64 * 4


class pkv_layout(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("v_dim", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
        ("rope_offset", ctypes.c_int32), ("rope_style", ctypes.c_int32),
        ("dst_capacity", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("src_k_stride", _i64x3), ("src_v_stride", _i64x3), ("dst_k_stride", _i64x3),
        ("dst_v_stride", _i64x3), ("err_flag", ctypes.c_void_p),
    ]


class pkv_segment(ctypes.Structure):
    _fields_ = [
        ("src_slot0", ctypes.c_int64), ("dst_seq_base", ctypes.c_int64), ("n_tokens", ctypes.c_int32),
        ("src_pos0", ctypes.c_int32), ("dst_pos0", ctypes.c_int32), ("dst_seq_len", ctypes.c_int32),
    ]


class pkv_attn_desc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("variant", ctypes.c_int32), ("n_layers", ctypes.c_int32),
        ("n_seqs", ctypes.c_int32), ("head_dim_v", ctypes.c_int32), ("total_q", ctypes.c_int32),
        ("max_q", ctypes.c_int32), ("max_kv_len", ctypes.c_int32), ("n_splits", ctypes.c_int32),
        ("window", ctypes.c_int32), ("cu_q", ctypes.c_void_p), ("kv_base", ctypes.c_void_p),
        ("cache_slots", ctypes.c_int64), ("q_stride", _i64x3), ("k_stride", _i64x3),
        ("v_stride", _i64x3), ("o_stride", _i64x3), ("lse_out", ctypes.c_void_p),
    ]


class pkv_paged_cache(ctypes.Structure):
    _fields_ = [
        ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p),
        ("n_pages", ctypes.c_int64), ("page_stride_k", ctypes.c_int64), ("page_stride_v", ctypes.c_int64),
        ("v_block_table", ctypes.c_void_p),
    ]


class pkv_block_scales(ctypes.Structure):
    _fields_ = [
        ("block_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32), ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p), ("k_stride", _i64x4), ("v_stride", _i64x4),
    ]


class pkv_segment_quant(ctypes.Structure):
    _fields_ = [
        ("src_slot0", ctypes.c_int64), ("seq", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
        ("src_pos0", ctypes.c_int32), ("dst_pos0", ctypes.c_int32),
    ]


class pkv_page_tensor(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p), ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
        ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("n_layers", ctypes.c_int32),
        ("n_slots", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("row_bytes", ctypes.c_int32),
    ]


class pkv_page_pool(ctypes.Structure):
    _fields_ = [
        ("page_size", ctypes.c_int32), ("n_tensors", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
        ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int64), ("tensors", pkv_page_tensor * 4),
        ("err_flag", ctypes.c_void_p),
    ]


class pkv_fork(ctypes.Structure):
    _fields_ = [("parent", ctypes.c_int32), ("child", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class pkv_draft(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", _i64x3), ("v_stride", _i64x3),
        ("mask", ctypes.c_void_p), ("mask_words", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class pkv_verify_desc(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("n_seqs", ctypes.c_int32), ("total_q", ctypes.c_int32), ("max_q", ctypes.c_int32),
        ("vocab", ctypes.c_int32), ("max_path", ctypes.c_int32), ("cu_q", ctypes.c_void_p),
        ("target_stride", ctypes.c_int64), ("draft_stride", ctypes.c_int64), ("err_flag", ctypes.c_void_p),
        ("reserved", ctypes.c_int64),
    ]


SYMBOLS = ("pkv_reposition_splice", "pkv_reposition_splice_freqs", "pkv_reposition_splice_paged",
           "pkv_reposition_splice_batched", "pkv_attention_workspace_size", "pkv_suffix_attention",
           "pkv_suffix_attention_paged", "pkv_suffix_attention_noalloc", "pkv_reposition_splice_quant",
           "pkv_attention_quant_workspace_size", "pkv_suffix_attention_quant", "pkv_pages_workspace_size", "pkv_pages_free",
           "pkv_pages_fork", "pkv_pages_compact", "pkv_tree_masks", "pkv_tree_attention_workspace_size", "pkv_tree_attention",
           "pkv_tree_verify_workspace_size", "pkv_tree_verify", "pkv_tree_commit_workspace_size", "pkv_tree_commit",
           "pkv_last_error", "pkv_version")
PKV_NOALLOC_SCRATCH_BYTES = 64 << 20

_lib = None


class PkvError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libpkv.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("libpkv.so is not built (run python -m paper_2606_17107_amd.build); "
                           "there is no fallback path")
    L = ctypes.CDLL(_LIB_PATH)
    P = ctypes.c_void_p
    L.pkv_reposition_splice.restype = ctypes.c_int
    L.pkv_reposition_splice.argtypes = [P, P, P, P, P, P, ctypes.c_float, ctypes.c_int32,
                                        ctypes.POINTER(pkv_layout), P]
    L.pkv_reposition_splice_freqs.restype = ctypes.c_int
    L.pkv_reposition_splice_freqs.argtypes = [P, P, P, P, P, P, P, ctypes.POINTER(ctypes.c_double),
                                              ctypes.c_int32, ctypes.POINTER(pkv_layout), P]
    L.pkv_reposition_splice_paged.restype = ctypes.c_int
    L.pkv_reposition_splice_paged.argtypes = [P, P, P, P, P, P, ctypes.c_float, ctypes.c_int32,
                                              ctypes.POINTER(pkv_layout), ctypes.POINTER(pkv_paged_cache), P]
    L.pkv_reposition_splice_batched.restype = ctypes.c_int
    L.pkv_reposition_splice_batched.argtypes = [P, P, P, P, P, ctypes.c_int32, ctypes.c_int32,
                                                ctypes.c_float, ctypes.c_int32, ctypes.POINTER(pkv_layout), P]
    L.pkv_attention_workspace_size.restype = ctypes.c_size_t
    L.pkv_attention_workspace_size.argtypes = [ctypes.POINTER(pkv_attn_desc), ctypes.c_int32,
                                               ctypes.c_int32, ctypes.c_int32]
    L.pkv_suffix_attention.restype = ctypes.c_int
    L.pkv_suffix_attention.argtypes = [P, P, P, P, P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_float, ctypes.POINTER(pkv_attn_desc), P, ctypes.c_size_t, P]
    L.pkv_suffix_attention_paged.restype = ctypes.c_int
    L.pkv_suffix_attention_paged.argtypes = [P, P, P, P, P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                             ctypes.c_float, ctypes.POINTER(pkv_attn_desc),
                                             ctypes.POINTER(pkv_paged_cache), P, ctypes.c_size_t, P]
    L.pkv_suffix_attention_noalloc.restype = ctypes.c_int
    L.pkv_suffix_attention_noalloc.argtypes = [P, P, P, P, P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                               ctypes.c_float, ctypes.POINTER(pkv_attn_desc), P]
    I, F = ctypes.c_int32, ctypes.c_float
    D, A, S = ctypes.POINTER(pkv_attn_desc), ctypes.POINTER(pkv_paged_cache), ctypes.POINTER(pkv_block_scales)
    pool = ctypes.POINTER(pkv_page_pool)
    L.pkv_reposition_splice_quant.restype = ctypes.c_int
    L.pkv_reposition_splice_quant.argtypes = [P, P, P, P, P, I, I, P, I, ctypes.POINTER(ctypes.c_double), F, I,
                                           ctypes.POINTER(pkv_layout), A, S, P]
    L.pkv_attention_quant_workspace_size.restype = ctypes.c_size_t
    L.pkv_attention_quant_workspace_size.argtypes = [D, I, I, I]
    L.pkv_suffix_attention_quant.restype = ctypes.c_int
    L.pkv_suffix_attention_quant.argtypes = [P, P, P, P, P, P, I, I, I, F, D, A, S, P, ctypes.c_size_t, P]
    L.pkv_pages_workspace_size.restype = ctypes.c_size_t
    L.pkv_pages_workspace_size.argtypes = [pool, I]
    L.pkv_pages_free.restype = ctypes.c_int
    L.pkv_pages_free.argtypes = [pool, P, P, P, P, I, P]
    L.pkv_pages_fork.restype = ctypes.c_int
    L.pkv_pages_fork.argtypes = [pool, P, P, P, P, I, P, ctypes.c_size_t, P]
    L.pkv_pages_compact.restype = ctypes.c_int
    L.pkv_pages_compact.argtypes = [pool, P, P, P, P, P, P, ctypes.c_size_t, P]
    L.pkv_tree_masks.restype = ctypes.c_int
    L.pkv_tree_masks.argtypes = [P, P, P, I, I, I, P, I, P, P, P]
    L.pkv_tree_attention_workspace_size.restype = ctypes.c_size_t
    L.pkv_tree_attention_workspace_size.argtypes = [D, I, I, I, I]
    L.pkv_tree_attention.restype = ctypes.c_int
    L.pkv_tree_attention.argtypes = [P, P, P, P, P, P, I, I, I, F, D, ctypes.POINTER(pkv_draft), A, S, P, ctypes.c_size_t, P]
    verify = ctypes.POINTER(pkv_verify_desc)
    L.pkv_tree_verify_workspace_size.restype = ctypes.c_size_t
    L.pkv_tree_verify_workspace_size.argtypes = [verify]
    L.pkv_tree_verify.restype = ctypes.c_int
    L.pkv_tree_verify.argtypes = [P, P, P, P, P, P, P, P, P, verify, P, ctypes.c_size_t, P]
    L.pkv_tree_commit_workspace_size.restype = ctypes.c_size_t
    L.pkv_tree_commit_workspace_size.argtypes = [I, I, I]
    L.pkv_tree_commit.restype = ctypes.c_int
    L.pkv_tree_commit.argtypes = [P, P, P, P, P, P, P, P, I, I, ctypes.POINTER(pkv_layout), A, S, P, ctypes.c_size_t, P]
    L.pkv_last_error.restype = ctypes.c_char_p
    L.pkv_last_error.argtypes = []
    L.pkv_version.restype = ctypes.c_int32
    L.pkv_version.argtypes = []
    _lib = L
    return L


def _check(status: int) -> None:
    if status != PKV_OK:
        raise PkvError(status, pkv_last_error())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _on_stream(make, device: torch.device, stream, returned: bool = False) -> torch.Tensor:
    """A tensor that a call on `stream` needs, made (and filled, if `make` fills) on that stream: what torch's current
    stream still does with the memory is behind it, and the call's kernels are behind a fill.  The caching allocator
    hands a block back to the stream it was made on, so scratch memory may go when the call returns; one that is
    returned may also be read on the current stream, and is kept until that is done."""
    if stream is None:
        return make()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    current = torch.cuda.current_stream(device)
    if stream.cuda_stream == current.cuda_stream:
        return make()
    with torch.cuda.stream(stream):
        t = make()
    if returned:
        t.record_stream(current)
    return t


def _scratch(nbytes: int, device: torch.device, stream) -> torch.Tensor:
    return _on_stream(lambda: torch.empty(nbytes, dtype=torch.uint8, device=device), device, stream)


# torch's raw accessors of the current stream and device; private, so a torch
# without them is served by the public ones.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        # torch's current stream on the current device, by the raw accessors once
        # torch has initialised the GPU: current_stream() looks the device up
        # through the environment and builds a Stream object (4 us a call).
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---- argument checks of the tensor-level calls --------------------------------
# The C entry points take raw device addresses; a host tensor's address handed
# to a kernel would fault the GPU.  The tensor-level calls below check type,
# dtype, size and device of every tensor they pass down (the raw pkv_* calls
# above do not).

def _need(t, name: str, device: torch.device, dtype=None, numel: Optional[int] = None,
          contiguous: bool = False) -> None:
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
    if dtype is not None and t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if numel is not None and t.numel() < numel:
        raise ValueError("%s holds %d elements, the call reads %d" % (name, t.numel(), numel))
    if contiguous and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.device != device:
        raise ValueError("%s is on %s, the call runs on %s" % (name, t.device, device))


def _gpu_device(t: torch.Tensor, name: str) -> torch.device:
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
    if t.device.type != "cuda":
        raise ValueError("libpkv tensors live on the GPU: %s is on %s" % (name, t.device))
    return t.device


def _room(t, name: str, *least) -> None:
    """t has at least these sizes: what a call reads or writes lies in it."""
    if t is not None and (t.dim() != len(least) or any(n < m for n, m in zip(t.shape, least))):
        raise ValueError("%s %s must be at least %s" % (name, tuple(t.shape), least))


def _check_splice_args(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, err_flag, dst_slot=None) -> None:
    dev = _gpu_device(src_k, "src_k")
    L, H, n, d = sk = src_k.shape
    for t, name in ((src_v, "src_v"), (dst_k, "dst_k"), (dst_v, "dst_v")):
        _need(t, name, dev, src_k.dtype)
    for t, name in ((src_pos, "src_pos"), (dst_pos, "dst_pos"), (dst_slot, "dst_slot")):
        _need(t, name, dev, torch.int32, n, contiguous=True)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    # The library takes the sizes from src_k and the bounds of the destination from dst_k (a pool has 5 dimensions).
    dv = 0 if src_v is None else src_v.shape[-1]
    if src_v is not None and src_v.shape != sk:
        _room(src_v, "src_v", L, H, n, dv)
    if dst_k is None:
        return
    dk = dst_k.shape
    heads = 3 if len(dk) == 5 else 1
    if len(dk) < 4 or dk[0] != L or dk[heads] != H or dk[-1] != d or (dst_v is not None and (dv != d or dst_v.shape != dk)):
        least = (L, *dk[1:3], H) if heads == 3 else (L, H, *dk[2:3])
        _room(dst_k, "dst_k", *least, d)
        _room(dst_v, "dst_v", *least, dv)


def _check_attention_args(q, k_cache, v_cache, out, q_pos, kv_len, n_seqs, cu_q, kv_base, lse_out,
                          workspace) -> None:
    dev = _gpu_device(q, "q")
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache"), (out, "out")):
        if t is None:
            raise TypeError("%s is required" % name)
        _need(t, name, dev, q.dtype)
    L, rows, H, d = shape = q.shape
    _need(q_pos, "q_pos", dev, torch.int32, rows, contiguous=True)
    _need(kv_len, "kv_len", dev, torch.int32, int(n_seqs), contiguous=True)
    _need(cu_q, "cu_q", dev, torch.int32, int(n_seqs) + 1, contiguous=True)
    _need(kv_base, "kv_base", dev, torch.int64, int(n_seqs), contiguous=True)
    _need(lse_out, "lse_out", dev, torch.float32, L * rows * H, contiguous=True)
    _need(workspace, "workspace", dev, contiguous=True)
    # As above: sizes from q and out, heads and bounds of the cache from k_cache.
    dv = out.shape[-1]
    if out.shape != shape:
        _room(out, "out", L, rows, H, dv)
    ks = k_cache.shape
    if ks[0] != L or ks[-1] != d or dv != d or (v_cache is not k_cache and v_cache.shape != ks):
        _room(k_cache, "k_cache", L, *ks[1:-1], d)
        _room(v_cache, "v_cache", L, *ks[1:-1], dv)


def _check_tables(block_table, v_block_table, n_seqs: int) -> None:
    if block_table.dim() != 2 or block_table.shape[0] < n_seqs:
        raise ValueError("block_table is [n_seqs][max_pages]")
    if v_block_table is not None and v_block_table.shape != block_table.shape:
        raise ValueError("block_table and v_block_table have different shapes")


# ---- raw C entry points (same names and arguments as pkv.h) -----------------

def pkv_reposition_splice(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, rope_theta, rope_dim, layout,
                          stream=None) -> int:
    return lib().pkv_reposition_splice(_ptr(src_k), _ptr(src_v), _ptr(dst_k), _ptr(dst_v), _ptr(src_pos),
                                       _ptr(dst_pos), float(rope_theta), int(rope_dim),
                                       ctypes.byref(layout) if layout is not None else None, _stream(stream))


def pkv_reposition_splice_freqs(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, dst_slot, omega, rope_dim, layout,
                                stream=None) -> int:
    w = None
    if omega is not None:
        w = (ctypes.c_double * len(omega))(*[float(x) for x in omega])
    return lib().pkv_reposition_splice_freqs(_ptr(src_k), _ptr(src_v), _ptr(dst_k), _ptr(dst_v), _ptr(src_pos),
                                             _ptr(dst_pos), _ptr(dst_slot), w, int(rope_dim),
                                             ctypes.byref(layout) if layout is not None else None, _stream(stream))


def pkv_reposition_splice_paged(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, rope_theta, rope_dim, layout, paging,
                                stream=None) -> int:
    return lib().pkv_reposition_splice_paged(_ptr(src_k), _ptr(src_v), _ptr(dst_k), _ptr(dst_v), _ptr(src_pos),
                                             _ptr(dst_pos), float(rope_theta), int(rope_dim),
                                             ctypes.byref(layout) if layout is not None else None,
                                             ctypes.byref(paging) if paging is not None else None, _stream(stream))


def pkv_reposition_splice_batched(src_k, src_v, dst_k, dst_v, segs, n_segs, max_seg_tokens, rope_theta,
                                  rope_dim, layout, stream=None) -> int:
    return lib().pkv_reposition_splice_batched(
        _ptr(src_k), _ptr(src_v), _ptr(dst_k), _ptr(dst_v), _ptr(segs), int(n_segs), int(max_seg_tokens),
        float(rope_theta), int(rope_dim), ctypes.byref(layout) if layout is not None else None,
        _stream(stream))


def pkv_attention_workspace_size(desc, n_q_heads, n_kv_heads, head_dim) -> int:
    return int(lib().pkv_attention_workspace_size(ctypes.byref(desc) if desc is not None else None,
                                                  int(n_q_heads), int(n_kv_heads), int(head_dim)))


def pkv_suffix_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale,
                         desc, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_suffix_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(out), _ptr(q_pos), _ptr(kv_len), int(n_q_heads),
        int(n_kv_heads), int(head_dim), float(scale), ctypes.byref(desc) if desc is not None else None,
        _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_suffix_attention_paged(q, k_pages, v_pages, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale,
                               desc, paging, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_suffix_attention_paged(
        _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(out), _ptr(q_pos), _ptr(kv_len), int(n_q_heads),
        int(n_kv_heads), int(head_dim), float(scale), ctypes.byref(desc) if desc is not None else None,
        ctypes.byref(paging) if paging is not None else None, _ptr(workspace), int(workspace_bytes),
        _stream(stream))


def pkv_suffix_attention_noalloc(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale,
                                 desc, stream=None) -> int:
    return lib().pkv_suffix_attention_noalloc(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(out), _ptr(q_pos), _ptr(kv_len), int(n_q_heads),
        int(n_kv_heads), int(head_dim), float(scale), ctypes.byref(desc) if desc is not None else None,
        _stream(stream))


def _ref(struct):
    return ctypes.byref(struct) if struct is not None else None


def _doubles(omega):
    return None if omega is None else (ctypes.c_double * len(omega))(*[float(x) for x in omega])


def pkv_reposition_splice_quant(src_k, src_v, k_pages, v_pages, segs, n_segs, max_seg_tokens, kv_len, n_seqs, omega,
                             rope_theta, rope_dim, layout, paging, scales, stream=None) -> int:
    return lib().pkv_reposition_splice_quant(_ptr(src_k), _ptr(src_v), _ptr(k_pages), _ptr(v_pages), _ptr(segs), int(n_segs),
                                          int(max_seg_tokens), _ptr(kv_len), int(n_seqs), _doubles(omega),
                                          float(rope_theta), int(rope_dim), _ref(layout), _ref(paging), _ref(scales),
                                          _stream(stream))


def pkv_attention_quant_workspace_size(desc, n_q_heads, n_kv_heads, head_dim) -> int:
    return int(lib().pkv_attention_quant_workspace_size(_ref(desc), int(n_q_heads), int(n_kv_heads), int(head_dim)))


def pkv_suffix_attention_quant(q, k_pages, v_pages, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc,
                            paging, scales, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_suffix_attention_quant(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(out), _ptr(q_pos), _ptr(kv_len),
                                         int(n_q_heads), int(n_kv_heads), int(head_dim), float(scale), _ref(desc),
                                         _ref(paging), _ref(scales), _ptr(workspace), int(workspace_bytes),
                                         _stream(stream))


def pkv_pages_workspace_size(pool, n_forks) -> int:
    return int(lib().pkv_pages_workspace_size(_ref(pool), int(n_forks)))


def pkv_pages_free(pool, ref, block_table, seqs, keep, n, stream=None) -> int:
    return lib().pkv_pages_free(_ref(pool), _ptr(ref), _ptr(block_table), _ptr(seqs), _ptr(keep), int(n),
                                _stream(stream))


def pkv_pages_fork(pool, ref, table_in, table_out, forks, n_forks, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_pages_fork(_ref(pool), _ptr(ref), _ptr(table_in), _ptr(table_out), _ptr(forks), int(n_forks),
                                _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_pages_compact(pool, ref_in, ref_out, table_in, table_out, n_used, workspace, workspace_bytes,
                      stream=None) -> int:
    return lib().pkv_pages_compact(_ref(pool), _ptr(ref_in), _ptr(ref_out), _ptr(table_in), _ptr(table_out),
                                   _ptr(n_used), _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_tree_masks(parent, cu_q, kv_len, n_seqs, total_q, max_q, mask, mask_words, q_pos, err_flag, stream=None) -> int:
    return lib().pkv_tree_masks(_ptr(parent), _ptr(cu_q), _ptr(kv_len), int(n_seqs), int(total_q), int(max_q), _ptr(mask),
                                int(mask_words), _ptr(q_pos), _ptr(err_flag), _stream(stream))


def pkv_tree_attention_workspace_size(desc, n_q_heads, n_kv_heads, head_dim, quant) -> int:
    return int(lib().pkv_tree_attention_workspace_size(_ref(desc), int(n_q_heads), int(n_kv_heads), int(head_dim), int(quant)))


def pkv_tree_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc, draft, paging,
                       scales, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_tree_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(out), _ptr(q_pos), _ptr(kv_len),
                                    int(n_q_heads), int(n_kv_heads), int(head_dim), float(scale), _ref(desc), _ref(draft),
                                    _ref(paging), _ref(scales), _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_tree_verify_workspace_size(desc) -> int:
    return int(lib().pkv_tree_verify_workspace_size(_ref(desc)))


def pkv_tree_verify(target_probs, draft_probs, tokens, parent, u_accept, u_sample, path, n_accepted, next_token, desc,
                    workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_tree_verify(_ptr(target_probs), _ptr(draft_probs), _ptr(tokens), _ptr(parent), _ptr(u_accept),
                                 _ptr(u_sample), _ptr(path), _ptr(n_accepted), _ptr(next_token), _ref(desc),
                                 _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_tree_commit_workspace_size(n_seqs, max_path, quant) -> int:
    return int(lib().pkv_tree_commit_workspace_size(int(n_seqs), int(max_path), int(quant)))


def pkv_tree_commit(draft_k, draft_v, cache_k, cache_v, path, n_accepted, kv_len, kv_base, n_seqs, max_path, layout, paging,
                    scales, workspace, workspace_bytes, stream=None) -> int:
    return lib().pkv_tree_commit(_ptr(draft_k), _ptr(draft_v), _ptr(cache_k), _ptr(cache_v), _ptr(path), _ptr(n_accepted),
                                 _ptr(kv_len), _ptr(kv_base), int(n_seqs), int(max_path), _ref(layout), _ref(paging),
                                 _ref(scales), _ptr(workspace), int(workspace_bytes), _stream(stream))


def pkv_last_error() -> str:
    return lib().pkv_last_error().decode()


def pkv_version() -> int:
    return int(lib().pkv_version())


# ---- descriptor builders from torch tensors ---------------------------------

def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return PKV_BF16
    if t.dtype == torch.float32:
        return PKV_F32
    raise TypeError("libpkv tensors are bfloat16 or float32, got %s" % t.dtype)


def _strides3(t: Optional[torch.Tensor]):
    if t is None:
        return _i64x3(0, 0, 0)
    st = t.stride()
    assert len(st) == 4 and st[3] == 1, "cache tensors are [layer][head][slot][channel], channels contiguous"
    return _i64x3(st[0], st[1], st[2])


def make_layout(src_k: torch.Tensor, src_v: Optional[torch.Tensor], dst_k: torch.Tensor,
                dst_v: Optional[torch.Tensor], rope_offset: int = 0, rope_style: int = PKV_ROPE_HALF,
                n_tokens: Optional[int] = None, err_flag: Optional[torch.Tensor] = None) -> pkv_layout:
    """Layout for [layer][kv_head][slot][channel] tensors (any strides, channels contiguous)."""
    n_layers, n_kv_heads, slots, head_dim = src_k.shape
    return pkv_layout(_dtype_code(src_k), n_layers, n_kv_heads, head_dim, 0 if src_v is None else src_v.shape[3],
                      slots if n_tokens is None else int(n_tokens), int(rope_offset), int(rope_style),
                      dst_k.shape[2], 0, _strides3(src_k), _strides3(src_v), _strides3(dst_k), _strides3(dst_v),
                      None if err_flag is None else err_flag.data_ptr())


def reposition_splice(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, rope_theta, rope_dim, rope_offset=0,
                      rope_style=PKV_ROPE_HALF, err_flag=None, stream=None) -> None:
    """Tensor-level call of pkv_reposition_splice; raises PkvError on a non-OK status."""
    _check_splice_args(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, err_flag)
    layout = make_layout(src_k, src_v, dst_k, dst_v, rope_offset, rope_style, err_flag=err_flag)
    _check(pkv_reposition_splice(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, rope_theta, rope_dim, layout,
                                 stream))


def reposition_splice_freqs(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, omega, rope_dim, rope_offset=0,
                            rope_style=PKV_ROPE_HALF, dst_slot=None, err_flag=None, stream=None) -> None:
    """Tensor-level call of pkv_reposition_splice_freqs (per-pair frequencies ``omega``; optional
    destination slots, else slot = dst_pos)."""
    _check_splice_args(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, err_flag, dst_slot)
    layout = make_layout(src_k, src_v, dst_k, dst_v, rope_offset, rope_style, err_flag=err_flag)
    _check(pkv_reposition_splice_freqs(src_k, src_v, dst_k, dst_v, src_pos, dst_pos, dst_slot, omega, rope_dim,
                                       layout, stream))


def make_segments(segs: Sequence[dict], device) -> torch.Tensor:
    """Pack segment dicts (src_slot0, dst_seq_base, n_tokens, src_pos0, dst_pos0, dst_seq_len) into a
    device buffer of pkv_segment records."""
    arr = (pkv_segment * max(1, len(segs)))()
    for i, s in enumerate(segs):
        arr[i] = pkv_segment(int(s["src_slot0"]), int(s["dst_seq_base"]), int(s["n_tokens"]),
                             int(s["src_pos0"]), int(s["dst_pos0"]), int(s["dst_seq_len"]))
    raw = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8)
    return raw.to(device)


def reposition_splice_batched(src_k, src_v, dst_k, dst_v, segs_dev: torch.Tensor, n_segs: int,
                              max_seg_tokens: int, rope_theta, rope_dim, rope_offset=0,
                              rope_style=PKV_ROPE_HALF, err_flag=None, stream=None) -> None:
    _check_splice_args(src_k, src_v, dst_k, dst_v, None, None, err_flag)
    _need(segs_dev, "segs_dev", src_k.device, torch.uint8, int(n_segs) * ctypes.sizeof(pkv_segment),
          contiguous=True)
    layout = make_layout(src_k, src_v, dst_k, dst_v, rope_offset, rope_style, err_flag=err_flag)
    _check(pkv_reposition_splice_batched(src_k, src_v, dst_k, dst_v, segs_dev, n_segs, max_seg_tokens,
                                         rope_theta, rope_dim, layout, stream))


def make_attn_desc(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, out: torch.Tensor,
                   max_kv_len: int, n_seqs: int = 1, cu_q: Optional[torch.Tensor] = None,
                   kv_base: Optional[torch.Tensor] = None, max_q: Optional[int] = None,
                   variant: int = PKV_ATTN_GQA, n_splits: int = 0,
                   lse_out: Optional[torch.Tensor] = None, window: int = 0) -> pkv_attn_desc:
    """Descriptor for q [L][rows][H][d], caches [L][Hkv][slots][*], out [L][rows][H][dv]."""
    n_layers, rows = q.shape[:2]
    qs, os_ = q.stride(), out.stride()
    assert qs[3] == 1 and os_[3] == 1
    return pkv_attn_desc(_dtype_code(q), int(variant), n_layers, int(n_seqs), out.shape[3], rows,
                         rows if max_q is None else int(max_q), int(max_kv_len), int(n_splits), int(window),
                         None if cu_q is None else cu_q.data_ptr(), None if kv_base is None else kv_base.data_ptr(),
                         k_cache.shape[2], _i64x3(*qs[:3]), _strides3(k_cache), _strides3(v_cache),
                         _i64x3(*os_[:3]), None if lse_out is None else lse_out.data_ptr())


def attention_workspace(desc: pkv_attn_desc, n_q_heads: int, n_kv_heads: int, head_dim: int,
                        device) -> Optional[torch.Tensor]:
    n = pkv_attention_workspace_size(desc, n_q_heads, n_kv_heads, head_dim)
    if n == 0:
        return None
    return torch.empty(n, dtype=torch.uint8, device=device)


def suffix_attention(q, k_cache, v_cache, out, q_pos, kv_len, scale, max_kv_len, n_seqs=1, cu_q=None,
                     kv_base=None, max_q=None, variant=PKV_ATTN_GQA, n_splits=0, lse_out=None,
                     workspace=None, stream=None, window=0) -> None:
    """Tensor-level call of pkv_suffix_attention (allocates the workspace with torch if not given)."""
    _check_attention_args(q, k_cache, v_cache, out, q_pos, kv_len, n_seqs, cu_q, kv_base, lse_out, workspace)
    H = q.shape[2]
    Hkv = k_cache.shape[1]
    D = q.shape[3]
    desc = make_attn_desc(q, k_cache, v_cache, out, max_kv_len, n_seqs, cu_q, kv_base, max_q, variant,
                          n_splits, lse_out, window)
    need = pkv_attention_workspace_size(desc, H, Hkv, D)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _scratch(need, q.device, stream)
    _check(pkv_suffix_attention(q, k_cache, v_cache, out, q_pos, kv_len, H, Hkv, D, scale, desc,
                                workspace, need, stream))


# ---- paged caches ------------------------------------------------------------
# Pools are [layer][page][in-page slot][kv_head][channel] (any strides, channels
# contiguous); a block table is int32 [n_seqs][max_pages] on the device.

def pool_strides3(pool: Optional[torch.Tensor]):
    """{layer, head, in-page slot} element strides of a 5-D pool."""
    if pool is None:
        return _i64x3(0, 0, 0)
    assert pool.dim() == 5 and pool.stride(4) == 1, "pools are [layer][page][slot][kv_head][channel]"
    return _i64x3(pool.stride(0), pool.stride(3), pool.stride(2))


def make_paging(block_table: torch.Tensor, k_pool: torch.Tensor, v_pool: Optional[torch.Tensor] = None,
                v_block_table: Optional[torch.Tensor] = None) -> pkv_paged_cache:
    assert block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.is_contiguous()
    if v_block_table is not None:
        assert v_block_table.dtype == torch.int32 and v_block_table.shape == block_table.shape
        assert v_block_table.is_contiguous()
    pg = pkv_paged_cache()
    pg.page_size = k_pool.shape[2]
    pg.max_pages = block_table.shape[1]
    pg.block_table = block_table.data_ptr()
    pg.n_pages = k_pool.shape[1]
    pg.page_stride_k = k_pool.stride(1)
    pg.page_stride_v = 0 if v_pool is None else v_pool.stride(1)
    pg.v_block_table = None if v_block_table is None else v_block_table.data_ptr()
    return pg


def reposition_splice_paged(src_k, src_v, k_pool, v_pool, src_pos, dst_pos, block_table, rope_theta, rope_dim,
                            rope_offset=0, rope_style=PKV_ROPE_HALF, dst_capacity=None, err_flag=None,
                            stream=None, v_block_table=None) -> None:
    """Tensor-level call of pkv_reposition_splice_paged: destination slots are logical slots of the
    sequence whose block-table row is block_table[0]."""
    _check_splice_args(src_k, src_v, k_pool, v_pool, src_pos, dst_pos, err_flag)
    _need(block_table, "block_table", src_k.device, torch.int32, contiguous=True)
    _need(v_block_table, "v_block_table", src_k.device, torch.int32, contiguous=True)
    _check_tables(block_table, v_block_table, 1)
    L = make_layout(src_k, src_v, src_k, src_v, rope_offset, rope_style, err_flag=err_flag)
    L.dst_capacity = (block_table.shape[1] * k_pool.shape[2]) if dst_capacity is None else int(dst_capacity)
    L.dst_k_stride = pool_strides3(k_pool)
    L.dst_v_stride = pool_strides3(v_pool)
    pg = make_paging(block_table, k_pool, v_pool, v_block_table)
    _check(pkv_reposition_splice_paged(src_k, src_v, k_pool, v_pool, src_pos, dst_pos, rope_theta, rope_dim, L, pg,
                                       stream))


def suffix_attention_paged(q, k_pool, v_pool, out, q_pos, kv_len, block_table, scale, max_kv_len, n_seqs=1,
                           cu_q=None, max_q=None, variant=PKV_ATTN_GQA, n_splits=0, lse_out=None, workspace=None,
                           stream=None, window=0, cache_slots=None, v_block_table=None) -> None:
    """Tensor-level call of pkv_suffix_attention_paged (q [L][rows][H][d], pools as above)."""
    _check_attention_args(q, k_pool, v_pool, out, q_pos, kv_len, n_seqs, cu_q, None, lse_out, workspace)
    _need(block_table, "block_table", q.device, torch.int32, contiguous=True)
    _need(v_block_table, "v_block_table", q.device, torch.int32, contiguous=True)
    _check_tables(block_table, v_block_table, int(n_seqs))
    H = q.shape[2]
    Hkv = k_pool.shape[3]
    D = q.shape[3]
    d = pkv_attn_desc()
    d.dtype = _dtype_code(q)
    d.variant = int(variant)
    d.n_layers = q.shape[0]
    d.n_seqs = int(n_seqs)
    d.head_dim_v = out.shape[3]
    d.total_q = q.shape[1]
    d.max_q = q.shape[1] if max_q is None else int(max_q)
    d.max_kv_len = int(max_kv_len)
    d.n_splits = int(n_splits)
    d.window = int(window)
    d.cu_q = None if cu_q is None else cu_q.data_ptr()
    d.kv_base = None
    d.cache_slots = block_table.shape[1] * k_pool.shape[2] if cache_slots is None else int(cache_slots)
    assert q.stride(3) == 1 and out.stride(3) == 1
    d.q_stride = _i64x3(q.stride(0), q.stride(1), q.stride(2))
    d.k_stride = pool_strides3(k_pool)
    d.v_stride = pool_strides3(v_pool)
    d.o_stride = _i64x3(out.stride(0), out.stride(1), out.stride(2))
    d.lse_out = None if lse_out is None else lse_out.data_ptr()
    pg = make_paging(block_table, k_pool, v_pool, v_block_table)
    need = pkv_attention_workspace_size(d, H, Hkv, D)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _scratch(need, q.device, stream)
    _check(pkv_suffix_attention_paged(q, k_pool, v_pool, out, q_pos, kv_len, H, Hkv, D, scale, d, pg, workspace,
                                      need, stream))


# ---- caches held in 8 bits ---------------------------------------------------
# Pools as above, of torch.float8_e4m3fn (or torch.uint8) codes; the scales of a
# pool are [layer][page][block in page][kv_head] bytes e (torch.uint8 or
# torch.float8_e8m0fnu) for 2^(e - 127).

_CODE_TYPES = tuple(t for t in (torch.uint8, getattr(torch, "float8_e4m3fn", None)) if t is not None)
_SCALE_TYPES = tuple(t for t in (torch.uint8, getattr(torch, "float8_e8m0fnu", None)) if t is not None)


def _check_q8_cache(dev, k_pool, v_pool, k_scale, v_scale, block_table, v_block_table, kv_len) -> None:
    """Types, shapes and devices of an 8-bit cache; v_pool and v_scale may both be None."""
    _need(block_table, "block_table", dev, torch.int32, contiguous=True)
    if block_table.dim() != 2:
        raise ValueError("block_table is [n_seqs][max_pages]")
    for pool, scale, name in ((k_pool, k_scale, "k"), (v_pool, v_scale, "v")):
        if pool is None and scale is None and name == "v":
            continue
        for t, what, types, dim in ((pool, "_pool", _CODE_TYPES, 5), (scale, "_scale", _SCALE_TYPES, 4)):
            if t is None:
                raise TypeError("%s%s is required" % (name, what))
            _need(t, name + what, dev)
            if t.dtype not in types:
                raise TypeError("%s%s must be one of %s, got %s" % (name, what, types, t.dtype))
            if t.dim() != dim:
                raise ValueError("%s%s must have %d dimensions" % (name, what, dim))
        if pool.shape != k_pool.shape or scale.shape != k_scale.shape:
            raise ValueError("keys and values have different shapes")
        L, pages, page, H = pool.shape[:4]
        if (scale.shape[0], scale.shape[1], scale.shape[3]) != (L, pages, H) or scale.shape[2] < 1 or page % scale.shape[2]:
            raise ValueError("%s_scale %s does not fit the pool %s" % (name, tuple(scale.shape), tuple(pool.shape)))
    _need(kv_len, "kv_len", dev, torch.int32, block_table.shape[0], contiguous=True)
    if v_block_table is not None:
        _need(v_block_table, "v_block_table", dev, torch.int32, contiguous=True)
        if v_block_table.shape != block_table.shape:
            raise ValueError("block_table and v_block_table have different shapes")


def make_block_scales(k_scale: torch.Tensor, v_scale: Optional[torch.Tensor], page_size: int) -> pkv_block_scales:
    """Scales [layer][page][block][kv_head] of pools with pages of page_size slots."""
    def strides(t):
        return _i64x4(0, 0, 0, 0) if t is None else _i64x4(t.stride(0), t.stride(3), t.stride(1), t.stride(2))

    return pkv_block_scales(page_size // k_scale.shape[2], 0, k_scale.data_ptr(),
                            None if v_scale is None else v_scale.data_ptr(), strides(k_scale), strides(v_scale))


def make_segments_quant(segs: Sequence[dict], device) -> torch.Tensor:
    """Pack segment dicts (src_slot0, seq, n_tokens, src_pos0, dst_pos0) into a device buffer of
    pkv_segment_quant records."""
    arr = (pkv_segment_quant * max(1, len(segs)))()
    for i, s in enumerate(segs):
        arr[i] = pkv_segment_quant(int(s["src_slot0"]), int(s["seq"]), int(s["n_tokens"]), int(s["src_pos0"]),
                                int(s["dst_pos0"]))
    return torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).to(device)


def make_layout_quant(src_k: torch.Tensor, src_v: Optional[torch.Tensor], k_pool: torch.Tensor,
                   v_pool: Optional[torch.Tensor], block_table: torch.Tensor, rope_offset: int = 0,
                   rope_style: int = PKV_ROPE_HALF, dst_capacity: Optional[int] = None,
                   err_flag: Optional[torch.Tensor] = None) -> pkv_layout:
    """Layout of a splice of [layer][kv_head][slot][channel] sources into 8-bit pools."""
    L = make_layout(src_k, src_v, src_k, src_v, rope_offset, rope_style, err_flag=err_flag)
    L.dst_capacity = block_table.shape[1] * k_pool.shape[2] if dst_capacity is None else int(dst_capacity)
    L.dst_k_stride = pool_strides3(k_pool)
    L.dst_v_stride = pool_strides3(v_pool)
    return L


def reposition_splice_quant(src_k, src_v, k_pool, v_pool, k_scale, v_scale, segs_dev, n_segs, max_seg_tokens, kv_len,
                         block_table, rope_theta, rope_dim, rope_offset=0, rope_style=PKV_ROPE_HALF, omega=None,
                         dst_capacity=None, err_flag=None, stream=None, v_block_table=None) -> None:
    """Tensor-level call of pkv_reposition_splice_quant (segs_dev: make_segments_quant; kv_len: the slots in use
    before the call, one for each row of block_table)."""
    dev = _gpu_device(src_k, "src_k")
    _need(src_v, "src_v", dev, src_k.dtype)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    _check_q8_cache(dev, k_pool, v_pool, k_scale, v_scale, block_table, v_block_table, kv_len)
    if (src_v is None) != (v_pool is None):
        raise ValueError("src_v and v_pool are given both or not at all")
    if src_k.dim() != 4 or (src_v is not None and src_v.shape != src_k.shape):
        raise ValueError("sources are [layer][kv_head][slot][channel], both of one shape")
    if (src_k.shape[0], src_k.shape[1], src_k.shape[3]) != (k_pool.shape[0], k_pool.shape[3], k_pool.shape[4]):
        raise ValueError("the source %s does not fit the pool %s" % (tuple(src_k.shape), tuple(k_pool.shape)))
    if omega is not None and len(omega) < int(rope_dim) // 2:
        raise ValueError("omega holds %d frequencies, the call reads %d" % (len(omega), int(rope_dim) // 2))
    _need(segs_dev, "segs_dev", dev, torch.uint8, int(n_segs) * ctypes.sizeof(pkv_segment_quant), contiguous=True)
    layout = make_layout_quant(src_k, src_v, k_pool, v_pool, block_table, rope_offset, rope_style, dst_capacity, err_flag)
    _check(pkv_reposition_splice_quant(src_k, src_v, k_pool, v_pool, segs_dev, n_segs, max_seg_tokens, kv_len,
                                    block_table.shape[0], omega, rope_theta, rope_dim, layout,
                                    make_paging(block_table, k_pool, v_pool, v_block_table),
                                    make_block_scales(k_scale, v_scale, k_pool.shape[2]), stream))


def make_attn_desc_quant(q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, out: torch.Tensor,
                      block_table: torch.Tensor, max_kv_len: int, n_seqs: int = 1, cu_q: Optional[torch.Tensor] = None,
                      max_q: Optional[int] = None, n_splits: int = 0, lse_out: Optional[torch.Tensor] = None,
                      window: int = 0, cache_slots: Optional[int] = None) -> pkv_attn_desc:
    """Descriptor for q [L][rows][H][d] over 8-bit pools."""
    assert q.stride(3) == 1 and out.stride(3) == 1
    return pkv_attn_desc(_dtype_code(q), PKV_ATTN_GQA, q.shape[0], int(n_seqs), out.shape[3], q.shape[1],
                         q.shape[1] if max_q is None else int(max_q), int(max_kv_len), int(n_splits), int(window),
                         None if cu_q is None else cu_q.data_ptr(), None,
                         block_table.shape[1] * k_pool.shape[2] if cache_slots is None else int(cache_slots),
                         _i64x3(*q.stride()[:3]), pool_strides3(k_pool), pool_strides3(v_pool),
                         _i64x3(*out.stride()[:3]), None if lse_out is None else lse_out.data_ptr())


def suffix_attention_quant(q, k_pool, v_pool, k_scale, v_scale, out, q_pos, kv_len, block_table, scale, max_kv_len,
                        n_seqs=1, cu_q=None, max_q=None, n_splits=0, lse_out=None, workspace=None, stream=None,
                        window=0, cache_slots=None, v_block_table=None) -> None:
    """Tensor-level call of pkv_suffix_attention_quant (allocates the workspace with torch if not given)."""
    dev = _gpu_device(q, "q")
    if out is None or v_pool is None:
        raise TypeError("out and v_pool are required")
    _need(out, "out", dev, q.dtype)
    if q.dim() != 4 or out.shape != q.shape:
        raise ValueError("q and out are [layer][row][q_head][channel], both of one shape")
    L, rows, H, D = q.shape
    _need(q_pos, "q_pos", dev, torch.int32, rows, contiguous=True)
    _need(cu_q, "cu_q", dev, torch.int32, int(n_seqs) + 1, contiguous=True)
    _need(lse_out, "lse_out", dev, torch.float32, L * rows * H, contiguous=True)
    _need(workspace, "workspace", dev, contiguous=True)
    _check_q8_cache(dev, k_pool, v_pool, k_scale, v_scale, block_table, v_block_table, None)
    _need(kv_len, "kv_len", dev, torch.int32, int(n_seqs), contiguous=True)
    if block_table.shape[0] < int(n_seqs):
        raise ValueError("block_table has %d rows for %d sequences" % (block_table.shape[0], int(n_seqs)))
    if k_pool.shape[0] != L or k_pool.shape[4] != D:
        raise ValueError("the pool %s does not fit q %s" % (tuple(k_pool.shape), tuple(q.shape)))
    if rows == 0:   # (an empty tensor has no address to pass down)
        return
    Hkv = k_pool.shape[3]
    desc = make_attn_desc_quant(q, k_pool, v_pool, out, block_table, max_kv_len, n_seqs, cu_q, max_q, n_splits, lse_out,
                             window, cache_slots)
    need = pkv_attention_quant_workspace_size(desc, H, Hkv, D)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _scratch(need, dev, stream)
    _check(pkv_suffix_attention_quant(q, k_pool, v_pool, out, q_pos, kv_len, H, Hkv, D, scale, desc,
                                   make_paging(block_table, k_pool, v_pool, v_block_table),
                                   make_block_scales(k_scale, v_scale, k_pool.shape[2]), workspace, need, stream))


# ---- pages ----------------------------------------------------------------------

def make_page_pool(tensors: Sequence[torch.Tensor], block_table: torch.Tensor, page_size: int,
                   err_flag: Optional[torch.Tensor] = None) -> pkv_page_pool:
    """The tensors of a page pool, [layer][page][slot or block in page][kv_head] and, for pools, [channel]
    (any strides, channels contiguous), under block tables of block_table's shape."""
    if not 1 <= len(tensors) <= 4:
        raise ValueError("a pool has 1 .. 4 tensors, got %d" % len(tensors))
    pool = pkv_page_pool()
    pool.page_size, pool.n_tensors = int(page_size), len(tensors)
    pool.n_seqs, pool.max_pages = block_table.shape
    pool.n_pages = tensors[0].shape[1]
    for i, t in enumerate(tensors):
        if t.dim() not in (4, 5) or t.shape[1] != pool.n_pages or (t.dim() == 5 and t.stride(4) != 1):
            raise ValueError("tensor %d must be [layer][page][slot][kv_head] or [..][channel] with %d pages, got %s"
                             % (i, pool.n_pages, tuple(t.shape)))
        b = t.element_size()
        st = t.stride()
        pool.tensors[i] = pkv_page_tensor(t.data_ptr(), st[0] * b, st[1] * b, st[2] * b, st[3] * b, t.shape[0],
                                          t.shape[2], t.shape[3], (t.shape[4] if t.dim() == 5 else 1) * b)
    pool.err_flag = None if err_flag is None else err_flag.data_ptr()
    return pool


def make_forks(forks: Sequence[dict], device) -> torch.Tensor:
    """Pack fork dicts (parent, child, n_tokens) into a device buffer of pkv_fork records."""
    arr = (pkv_fork * max(1, len(forks)))()
    for i, f in enumerate(forks):
        arr[i] = pkv_fork(int(f["parent"]), int(f["child"]), int(f["n_tokens"]), 0)
    return torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).to(device)


def _check_pages_args(tensors, ref, block_table, page_size, err_flag) -> torch.device:
    dev = _gpu_device(block_table, "block_table")
    _need(block_table, "block_table", dev, torch.int32, contiguous=True)
    if block_table.dim() != 2:
        raise ValueError("block_table is [n_seqs][max_pages]")
    for i, t in enumerate(tensors):
        if t is None:
            raise TypeError("tensor %d is None" % i)
        _need(t, "tensor %d" % i, dev)
    pages = tensors[0].shape[1] if tensors else 0
    _need(ref, "ref", dev, torch.int32, pages, contiguous=True)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    return dev


def _pages_workspace(pool, n_forks, workspace, dev, stream):
    need = pkv_pages_workspace_size(pool, n_forks)
    _need(workspace, "workspace", dev, contiguous=True)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = _scratch(max(16, need), dev, stream)
    return workspace, workspace.numel() * workspace.element_size()


def pages_free(tensors, ref, block_table, page_size, seqs, keep=None, err_flag=None, stream=None) -> None:
    """Tensor-level call of pkv_pages_free: rows seqs (int32) give back their pages behind the first keep
    slots (int32, or None for all)."""
    dev = _check_pages_args(tensors, ref, block_table, page_size, err_flag)
    _need(seqs, "seqs", dev, torch.int32, contiguous=True)
    _need(keep, "keep", dev, torch.int32, seqs.numel(), contiguous=True)
    pool = make_page_pool(tensors, block_table, page_size, err_flag)
    _check(pkv_pages_free(pool, ref, block_table, seqs, keep, seqs.numel(), stream))


def pages_fork(tensors, ref, block_table, page_size, forks_dev, n_forks, block_table_out=None, err_flag=None,
               workspace=None, stream=None) -> None:
    """Tensor-level call of pkv_pages_fork (forks_dev: make_forks); children are rows of block_table_out,
    by default block_table itself."""
    dev = _check_pages_args(tensors, ref, block_table, page_size, err_flag)
    _need(forks_dev, "forks_dev", dev, torch.uint8, int(n_forks) * ctypes.sizeof(pkv_fork), contiguous=True)
    out = block_table if block_table_out is None else block_table_out
    _need(out, "block_table_out", dev, torch.int32, contiguous=True)
    if out.shape != block_table.shape:
        raise ValueError("block_table and block_table_out have different shapes")
    pool = make_page_pool(tensors, block_table, page_size, err_flag)
    workspace, size = _pages_workspace(pool, n_forks, workspace, dev, stream)
    _check(pkv_pages_fork(pool, ref, block_table, out, forks_dev, n_forks, workspace, size, stream))


def pages_compact(tensors, ref, block_table, page_size, ref_out=None, block_table_out=None, n_used=None, err_flag=None,
                  workspace=None, stream=None) -> torch.Tensor:
    """Tensor-level call of pkv_pages_compact, in place unless other outputs are given; returns n_used
    (int32 [1] on the device)."""
    dev = _check_pages_args(tensors, ref, block_table, page_size, err_flag)
    ref_out = ref if ref_out is None else ref_out
    out = block_table if block_table_out is None else block_table_out
    _need(ref_out, "ref_out", dev, torch.int32, tensors[0].shape[1], contiguous=True)
    _need(out, "block_table_out", dev, torch.int32, contiguous=True)
    if out.shape != block_table.shape:
        raise ValueError("block_table and block_table_out have different shapes")
    if n_used is None:
        n_used = _on_stream(lambda: torch.empty(1, dtype=torch.int32, device=dev), dev, stream, returned=True)
    _need(n_used, "n_used", dev, torch.int32, 1)
    pool = make_page_pool(tensors, block_table, page_size, err_flag)
    workspace, size = _pages_workspace(pool, 0, workspace, dev, stream)
    _check(pkv_pages_compact(pool, ref, ref_out, block_table, out, n_used, workspace, size, stream))
    return n_used


# ---- trees of drafted tokens -------------------------------------------------------
# The tensor-level calls run on the device of their tensors, whichever is current.
# Rows are packed as for suffix attention (cu_q); drafted keys and values are
# [layer][kv_head][row][channel] (any strides, channels contiguous) beside the cache.
# Masks are int32 (or uint32) words [total_q][ceil(max_q / 32)].

_MASK_TYPES = tuple(t for t in (torch.int32, getattr(torch, "uint32", None)) if t is not None)


def _check_mask(mask, dev, rows: int, max_q: int) -> None:
    if mask is None:
        return
    _need(mask, "mask", dev, contiguous=True)
    if mask.dtype not in _MASK_TYPES:
        raise TypeError("mask must be one of %s, got %s" % (_MASK_TYPES, mask.dtype))
    if mask.dim() != 2 or mask.shape[0] < rows or mask.shape[1] * 32 < max_q:
        raise ValueError("mask %s must be [total_q][mask_words] for %d rows of %d bits" % (tuple(mask.shape), rows, max_q))


def _check_values(k_cache, v_cache, block_table, v_block_table, slots: Optional[int]) -> None:
    """The library takes its bounds (slots, or pages and their size) from the key cache: the values have at least as many, and
    `slots` of a contiguous cache lie in it."""
    if block_table is None:
        if slots is not None and int(slots) > k_cache.shape[2]:
            raise ValueError("%d slots, the caches have %d" % (int(slots), k_cache.shape[2]))
        if v_cache is not None and v_cache.shape[2] < k_cache.shape[2]:
            raise ValueError("the value cache has %d slots, the key cache %d" % (v_cache.shape[2], k_cache.shape[2]))
        return
    if v_cache is not None and (v_cache.shape[1] < k_cache.shape[1] or v_cache.shape[2] != k_cache.shape[2]):
        raise ValueError("the value pool has %d pages of %d slots, the key pool %d of %d" % (*v_cache.shape[1:3], *k_cache.shape[1:3]))
    if v_block_table is not None and v_block_table.shape != block_table.shape:
        raise ValueError("block_table and v_block_table have different shapes")


def _most_rows(rows: int, max_q: Optional[int]) -> int:
    return rows if max_q is None else int(max_q)


def tree_masks(parent, kv_len, n_seqs=1, cu_q=None, max_q=None, mask=None, q_pos=None, err_flag=None, stream=None):
    """Tensor-level call of pkv_tree_masks: parent int32 [total_q], numbers within each sequence.  Returns (mask, q_pos),
    allocated with torch if not given."""
    dev = _gpu_device(parent, "parent")
    _need(parent, "parent", dev, torch.int32, contiguous=True)
    rows = parent.numel()
    _need(kv_len, "kv_len", dev, torch.int32, int(n_seqs), contiguous=True)
    _need(cu_q, "cu_q", dev, torch.int32, int(n_seqs) + 1, contiguous=True)
    _need(q_pos, "q_pos", dev, torch.int32, rows, contiguous=True)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    most = _most_rows(rows, max_q)
    if mask is None:
        words = max(1, -(-most // 32))
        mask = _on_stream(lambda: torch.zeros(rows, words, dtype=torch.int32, device=dev), dev, stream, returned=True)
    if q_pos is None:
        q_pos = _on_stream(lambda: torch.zeros(rows, dtype=torch.int32, device=dev), dev, stream, returned=True)
    _check_mask(mask, dev, rows, most)
    if rows == 0:   # (an empty tensor has no address to pass down)
        return mask, q_pos
    with torch.cuda.device(dev):
        _check(pkv_tree_masks(parent, cu_q, kv_len, n_seqs, rows, most, mask, mask.shape[1], q_pos, err_flag, stream))
    return mask, q_pos


def make_draft(draft_k: torch.Tensor, draft_v: torch.Tensor, mask: Optional[torch.Tensor] = None) -> pkv_draft:
    """The drafted rows of a tree-attention call (MLA: draft_v is draft_k)."""
    return pkv_draft(draft_k.data_ptr(), draft_v.data_ptr(), _strides3(draft_k), _strides3(draft_v),
                     None if mask is None else mask.data_ptr(), 0 if mask is None else mask.shape[1], 0)


def make_tree_desc(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, out: torch.Tensor, max_kv_len: int,
                   n_seqs: int = 1, cu_q: Optional[torch.Tensor] = None, max_q: Optional[int] = None,
                   variant: int = PKV_ATTN_GQA, n_splits: int = 0, lse_out: Optional[torch.Tensor] = None, window: int = 0,
                   kv_base: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                   cache_slots: Optional[int] = None) -> pkv_attn_desc:
    """Descriptor of a tree-attention call: contiguous caches [L][Hkv][slots][*], or (block_table given) pools
    [L][page][slot][Hkv][*]."""
    if block_table is None:
        d = make_attn_desc(q, k_cache, v_cache, out, max_kv_len, n_seqs, cu_q, kv_base, max_q, variant, n_splits, lse_out, window)
        if cache_slots is not None:
            d.cache_slots = int(cache_slots)
        return d
    d = make_attn_desc_quant(q, k_cache, v_cache, out, block_table, max_kv_len, n_seqs, cu_q, max_q, n_splits, lse_out, window,
                             cache_slots)
    d.variant = int(variant)
    return d


def tree_attention(q, k_cache, v_cache, draft_k, draft_v, out, q_pos, kv_len, scale, max_kv_len, mask=None, n_seqs=1, cu_q=None,
                   kv_base=None, max_q=None, variant=PKV_ATTN_GQA, n_splits=0, lse_out=None, workspace=None, stream=None,
                   window=0, block_table=None, v_block_table=None, k_scale=None, v_scale=None, cache_slots=None) -> None:
    """Tensor-level call of pkv_tree_attention (allocates the workspace with torch if not given).  block_table: the caches
    are pools; k_scale and v_scale: pools of 8-bit codes.  MLA: v_cache is k_cache and draft_v is draft_k."""
    dev = _gpu_device(q, "q")
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache"), (draft_k, "draft_k"), (draft_v, "draft_v"), (out, "out")):
        if t is None:
            raise TypeError("%s is required" % name)
    quant = k_scale is not None or v_scale is not None
    for t, name in ((draft_k, "draft_k"), (draft_v, "draft_v"), (out, "out")):
        _need(t, name, dev, q.dtype)
    if q.dim() != 4 or out.dim() != 4 or out.shape[:3] != q.shape[:3]:
        raise ValueError("q and out are [layer][row][q_head][channel]")
    L, rows, H, D = q.shape
    most = _most_rows(rows, max_q)
    _need(q_pos, "q_pos", dev, torch.int32, rows, contiguous=True)
    _need(kv_len, "kv_len", dev, torch.int32, int(n_seqs), contiguous=True)
    _need(cu_q, "cu_q", dev, torch.int32, int(n_seqs) + 1, contiguous=True)
    _need(kv_base, "kv_base", dev, torch.int64, int(n_seqs), contiguous=True)
    _need(lse_out, "lse_out", dev, torch.float32, L * rows * H, contiguous=True)
    _need(workspace, "workspace", dev, contiguous=True)
    _check_mask(mask, dev, rows, most)
    if quant:
        if block_table is None:
            raise ValueError("a cache held in 8 bits is paged: block_table is required")
        _check_q8_cache(dev, k_cache, v_cache, k_scale, v_scale, block_table, v_block_table, None)
    else:
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            _need(t, name, dev, q.dtype)
    if block_table is not None:
        _need(block_table, "block_table", dev, torch.int32, contiguous=True)
        _need(v_block_table, "v_block_table", dev, torch.int32, contiguous=True)
        if block_table.dim() != 2 or block_table.shape[0] < int(n_seqs):
            raise ValueError("block_table is [n_seqs][max_pages]")
    dim = 4 if block_table is None else 5
    if k_cache.dim() != dim or v_cache.dim() != dim:
        raise ValueError("caches are [layer][kv_head][slot][channel], pools [layer][page][slot][kv_head][channel]")
    Hkv = k_cache.shape[1 if block_table is None else 3]
    for cache, draft, width, name in ((k_cache, draft_k, D, "k"), (v_cache, draft_v, D if variant == PKV_ATTN_MLA else out.shape[3], "v")):
        if cache.shape[0] != L or cache.shape[-1] != width:
            raise ValueError("%s_cache %s does not fit q %s" % (name, tuple(cache.shape), tuple(q.shape)))
        if draft.dim() != 4 or (draft.shape[0], draft.shape[1], draft.shape[3]) != (L, Hkv, width) or draft.shape[2] < rows:
            raise ValueError("draft_%s %s must be [%d][%d][%d][%d]" % (name, tuple(draft.shape), L, Hkv, rows, width))
    if v_cache.shape[1 if block_table is None else 3] != Hkv:
        raise ValueError("k_cache %s and v_cache %s have different heads" % (tuple(k_cache.shape), tuple(v_cache.shape)))
    _check_values(k_cache, v_cache, block_table, v_block_table, cache_slots)
    if rows == 0:   # (an empty tensor has no address to pass down)
        return
    desc = make_tree_desc(q, k_cache, v_cache, out, max_kv_len, n_seqs, cu_q, max_q, variant, n_splits, lse_out, window, kv_base,
                          block_table, cache_slots)
    need = pkv_tree_attention_workspace_size(desc, H, Hkv, D, quant)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = _scratch(need, dev, stream)
    paging = None if block_table is None else make_paging(block_table, k_cache, v_cache, v_block_table)
    scales = make_block_scales(k_scale, v_scale, k_cache.shape[2]) if quant else None
    with torch.cuda.device(dev):
        _check(pkv_tree_attention(q, k_cache, v_cache, out, q_pos, kv_len, H, Hkv, D, scale, desc,
                                  make_draft(draft_k, draft_v, mask), paging, scales, workspace, need, stream))


def make_verify_desc(target_probs: torch.Tensor, draft_probs: Optional[torch.Tensor], cu_q: Optional[torch.Tensor], n_seqs: int,
                     max_q: int, max_path: int, err_flag: Optional[torch.Tensor] = None) -> pkv_verify_desc:
    """Descriptor of a verification of probabilities [total_q][vocab] (any row stride)."""
    rows, vocab = target_probs.shape
    assert target_probs.stride(1) == 1 and (draft_probs is None or draft_probs.stride(1) == 1)
    return pkv_verify_desc(_dtype_code(target_probs), int(n_seqs), rows, int(max_q), vocab, int(max_path),
                           None if cu_q is None else cu_q.data_ptr(), target_probs.stride(0),
                           0 if draft_probs is None else draft_probs.stride(0),
                           None if err_flag is None else err_flag.data_ptr(), 0)


def tree_verify(target_probs, tokens, parent, u_accept, u_sample, max_path, draft_probs=None, n_seqs=1, cu_q=None, max_q=None,
                path=None, n_accepted=None, next_token=None, err_flag=None, workspace=None, stream=None):
    """Tensor-level call of pkv_tree_verify; returns (path, n_accepted, next_token), allocated with torch if not given."""
    dev = _gpu_device(target_probs, "target_probs")
    if target_probs.dim() != 2 or target_probs.stride(1) != 1:
        raise ValueError("target_probs is [total_q][vocab], contiguous along the vocabulary")
    rows = target_probs.shape[0]
    _need(draft_probs, "draft_probs", dev, target_probs.dtype)
    if draft_probs is not None and (draft_probs.shape != target_probs.shape or draft_probs.stride(1) != 1):
        raise ValueError("draft_probs must have target_probs' shape and be contiguous along the vocabulary")
    for t, name, kind, n in ((tokens, "tokens", torch.int32, rows), (parent, "parent", torch.int32, rows),
                             (u_accept, "u_accept", torch.float32, rows), (u_sample, "u_sample", torch.float32, int(n_seqs))):
        if t is None:
            raise TypeError("%s is required" % name)
        _need(t, name, dev, kind, n, contiguous=True)
    _need(cu_q, "cu_q", dev, torch.int32, int(n_seqs) + 1, contiguous=True)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    _need(workspace, "workspace", dev, contiguous=True)
    outs = []
    for t, name, shape in ((path, "path", (int(n_seqs), int(max_path))), (n_accepted, "n_accepted", (int(n_seqs),)),
                           (next_token, "next_token", (int(n_seqs),))):
        if t is None:
            t = _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=dev), dev, stream, returned=True)
        _need(t, name, dev, torch.int32, contiguous=True)
        if tuple(t.shape) != shape:
            raise ValueError("%s must be %s, got %s" % (name, shape, tuple(t.shape)))
        outs.append(t)
    desc = make_verify_desc(target_probs, draft_probs, cu_q, n_seqs, _most_rows(rows, max_q), max_path, err_flag)
    need = pkv_tree_verify_workspace_size(desc)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = _scratch(max(16, need), dev, stream)
    with torch.cuda.device(dev):
        _check(pkv_tree_verify(target_probs, draft_probs, tokens, parent, u_accept, u_sample, *outs, desc, workspace,
                               workspace.numel() * workspace.element_size(), stream))
    return tuple(outs)


def make_commit_layout(draft_k: torch.Tensor, draft_v: Optional[torch.Tensor], cache_k: torch.Tensor,
                       cache_v: Optional[torch.Tensor], block_table: Optional[torch.Tensor] = None, slots: int = 0,
                       err_flag: Optional[torch.Tensor] = None) -> pkv_layout:
    """Layout of a commit of drafted rows into contiguous caches (slots: those of the tensors) or, with a block table,
    into pools (slots: those of a sequence, 0 for all that its row of the table holds)."""
    L = make_layout(draft_k, draft_v, draft_k, draft_v, err_flag=err_flag)
    if block_table is None:
        L.dst_capacity = int(slots)
        L.dst_k_stride, L.dst_v_stride = _strides3(cache_k), _strides3(cache_v)
    else:
        L.dst_capacity = int(slots) or block_table.shape[1] * cache_k.shape[2]
        L.dst_k_stride, L.dst_v_stride = pool_strides3(cache_k), pool_strides3(cache_v)
    return L


def tree_commit(draft_k, draft_v, cache_k, cache_v, path, n_accepted, kv_len, kv_base=None, block_table=None, v_block_table=None,
                k_scale=None, v_scale=None, slots=None, err_flag=None, workspace=None, stream=None) -> None:
    """Tensor-level call of pkv_tree_commit (path int32 [n_seqs][max_path]); values may be None (MLA).  No workspace is needed:
    pkv_tree_commit_workspace_size is 0."""
    dev = _gpu_device(draft_k, "draft_k")
    quant = k_scale is not None or v_scale is not None
    _need(path, "path", dev, torch.int32, contiguous=True)
    if path.dim() != 2:
        raise ValueError("path is [n_seqs][max_path]")
    n_seqs, max_path = path.shape
    for t, name in ((n_accepted, "n_accepted"), (kv_len, "kv_len")):
        if t is None:
            raise TypeError("%s is required" % name)
        _need(t, name, dev, torch.int32, n_seqs, contiguous=True)
    _need(kv_base, "kv_base", dev, torch.int64, n_seqs, contiguous=True)
    _need(err_flag, "err_flag", dev, torch.int32, 1)
    _need(workspace, "workspace", dev, contiguous=True)
    if cache_k is None:
        raise TypeError("cache_k is required")
    if (draft_v is None) != (cache_v is None):
        raise ValueError("draft_v and cache_v are given both or not at all")
    if quant:
        if block_table is None:
            raise ValueError("a cache held in 8 bits is paged: block_table is required")
        _check_q8_cache(dev, cache_k, cache_v, k_scale, v_scale, block_table, v_block_table, None)
        _need(draft_v, "draft_v", dev, draft_k.dtype)
    else:
        for t, name in ((draft_v, "draft_v"), (cache_k, "cache_k"), (cache_v, "cache_v")):
            _need(t, name, dev, draft_k.dtype)
    if block_table is not None:
        _need(block_table, "block_table", dev, torch.int32, contiguous=True)
        _need(v_block_table, "v_block_table", dev, torch.int32, contiguous=True)
        if block_table.dim() != 2 or block_table.shape[0] < n_seqs:
            raise ValueError("block_table is [n_seqs][max_pages]")
    dim, heads = (4, 1) if block_table is None else (5, 3)
    for draft, cache, name in ((draft_k, cache_k, "k"), (draft_v, cache_v, "v")):
        if draft is None:
            continue
        if draft.dim() != 4 or cache.dim() != dim or draft.shape[:2] != draft_k.shape[:2] or draft.shape[2] != draft_k.shape[2] \
                or (draft.shape[0], draft.shape[1], draft.shape[3]) != (cache.shape[0], cache.shape[heads], cache.shape[-1]):
            raise ValueError("draft_%s %s does not fit cache_%s %s" % (name, tuple(draft.shape), name, tuple(cache.shape)))
    _check_values(cache_k, cache_v, block_table, v_block_table, slots)
    if slots is None:
        slots = cache_k.shape[2] if block_table is None else 0
    layout = make_commit_layout(draft_k, draft_v, cache_k, cache_v, block_table, slots, err_flag)
    paging = None if block_table is None else make_paging(block_table, cache_k, cache_v, v_block_table)
    scales = make_block_scales(k_scale, v_scale, cache_k.shape[2]) if quant else None
    with torch.cuda.device(dev):
        _check(pkv_tree_commit(draft_k, draft_v, cache_k, cache_v, path, n_accepted, kv_len, kv_base, n_seqs, max_path, layout,
                               paging, scales, workspace, 0 if workspace is None else workspace.numel() * workspace.element_size(),
                               stream))
