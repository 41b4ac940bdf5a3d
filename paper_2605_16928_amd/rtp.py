"""ctypes binding of librtp.so -- argument marshalling only.

Every function has the name and argument order of its C entry point (see
include/rtp.h); tensors are torch tensors on the GPU (only their data_ptr() is
used), sizes are Python ints, and the HIP stream defaults to torch's current
stream.  A non-zero return code raises RtpError with the library's message.
There is no fallback: if the library cannot be loaded, importing succeeds but
the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("RTP_LIB", os.path.join(HERE, "librtp.so"))

RTP_OK, RTP_ERR_INVALID_ARG, RTP_ERR_UNSUPPORTED, RTP_ERR_WORKSPACE, RTP_ERR_HIP = 0, -1, -2, -3, -4

EXPORTS = [
    "rtp_last_error", "rtp_version", "rtp_profile_start", "rtp_profile_stop", "rtp_index_score_traffic_probe",
    "rtp_index_score",
    "rtp_topp_workspace_bytes", "rtp_topp_workspace_init", "rtp_topp_select", "rtp_topp_select_noalloc",
    "rtp_sparse_attn_decode_workspace_bytes", "rtp_sparse_attn_decode",
    "rtp_sparse_attn_prefill_workspace_bytes", "rtp_sparse_attn_prefill", "rtp_sparse_attn_prefill_tile_stats",
    "rtp_local_attn_workspace_bytes", "rtp_local_attn",
    "rtp_dense_attn_workspace_bytes", "rtp_dense_attn",
    "rtp_index_project", "rtp_topk_select",
    "rtp_block_topp_workspace_bytes", "rtp_block_topp_select", "rtp_sparsity_stats",
    "rtp_select_attend_decode_workspace_bytes", "rtp_select_attend_decode",
    "rtp_decode_attention", "rtp_decode_attention_paged", "rtp_sparse_attn_decode_paged",
    "rtp_kv_ring_heads", "rtp_kv_ring_append", "rtp_kv_ring_fill",
    "rtp_local_attn_ring_workspace_bytes", "rtp_local_attn_ring",
    "rtp_kv4_append", "rtp_kv4_read",
    "rtp_sparse_attn_decode_kv4_workspace_bytes", "rtp_sparse_attn_decode_kv4",
    "rtp_local_attn_kv4_workspace_bytes", "rtp_local_attn_kv4",
    "rtp_dense_attn_kv4_workspace_bytes", "rtp_dense_attn_kv4",
    "rtp_kv_pages_workspace_bytes", "rtp_kv_pages_init", "rtp_kv_pages_extend", "rtp_kv_pages_fork",
    "rtp_kv_pages_truncate", "rtp_kv_pages_compact", "rtp_kv_pages_copy",
    "rtp_kv_append", "rtp_dense_attn_chunk_workspace_bytes", "rtp_dense_attn_chunk", "rtp_dense_attn_chunk_kv4",
    "rtp_local_attn_chunk_workspace_bytes", "rtp_local_attn_chunk", "rtp_local_attn_chunk_kv4",
]
RTP_SIDE_QUERY, RTP_SIDE_KEY = 0, 1
RTP_DTYPE_BF16, RTP_DTYPE_FP16 = 0, 1
RTP_HEADS_ALL, RTP_HEADS_RETRIEVAL = 0, 1


class RtpError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"rtp error {code}: {msg}")
        self.code = code


class rtp_launch_time(C.Structure):
    _fields_ = [("kernel", C.c_char_p), ("us", C.c_float)]


class rtp_layer_desc(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("index_dim", C.c_int32),
        ("n_ret", C.c_int32), ("ret_heads", C.POINTER(C.c_int32)),
        ("sink", C.c_int32), ("window", C.c_int32),
        ("softmax_scale", C.c_float), ("index_scale", C.c_float), ("kv_dtype", C.c_int32),
    ]


class rtp_kv4_cache(C.Structure):
    _fields_ = [
        ("codes", C.c_void_p), ("code_page_stride", C.c_int64), ("code_head_stride", C.c_int64),
        ("scales", C.c_void_p), ("scale_page_stride", C.c_int64), ("scale_head_stride", C.c_int64),
        ("page_table", C.c_void_p), ("pt_stride", C.c_int64), ("page_size", C.c_int32), ("n_pages", C.c_int32),
    ]
    n_heads = n_seqs = 1 << 31                      # KV heads of the pools, rows of the table: known where kv4_cache made it
    _device = _dtype = None                         # and of which device and (16-bit rows) type


def _held(who: str, layer, cache, B: int):
    """The C struct has no head and no row count; what a cache of tensors holds is checked here."""
    if layer.n_kv_heads > cache.n_heads or B > cache.n_seqs:
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: a cache of {cache.n_heads} KV heads and {cache.n_seqs} sequences, a call over "
                                            f"{layer.n_kv_heads} and {B}")


def _int32(t) -> bool:
    return str(t.dtype) == "torch.int32" and t.is_contiguous()


def kv4_cache(codes, scales, page_table) -> rtp_kv4_cache:
    """Descriptor of a 4-bit cache in torch tensors: codes uint8 [n_kv_heads, n_pages, page_size, 128], scales uint8 with
    n_kv_heads and n_pages in front and page_size * 8 bytes behind them, page_table int32 [B, pages].  The first two dims of codes
    and scales may have any strides (a page-major pool as a transposed view).  Calls over more KV heads or sequences than these
    tensors hold are refused."""
    ok = codes.dim() == 4 and codes.shape[3] == 128 and min(codes.shape) > 0 and codes.element_size() == 1 \
        and scales.dim() >= 3 and scales.shape[:2] == codes.shape[:2] and scales.element_size() == 1 \
        and scales[0, 0].numel() == 8 * codes.shape[2] and codes[0, 0].is_contiguous() and scales[0, 0].is_contiguous() \
        and page_table.dim() == 2 and _int32(page_table) and codes.device == scales.device == page_table.device
    if not ok:
        raise RtpError(RTP_ERR_INVALID_ARG, "kv4_cache: bytes in codes [heads, pages, page_size, 128] and scales [heads, pages, "
                                            "8 * page_size], a page's own contiguous, and a contiguous int32 page_table [B, pages], on one device")
    c = rtp_kv4_cache(codes.data_ptr(), codes.stride(1), codes.stride(0), scales.data_ptr(), scales.stride(1), scales.stride(0),
                      page_table.data_ptr(), page_table.shape[1], codes.shape[2], codes.shape[1])
    c.n_heads, c.n_seqs = codes.shape[0], page_table.shape[0]
    c._keepalive, c._device = (codes, scales, page_table), codes.get_device()
    return c


class rtp_kv_cache(C.Structure):
    _fields_ = [
        ("K", C.c_void_p), ("V", C.c_void_p), ("row_stride", C.c_int64), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
        ("page_table", C.c_void_p), ("pt_stride", C.c_int64), ("page_size", C.c_int32), ("n_pages", C.c_int32),
    ]
    n_heads = n_seqs = 1 << 31                      # as in rtp_kv4_cache
    _device = _dtype = None


class rtp_chunk(C.Structure):
    _fields_ = [("q_offset", C.c_void_p), ("ctx_len", C.c_void_p), ("B", C.c_int32), ("total_q", C.c_int32), ("max_q", C.c_int32),
                ("max_ctx", C.c_int64)]
    _device = None


class rtp_rope(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float)]
    _device = None


def kv_cache(K, V, page_table) -> rtp_kv_cache:
    """Descriptor of a 16-bit cache in torch tensors: K and V [n_kv_heads, n_pages, page_size, 128] of the same strides (any but the
    last's: a pool with the pages, or the tokens, in front as a permuted view), page_table int32 [B, pages].  Calls over more KV heads or
    sequences than these tensors hold, or of a layer of another type, are refused."""
    ok = K.dim() == 4 and K.shape[3] == 128 and min(K.shape) > 0 and K.element_size() == 2 and K.stride(3) == 1 and K.dtype == V.dtype \
        and K.shape == V.shape and K.stride() == V.stride() and page_table.dim() == 2 and _int32(page_table) \
        and K.device == V.device == page_table.device
    if not ok:
        raise RtpError(RTP_ERR_INVALID_ARG, "kv_cache: 16-bit K and V [heads, pages, page_size, 128] of the same strides, rows contiguous, and a "
                                            "contiguous int32 page_table [B, pages], on one device")
    c = rtp_kv_cache(K.data_ptr(), V.data_ptr(), K.stride(2), K.stride(1), K.stride(0), page_table.data_ptr(), page_table.shape[1], K.shape[2],
                     K.shape[1])
    c.n_heads, c.n_seqs = K.shape[0], page_table.shape[0]
    c._keepalive, c._device, c._dtype = (K, V, page_table), K.get_device(), K.dtype
    return c


def chunk_desc(q_offset, ctx_len, total_q: int, max_q: int, max_ctx: int) -> rtp_chunk:
    """Descriptor of a batch of new tokens: q_offset int32 [B + 1], ctx_len int32 [B], and the host's bounds."""
    if q_offset.dim() != 1 or ctx_len.dim() != 1 or not _int32(q_offset) or not _int32(ctx_len) or q_offset.shape[0] != ctx_len.shape[0] + 1 \
            or q_offset.device != ctx_len.device:
        raise RtpError(RTP_ERR_INVALID_ARG, "chunk_desc: contiguous int32 q_offset [B + 1] and ctx_len [B] on one device expected")
    c = rtp_chunk(q_offset.data_ptr(), ctx_len.data_ptr(), ctx_len.shape[0], total_q, max_q, max_ctx)
    c._keepalive, c._device = (q_offset, ctx_len), q_offset.get_device()
    return c


def rope_desc(inv_freq, interleaved: bool = False, scale: float = 0.0) -> rtp_rope:
    """Descriptor of a rotation: inv_freq fp32 [rotary_dim / 2]."""
    if inv_freq.dim() != 1 or str(inv_freq.dtype) != "torch.float32" or not inv_freq.is_contiguous():
        raise RtpError(RTP_ERR_INVALID_ARG, "rope_desc: contiguous float32 inv_freq [rotary_dim / 2] expected")
    r = rtp_rope(inv_freq.data_ptr(), 2 * inv_freq.shape[0], 1 if interleaved else 0, scale)
    r._keepalive, r._device = (inv_freq,), inv_freq.get_device()
    return r


def _on_one_device(who: str, descriptors, tensors):
    """The tensors of a call, and those that its descriptors were made of, lie on the current device, whose stream takes the launches.
    (Integers, not device objects: a call of one short kernel is bound by its host time.)"""
    at = [d._device for d in descriptors if d is not None and d._device is not None]
    for t in tensors:
        if t is not None and t.__class__ is not int and hasattr(t, "get_device"):
            at.append(t.get_device())
    if at:
        current = _current_device()
        if min(at) != current or max(at) != current:
            raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: tensors on devices {sorted(set(at))}, the current one is {current}")


_torch_types = None


def _type_of(who: str, layer, cache):
    """The layer's 16-bit type as torch names it (None: a layer that the call refuses), which is the cache's."""
    global _torch_types
    if _torch_types is None:
        import torch
        _torch_types = {RTP_DTYPE_BF16: torch.bfloat16, RTP_DTYPE_FP16: torch.float16, "lse": torch.float32}
    kind = _torch_types.get(layer.kv_dtype)
    if cache._dtype is not kind and cache._dtype is not None and kind is not None:
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: a cache of {kind} expected, as the layer's type is; it is of {cache._dtype}")
    return kind


def _rows(who: str, t, total: int, heads: int, name: str, stride: int, kind):
    """The address of packed rows [total or more, heads, 128] of type `kind`, whose tokens are `stride` apart and whose heads are not."""
    if t is None or t.__class__ is int:
        return t
    n, s = t.shape, t.stride()
    if len(n) != 3 or n[0] < total or n[1] != heads or n[2] != 128 or t.element_size() != 2 \
            or (total and (s[2] != 1 or (s[1] != 128 and heads > 1))):
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: {name} of 16 bits [{total} or more, {heads}, 128] expected, a token's rows contiguous")
    if total > 1 and s[0] != stride:
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: {name} with tokens {stride} elements apart expected, they are {s[0]}")
    if t.dtype is not kind and kind is not None:
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: {name} of {kind} expected, as the layer's type is; it is of {t.dtype}")
    return t.data_ptr()


class rtp_page_map(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("pt_stride", C.c_int64), ("page_refs", C.c_void_p),
                ("n_seqs", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32)]


class rtp_page_pool(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("page_bytes", C.c_int64),
                ("n_heads", C.c_int32)]


def page_map(page_table, page_refs, page_size: int) -> rtp_page_map:
    """Descriptor of a page table int32 [n_seqs, pages] and reference counts int32 [n_pages], both contiguous."""
    if page_table.dim() != 2 or page_refs.dim() != 1 or not _int32(page_table) or not _int32(page_refs) \
            or page_table.device != page_refs.device:
        raise RtpError(RTP_ERR_INVALID_ARG, "page_map: contiguous int32 page_table [n_seqs, pages] and page_refs [n_pages] on one "
                                            "device expected")
    m = rtp_page_map(page_table.data_ptr(), page_table.shape[1], page_refs.data_ptr(), page_table.shape[0], page_refs.shape[0], page_size)
    m._keepalive = (page_table, page_refs)
    return m


def page_pools(pools: Sequence):
    """Descriptors of pools in torch tensors [heads, n_pages, ...]: a page's own bytes contiguous, the first two dims of any
    strides (the K and V pools of the paged calls as [n_kv_heads, n_pages, page_size * 128], a 4-bit cache's codes and scales)."""
    arr = (rtp_page_pool * max(len(pools), 1))()
    for i, t in enumerate(pools):
        if t.dim() < 3 or min(t.shape) == 0 or not t[0, 0].is_contiguous() or t.device != pools[0].device:
            raise RtpError(RTP_ERR_INVALID_ARG, "page_pools: tensors [heads, n_pages, ...] with contiguous pages on one device expected")
        e = t.element_size()
        arr[i] = rtp_page_pool(t.data_ptr(), t.stride(1) * e, t.stride(0) * e, t[0, 0].numel() * e, t.shape[0])
    arr._keepalive = list(pools)
    arr.n_pages = min((t.shape[1] for t in pools), default=0)
    arr.n_pools = len(pools)
    return arr


def layer_desc(n_q_heads: int, n_kv_heads: int, ret_heads: Sequence[int], sink: int, window: int,
               head_dim: int = 128, index_dim: int = 16, softmax_scale: float = 0.0,
               index_scale: float = 0.0, kv_dtype: int = 0) -> rtp_layer_desc:
    arr = (C.c_int32 * max(len(ret_heads), 1))(*ret_heads)
    d = rtp_layer_desc(n_q_heads, n_kv_heads, head_dim, index_dim, len(ret_heads),
                       C.cast(arr, C.POINTER(C.c_int32)), sink, window, softmax_scale, index_scale, kv_dtype)
    d._keepalive = arr
    return d


_lib = None


def lib() -> C.CDLL:
    """Loads librtp.so (built by paper_2605_16928_amd.build); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RtpError(-100, f"{LIB_PATH} is missing: build it with `python -m paper_2605_16928_amd.build` "
                             f"(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    dp = C.POINTER(rtp_layer_desc)
    L.rtp_last_error.restype = C.c_char_p
    L.rtp_last_error.argtypes = []
    L.rtp_version.restype = C.c_char_p
    L.rtp_version.argtypes = []
    L.rtp_index_score.restype = i32
    L.rtp_index_score.argtypes = [dp, vp, vp, vp, i64, vp, vp, vp, i32, i32, i64, vp, i64, vp, vp, sz, vp]
    L.rtp_topp_workspace_bytes.restype = sz
    L.rtp_topp_workspace_bytes.argtypes = [i32, i64]
    L.rtp_topp_select.restype = i32
    L.rtp_topp_select.argtypes = [vp, i64, vp, vp, i32, i64, vp, i64, vp, vp, vp, i32, vp, sz, vp]
    L.rtp_index_score_traffic_probe.restype = i32
    L.rtp_index_score_traffic_probe.argtypes = [dp, vp, vp, vp, i64, vp, vp, vp, i32, i32, i64, vp, i64, vp]
    L.rtp_profile_start.restype = i32
    L.rtp_profile_start.argtypes = [i32]
    L.rtp_profile_stop.restype = i32
    L.rtp_profile_stop.argtypes = [C.POINTER(rtp_launch_time), i32, C.POINTER(i32)]
    L.rtp_topp_select_noalloc.restype = i32
    L.rtp_topp_select_noalloc.argtypes = [vp, i64, vp, vp, i32, i64, vp, i64, vp, vp, vp, vp]
    L.rtp_topp_workspace_init.restype = i32
    L.rtp_topp_workspace_init.argtypes = [vp, sz, vp]
    L.rtp_sparse_attn_decode_workspace_bytes.restype = sz
    L.rtp_sparse_attn_decode_workspace_bytes.argtypes = [dp, i32, i64]
    L.rtp_sparse_attn_decode.restype = i32
    L.rtp_sparse_attn_decode.argtypes = [dp, vp, vp, vp, i64, i64, vp, vp, i64, vp, i64, i32, vp, vp, vp, sz, vp]
    L.rtp_sparse_attn_prefill_workspace_bytes.restype = sz
    L.rtp_sparse_attn_prefill_workspace_bytes.argtypes = [dp, i32, i64]
    L.rtp_sparse_attn_prefill_tile_stats.restype = i32
    L.rtp_sparse_attn_prefill_tile_stats.argtypes = [dp, i32, i64, vp, sz, vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    L.rtp_sparse_attn_prefill.restype = i32
    L.rtp_sparse_attn_prefill.argtypes = [dp, vp, vp, vp, vp, i64, vp, vp, i64, i64, i64, i32, C.c_float,
                                          vp, vp, vp, vp, vp, vp, sz, vp]
    for name in ("rtp_local_attn", "rtp_dense_attn"):
        getattr(L, name + "_workspace_bytes").restype = sz
        getattr(L, name + "_workspace_bytes").argtypes = [dp, i32, i32, i64]
        getattr(L, name).restype = i32
        getattr(L, name).argtypes = [dp, vp, vp, vp, i64, i64, vp, vp, vp, i32, i32, i64, vp, vp, vp, sz, vp]
    L.rtp_index_project.restype = i32
    L.rtp_index_project.argtypes = [dp, vp, vp, i32, i32, vp, i64, i64, vp]
    L.rtp_topk_select.restype = i32
    L.rtp_topk_select.argtypes = [vp, i64, vp, vp, i32, i64, vp, i64, vp, vp, vp, sz, vp]
    L.rtp_block_topp_workspace_bytes.restype = sz
    L.rtp_block_topp_workspace_bytes.argtypes = [i32, i64]
    L.rtp_block_topp_select.restype = i32
    L.rtp_block_topp_select.argtypes = [vp, i64, vp, vp, i32, i64, i32, C.c_float, C.c_float, vp, i64, vp, vp, vp,
                                        vp, i64, vp, sz, vp]
    L.rtp_select_attend_decode_workspace_bytes.restype = sz
    L.rtp_select_attend_decode_workspace_bytes.argtypes = [dp, i32, i64]
    L.rtp_select_attend_decode.restype = i32
    L.rtp_select_attend_decode.argtypes = [dp, vp, i64, vp, vp, i32, i64, vp, vp, vp, i64, i64, vp, vp, i64, vp, vp, vp,
                                           i32, vp, vp, vp, sz, vp, sz, vp]
    L.rtp_sparse_attn_decode_paged.restype = i32
    L.rtp_sparse_attn_decode_paged.argtypes = [dp, vp, vp, vp, i64, i64, vp, i64, i32, vp, i64, vp, i64, i32, vp, vp, vp, sz, vp]
    L.rtp_decode_attention.restype = i32
    L.rtp_decode_attention.argtypes = [dp, vp, i64, vp, vp, vp, i32, i64, vp, vp, vp, i64, i64, vp, vp, i64, vp, vp, vp,
                                       i32, vp, vp, vp, sz, vp, sz, vp, sz, vp]
    L.rtp_decode_attention_paged.restype = i32
    L.rtp_decode_attention_paged.argtypes = [dp, vp, i64, vp, vp, vp, i32, i64, vp, vp, vp, i64, i64, vp, i64, i32, vp, i64,
                                             vp, vp, vp, i32, vp, vp, vp, sz, vp, sz, vp, sz, vp]
    L.rtp_kv_ring_heads.restype = i32
    L.rtp_kv_ring_heads.argtypes = [dp, vp]
    L.rtp_kv_ring_append.restype = i32
    L.rtp_kv_ring_append.argtypes = [dp, vp, vp, vp, i32, vp, vp, i64, i64, vp, vp]
    L.rtp_kv_ring_fill.restype = i32
    L.rtp_kv_ring_fill.argtypes = [dp, vp, vp, i64, i64, vp, vp, i32, vp, vp, i64, i64, vp, vp]
    L.rtp_local_attn_ring_workspace_bytes.restype = sz
    L.rtp_local_attn_ring_workspace_bytes.argtypes = [dp, i32, i64]
    L.rtp_local_attn_ring.restype = i32
    L.rtp_local_attn_ring.argtypes = [dp, vp, vp, vp, i64, i64, vp, vp, vp, i64, i64, vp, vp, i32, i64, vp, vp, vp, sz, vp]
    cp = C.POINTER(rtp_kv4_cache)
    L.rtp_kv4_append.restype = i32
    L.rtp_kv4_append.argtypes = [dp, cp, vp, vp, i64, i64, i64, vp, vp, i32, i32, vp]
    L.rtp_kv4_read.restype = i32
    L.rtp_kv4_read.argtypes = [dp, cp, vp, vp, i32, i32, vp, vp, i64, i64, i64, vp]
    L.rtp_sparse_attn_decode_kv4_workspace_bytes.restype = sz
    L.rtp_sparse_attn_decode_kv4_workspace_bytes.argtypes = [dp, i32, i64]
    L.rtp_sparse_attn_decode_kv4.restype = i32
    L.rtp_sparse_attn_decode_kv4.argtypes = [dp, vp, cp, vp, i64, vp, i64, i32, vp, vp, vp, sz, vp]
    for name in ("rtp_local_attn_kv4", "rtp_dense_attn_kv4"):
        getattr(L, name + "_workspace_bytes").restype = sz
        getattr(L, name + "_workspace_bytes").argtypes = [dp, i32, i64]
        getattr(L, name).restype = i32
        getattr(L, name).argtypes = [dp, vp, cp, vp, i32, i64, vp, vp, vp, sz, vp]
    kp, chp, rp = C.POINTER(rtp_kv_cache), C.POINTER(rtp_chunk), C.POINTER(rtp_rope)
    L.rtp_kv_append.restype = i32
    L.rtp_kv_append.argtypes = [dp, kp, chp, rp, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    L.rtp_dense_attn_chunk_workspace_bytes.restype = sz
    L.rtp_dense_attn_chunk_workspace_bytes.argtypes = [dp, i32, i32, i32, i64, i32]
    L.rtp_local_attn_chunk_workspace_bytes.restype = sz
    L.rtp_local_attn_chunk_workspace_bytes.argtypes = [dp, i32, i32, i32, i64]
    for suffix, ptr in (("", kp), ("_kv4", cp)):
        getattr(L, "rtp_dense_attn_chunk" + suffix).restype = i32
        getattr(L, "rtp_dense_attn_chunk" + suffix).argtypes = [dp, vp, i64, ptr, chp, i32, vp, vp, vp, sz, vp]
        getattr(L, "rtp_local_attn_chunk" + suffix).restype = i32
        getattr(L, "rtp_local_attn_chunk" + suffix).argtypes = [dp, vp, i64, ptr, chp, vp, vp, vp, sz, vp]
    mp = C.POINTER(rtp_page_map)
    L.rtp_kv_pages_workspace_bytes.restype = sz
    L.rtp_kv_pages_workspace_bytes.argtypes = [mp, i32]
    for name, args in (("init", [mp, vp]), ("extend", [mp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]),
                       ("fork", [mp, vp, vp, vp, i32, vp]), ("truncate", [mp, vp, vp, i32, vp]),
                       ("compact", [mp, vp, vp, vp, vp, sz, vp]),
                       ("copy", [C.POINTER(rtp_page_pool), i32, i32, vp, vp, i32, vp, vp])):
        getattr(L, "rtp_kv_pages_" + name).restype = i32
        getattr(L, "rtp_kv_pages_" + name).argtypes = args
    L.rtp_sparsity_stats.restype = i32
    L.rtp_sparsity_stats.argtypes = [dp, vp, vp, i64, vp, vp, vp, i32, vp, vp, vp]
    _lib = L
    return L


def _ptr(t) -> Optional[int]:
    return t if t is None or isinstance(t, int) else t.data_ptr()


_raw_stream = None


def _forget_raw_stream():
    global _raw_stream
    _raw_stream = None


os.register_at_fork(after_in_child=_forget_raw_stream)      # (torch refuses the device in a child: ask it again there)


def _stream(stream) -> Optional[int]:
    if stream is None:
        # torch's current stream as a bare handle: a Stream object per call costs more than the rest of the marshalling
        # (1.5 against 0.3 us; a call of one short kernel is bound by its host time)
        global _raw_stream
        if _raw_stream is None:
            import torch
            handle = torch.cuda.current_stream().cuda_stream     # (initialises the device, or raises where there is none)
            if not (hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice")):
                return handle                                    # (not part of torch's interface)
            _raw_stream = (torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)
        raw, device = _raw_stream
        return raw(device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _current_device() -> int:
    if _raw_stream is not None:
        return _raw_stream[1]()
    import torch
    return torch.cuda.current_device()


def _check(rc: int):
    if rc != 0:
        raise RtpError(rc, lib().rtp_last_error().decode())


def _nbytes(t) -> int:
    return 0 if t is None else t.nbytes


def rtp_version() -> str:
    return lib().rtp_version().decode()


def rtp_last_error() -> str:
    return lib().rtp_last_error().decode()


def rtp_index_score(layer, q_in, WQ, kI, kI_head_stride, seq_start, ctx_len, q_start, B, n_q, max_ctx,
                    scores, score_stride, qI_out=None, topp_ws=None, stream=None):
    _check(lib().rtp_index_score(C.byref(layer), _ptr(q_in), _ptr(WQ), _ptr(kI), kI_head_stride, _ptr(seq_start),
                                 _ptr(ctx_len), _ptr(q_start), B, n_q, max_ctx, _ptr(scores), score_stride,
                                 _ptr(qI_out), _ptr(topp_ws), _nbytes(topp_ws), _stream(stream)))


def rtp_topp_workspace_bytes(R, max_len) -> int:
    return lib().rtp_topp_workspace_bytes(R, max_len)


def rtp_topp_workspace_init(ws, stream=None):
    _check(lib().rtp_topp_workspace_init(_ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_topp_select(scores, score_stride, row_len, p, R, max_len, sel_idx, sel_stride, sel_count,
                    tau, mass, ws, level1_ready=0, stream=None):
    _check(lib().rtp_topp_select(_ptr(scores), score_stride, _ptr(row_len), _ptr(p), R, max_len, _ptr(sel_idx),
                                 sel_stride, _ptr(sel_count), _ptr(tau), _ptr(mass), level1_ready, _ptr(ws),
                                 _nbytes(ws), _stream(stream)))


def rtp_index_score_traffic_probe(layer, q_in, WQ, kI, kI_head_stride, seq_start, ctx_len, q_start, B, n_q, max_ctx,
                                  scores, score_stride, stream=None):
    _check(lib().rtp_index_score_traffic_probe(C.byref(layer), _ptr(q_in), _ptr(WQ), _ptr(kI), kI_head_stride,
                                               _ptr(seq_start), _ptr(ctx_len), _ptr(q_start), B, n_q, max_ctx,
                                               _ptr(scores), score_stride, _stream(stream)))


def rtp_profile_start(max_launches: int) -> None:
    _check(lib().rtp_profile_start(max_launches))


def rtp_profile_stop(max_launches: int = 1 << 16):
    """[(kernel name, microseconds)] of the launches recorded since rtp_profile_start, in launch order."""
    buf = (rtp_launch_time * max_launches)()
    n = C.c_int32(0)
    _check(lib().rtp_profile_stop(buf, max_launches, C.byref(n)))
    return [(buf[i].kernel.decode().strip("()"), float(buf[i].us)) for i in range(n.value)]


def rtp_topp_select_noalloc(scores, score_stride, row_len, p, R, max_len, sel_idx, sel_stride, sel_count,
                            tau, mass, stream=None):
    _check(lib().rtp_topp_select_noalloc(_ptr(scores), score_stride, _ptr(row_len), _ptr(p), R, max_len, _ptr(sel_idx),
                                         sel_stride, _ptr(sel_count), _ptr(tau), _ptr(mass), _stream(stream)))


def rtp_sparse_attn_decode_workspace_bytes(layer, B, max_sel) -> int:
    return lib().rtp_sparse_attn_decode_workspace_bytes(C.byref(layer), B, max_sel)


def rtp_sparse_attn_decode(layer, q, K, V, kv_row_stride, kv_head_stride, seq_start, sel_idx, sel_stride,
                           sel_count, max_sel, B, out, lse, ws, stream=None):
    _check(lib().rtp_sparse_attn_decode(C.byref(layer), _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                        _ptr(seq_start), _ptr(sel_idx), sel_stride, _ptr(sel_count), max_sel, B,
                                        _ptr(out), _ptr(lse), _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_select_attend_decode_workspace_bytes(layer, B, max_ctx) -> int:
    return lib().rtp_select_attend_decode_workspace_bytes(C.byref(layer), B, max_ctx)


def rtp_select_attend_decode(layer, scores, score_stride, row_len, p, B, max_ctx, q, K, V, kv_row_stride,
                             kv_head_stride, seq_start, sel_idx, sel_stride, sel_count, tau, mass, out, lse,
                             topp_ws, attn_ws, level1_ready=0, stream=None):
    _check(lib().rtp_select_attend_decode(C.byref(layer), _ptr(scores), score_stride, _ptr(row_len), _ptr(p), B,
                                          max_ctx, _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                          _ptr(seq_start), _ptr(sel_idx), sel_stride, _ptr(sel_count), _ptr(tau),
                                          _ptr(mass), level1_ready, _ptr(out), _ptr(lse), _ptr(topp_ws),
                                          _nbytes(topp_ws), _ptr(attn_ws), _nbytes(attn_ws), _stream(stream)))


def rtp_sparse_attn_decode_paged(layer, q, K, V, kv_row_stride, kv_head_stride, page_table, pt_stride, page_size,
                                 sel_idx, sel_stride, sel_count, max_sel, B, out, lse, ws, stream=None):
    _check(lib().rtp_sparse_attn_decode_paged(C.byref(layer), _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                              _ptr(page_table), pt_stride, page_size, _ptr(sel_idx), sel_stride,
                                              _ptr(sel_count), max_sel, B, _ptr(out), _ptr(lse), _ptr(ws), _nbytes(ws),
                                              _stream(stream)))


def rtp_decode_attention_paged(layer, scores, score_stride, row_len, p, ctx_len, B, max_ctx, q, K, V, kv_row_stride,
                               kv_head_stride, page_table, pt_stride, page_size, sel_idx, sel_stride, sel_count, tau, mass,
                               out, lse, topp_ws, attn_ws, local_ws, level1_ready=0, stream=None):
    _check(lib().rtp_decode_attention_paged(C.byref(layer), _ptr(scores), score_stride, _ptr(row_len), _ptr(p),
                                            _ptr(ctx_len), B, max_ctx, _ptr(q), _ptr(K), _ptr(V), kv_row_stride,
                                            kv_head_stride, _ptr(page_table), pt_stride, page_size, _ptr(sel_idx),
                                            sel_stride, _ptr(sel_count), _ptr(tau), _ptr(mass), level1_ready, _ptr(out),
                                            _ptr(lse), _ptr(topp_ws), _nbytes(topp_ws), _ptr(attn_ws), _nbytes(attn_ws),
                                            _ptr(local_ws), _nbytes(local_ws), _stream(stream)))


def rtp_decode_attention(layer, scores, score_stride, row_len, p, ctx_len, B, max_ctx, q, K, V, kv_row_stride,
                         kv_head_stride, seq_start, sel_idx, sel_stride, sel_count, tau, mass, out, lse,
                         topp_ws, attn_ws, local_ws, level1_ready=0, stream=None):
    _check(lib().rtp_decode_attention(C.byref(layer), _ptr(scores), score_stride, _ptr(row_len), _ptr(p), _ptr(ctx_len),
                                      B, max_ctx, _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                      _ptr(seq_start), _ptr(sel_idx), sel_stride, _ptr(sel_count), _ptr(tau), _ptr(mass),
                                      level1_ready, _ptr(out), _ptr(lse), _ptr(topp_ws), _nbytes(topp_ws), _ptr(attn_ws),
                                      _nbytes(attn_ws), _ptr(local_ws), _nbytes(local_ws), _stream(stream)))


def rtp_kv_ring_heads(layer) -> list:
    """The KV heads whose query heads are all local (they may live in the bounded cache), ascending."""
    buf = (C.c_int32 * max(1, layer.n_kv_heads))()
    n = lib().rtp_kv_ring_heads(C.byref(layer), buf)
    if n < 0:
        raise RtpError(RTP_ERR_INVALID_ARG, lib().rtp_last_error().decode())
    return [int(buf[i]) for i in range(n)]


def rtp_kv_ring_append(layer, k_new, v_new, pos, B, ring_K, ring_V, ring_row_stride, ring_head_stride, ring_seq_start,
                       stream=None):
    _check(lib().rtp_kv_ring_append(C.byref(layer), _ptr(k_new), _ptr(v_new), _ptr(pos), B, _ptr(ring_K), _ptr(ring_V),
                                    ring_row_stride, ring_head_stride, _ptr(ring_seq_start), _stream(stream)))


def rtp_kv_ring_fill(layer, K, V, kv_row_stride, kv_head_stride, seq_start, ctx_len, B, ring_K, ring_V,
                     ring_row_stride, ring_head_stride, ring_seq_start, stream=None):
    _check(lib().rtp_kv_ring_fill(C.byref(layer), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride, _ptr(seq_start),
                                  _ptr(ctx_len), B, _ptr(ring_K), _ptr(ring_V), ring_row_stride, ring_head_stride,
                                  _ptr(ring_seq_start), _stream(stream)))


def rtp_local_attn_ring_workspace_bytes(layer, B, max_ctx) -> int:
    return lib().rtp_local_attn_ring_workspace_bytes(C.byref(layer), B, max_ctx)


def rtp_local_attn_ring(layer, q, K, V, kv_row_stride, kv_head_stride, seq_start, ring_K, ring_V, ring_row_stride,
                        ring_head_stride, ring_seq_start, ctx_len, B, max_ctx, out, lse, ws, stream=None):
    _check(lib().rtp_local_attn_ring(C.byref(layer), _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                     _ptr(seq_start), _ptr(ring_K), _ptr(ring_V), ring_row_stride, ring_head_stride,
                                     _ptr(ring_seq_start), _ptr(ctx_len), B, max_ctx, _ptr(out), _ptr(lse), _ptr(ws),
                                     _nbytes(ws), _stream(stream)))


def rtp_sparse_attn_prefill_workspace_bytes(layer, T, chunk_start) -> int:
    return lib().rtp_sparse_attn_prefill_workspace_bytes(C.byref(layer), T, chunk_start)


def rtp_sparse_attn_prefill(layer, q_pre, q, WQ, kI, kI_head_stride, K, V, kv_row_stride, kv_head_stride,
                            chunk_start, T, p, out, lse, tau, count, mass, ws, stream=None):
    _check(lib().rtp_sparse_attn_prefill(C.byref(layer), _ptr(q_pre), _ptr(q), _ptr(WQ), _ptr(kI), kI_head_stride,
                                         _ptr(K), _ptr(V), kv_row_stride, kv_head_stride, chunk_start, T, p,
                                         _ptr(out), _ptr(lse), _ptr(tau), _ptr(count), _ptr(mass), _ptr(ws),
                                         _nbytes(ws), _stream(stream)))


def rtp_sparse_attn_prefill_tile_stats(layer, T, chunk_start, ws, stream=None):
    """(tiles_visited, tiles_causal) of the last p < 1 call on this workspace."""
    vis, causal = C.c_int64(0), C.c_int64(0)
    _check(lib().rtp_sparse_attn_prefill_tile_stats(C.byref(layer), T, chunk_start, _ptr(ws), _nbytes(ws), _stream(stream),
                                                    C.byref(vis), C.byref(causal)))
    return vis.value, causal.value


def rtp_local_attn_workspace_bytes(layer, B, n_q, max_ctx) -> int:
    return lib().rtp_local_attn_workspace_bytes(C.byref(layer), B, n_q, max_ctx)


def rtp_dense_attn_workspace_bytes(layer, B, n_q, max_ctx) -> int:
    return lib().rtp_dense_attn_workspace_bytes(C.byref(layer), B, n_q, max_ctx)


def rtp_local_attn(layer, q, K, V, kv_row_stride, kv_head_stride, seq_start, ctx_len, q_start, B, n_q, max_ctx,
                   out, lse, ws, stream=None):
    _check(lib().rtp_local_attn(C.byref(layer), _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                _ptr(seq_start), _ptr(ctx_len), _ptr(q_start), B, n_q, max_ctx, _ptr(out), _ptr(lse),
                                _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_dense_attn(layer, q, K, V, kv_row_stride, kv_head_stride, seq_start, ctx_len, q_start, B, n_q, max_ctx,
                   out, lse, ws, stream=None):
    _check(lib().rtp_dense_attn(C.byref(layer), _ptr(q), _ptr(K), _ptr(V), kv_row_stride, kv_head_stride,
                                _ptr(seq_start), _ptr(ctx_len), _ptr(q_start), B, n_q, max_ctx, _ptr(out), _ptr(lse),
                                _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_index_project(layer, W, x_pre, side, T, xI_out, out_head_stride, out_t0=0, stream=None):
    _check(lib().rtp_index_project(C.byref(layer), _ptr(W), _ptr(x_pre), side, T, _ptr(xI_out), out_head_stride,
                                   out_t0, _stream(stream)))


def rtp_topk_select(scores, score_stride, row_len, k, R, max_len, sel_idx, sel_stride, sel_count, tau, ws,
                    stream=None):
    _check(lib().rtp_topk_select(_ptr(scores), score_stride, _ptr(row_len), _ptr(k), R, max_len, _ptr(sel_idx),
                                 sel_stride, _ptr(sel_count), _ptr(tau), _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_block_topp_workspace_bytes(R, max_len) -> int:
    return lib().rtp_block_topp_workspace_bytes(R, max_len)


def rtp_block_topp_select(scores, score_stride, row_len, p, R, max_len, block, bin_lo, bin_width, sel_idx,
                          sel_stride, sel_count, threshold_bin, mass, block_mask, mask_stride, ws, stream=None):
    _check(lib().rtp_block_topp_select(_ptr(scores), score_stride, _ptr(row_len), _ptr(p), R, max_len, block,
                                       bin_lo, bin_width, _ptr(sel_idx), sel_stride, _ptr(sel_count),
                                       _ptr(threshold_bin), _ptr(mass), _ptr(block_mask), mask_stride,
                                       _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_sparsity_stats(layer, ctx_len, sel_idx, sel_stride, sel_count, lse_selected, lse_full, B, stats,
                       union_size=None, stream=None):
    _check(lib().rtp_sparsity_stats(C.byref(layer), _ptr(ctx_len), _ptr(sel_idx), sel_stride, _ptr(sel_count),
                                    _ptr(lse_selected), _ptr(lse_full), B, _ptr(stats), _ptr(union_size),
                                    _stream(stream)))


def rtp_kv4_append(layer, cache, k, v, batch_stride, token_stride, head_stride, start, count, B, T, stream=None):
    _held("rtp_kv4_append", layer, cache, B)
    _check(lib().rtp_kv4_append(C.byref(layer), C.byref(cache), _ptr(k), _ptr(v), batch_stride, token_stride, head_stride,
                                _ptr(start), _ptr(count), B, T, _stream(stream)))


def rtp_kv4_read(layer, cache, start, count, B, T, k, v, batch_stride, token_stride, head_stride, stream=None):
    _held("rtp_kv4_read", layer, cache, B)
    _check(lib().rtp_kv4_read(C.byref(layer), C.byref(cache), _ptr(start), _ptr(count), B, T, _ptr(k), _ptr(v), batch_stride,
                              token_stride, head_stride, _stream(stream)))


def rtp_sparse_attn_decode_kv4_workspace_bytes(layer, B, max_sel) -> int:
    return lib().rtp_sparse_attn_decode_kv4_workspace_bytes(C.byref(layer), B, max_sel)


def rtp_sparse_attn_decode_kv4(layer, q, cache, sel_idx, sel_stride, sel_count, max_sel, B, out, lse, ws, stream=None):
    _held("rtp_sparse_attn_decode_kv4", layer, cache, B)
    _check(lib().rtp_sparse_attn_decode_kv4(C.byref(layer), _ptr(q), C.byref(cache), _ptr(sel_idx), sel_stride, _ptr(sel_count),
                                            max_sel, B, _ptr(out), _ptr(lse), _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_local_attn_kv4_workspace_bytes(layer, B, max_ctx) -> int:
    return lib().rtp_local_attn_kv4_workspace_bytes(C.byref(layer), B, max_ctx)


def rtp_local_attn_kv4(layer, q, cache, ctx_len, B, max_ctx, out, lse, ws, stream=None):
    _held("rtp_local_attn_kv4", layer, cache, B)
    _check(lib().rtp_local_attn_kv4(C.byref(layer), _ptr(q), C.byref(cache), _ptr(ctx_len), B, max_ctx, _ptr(out), _ptr(lse),
                                    _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_dense_attn_kv4_workspace_bytes(layer, B, max_ctx) -> int:
    return lib().rtp_dense_attn_kv4_workspace_bytes(C.byref(layer), B, max_ctx)


def rtp_dense_attn_kv4(layer, q, cache, ctx_len, B, max_ctx, out, lse, ws, stream=None):
    _held("rtp_dense_attn_kv4", layer, cache, B)
    _check(lib().rtp_dense_attn_kv4(C.byref(layer), _ptr(q), C.byref(cache), _ptr(ctx_len), B, max_ctx, _ptr(out), _ptr(lse),
                                    _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_kv_pages_workspace_bytes(map, n) -> int:
    return lib().rtp_kv_pages_workspace_bytes(C.byref(map), n)


def rtp_kv_pages_init(map, stream=None):
    _check(lib().rtp_kv_pages_init(C.byref(map), _stream(stream)))


def rtp_kv_pages_extend(map, seq, old_len, new_len, n, copy_src, copy_dst, status, ws, stream=None):
    _check(lib().rtp_kv_pages_extend(C.byref(map), _ptr(seq), _ptr(old_len), _ptr(new_len), n, _ptr(copy_src), _ptr(copy_dst),
                                     _ptr(status), _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_kv_pages_fork(map, src_seq, dst_seq, len, n, stream=None):
    _check(lib().rtp_kv_pages_fork(C.byref(map), _ptr(src_seq), _ptr(dst_seq), _ptr(len), n, _stream(stream)))


def rtp_kv_pages_truncate(map, seq, keep_len, n, stream=None):
    _check(lib().rtp_kv_pages_truncate(C.byref(map), _ptr(seq), _ptr(keep_len), n, _stream(stream)))


def rtp_kv_pages_compact(map, move_src, move_dst, status, ws, stream=None):
    _check(lib().rtp_kv_pages_compact(C.byref(map), _ptr(move_src), _ptr(move_dst), _ptr(status), _ptr(ws), _nbytes(ws),
                                      _stream(stream)))


def rtp_kv_pages_copy(pools, n_pages, src, dst, n, count=None, stream=None):
    """pools: what page_pools returned; n_pages: at most what its tensors have."""
    if n_pages > pools.n_pages:
        raise RtpError(RTP_ERR_INVALID_ARG, f"rtp_kv_pages_copy: n_pages = {n_pages}, the pools have {pools.n_pages}")
    _check(lib().rtp_kv_pages_copy(pools, pools.n_pools, n_pages, _ptr(src), _ptr(dst), n, _ptr(count), _stream(stream)))


# (The calls below hand ctypes the structs themselves, which costs a third less than references made for it.  A call of rtp_kv_append takes 8.4 us of
# host time with checks that look up what they need several times, 7.3 with these.)
def rtp_kv_append(layer, cache, chunk, rope, q, q_stride, k, k_stride, v, v_stride, q_out, q_out_stride, stream=None):
    who, total, n_q, n_kv = "rtp_kv_append", chunk.total_q, layer.n_q_heads, layer.n_kv_heads
    _held(who, layer, cache, chunk.B)
    kind = _type_of(who, layer, cache)
    _on_one_device(who, (cache, chunk, rope), (q, k, v, q_out))
    _check(lib().rtp_kv_append(layer, cache, chunk, rope, _rows(who, q, total, n_q, "q", q_stride, kind), q_stride,
                               _rows(who, k, total, n_kv, "k", k_stride, kind), k_stride, _rows(who, v, total, n_kv, "v", v_stride, kind), v_stride,
                               _rows(who, q_out, total, n_q, "q_out", q_out_stride, kind), q_out_stride, _stream(stream)))


def rtp_dense_attn_chunk_workspace_bytes(layer, B, total_q, max_q, max_ctx, heads) -> int:
    return lib().rtp_dense_attn_chunk_workspace_bytes(C.byref(layer), B, total_q, max_q, max_ctx, heads)


def rtp_local_attn_chunk_workspace_bytes(layer, B, total_q, max_q, max_ctx) -> int:
    return lib().rtp_local_attn_chunk_workspace_bytes(C.byref(layer), B, total_q, max_q, max_ctx)


def _chunk_attn(who, layer, q, q_stride, cache, chunk, heads, out, lse, ws, stream):
    total, n_q = chunk.total_q, layer.n_q_heads
    _held(who, layer, cache, chunk.B)
    kind = _type_of(who, layer, cache)
    _on_one_device(who, (cache, chunk), (q, out, lse, ws))
    q, out = _rows(who, q, total, n_q, "q", q_stride, kind), _rows(who, out, total, n_q, "out", n_q * 128, kind)
    if lse is not None and lse.__class__ is not int and (lse.numel() < total * n_q or lse.element_size() != 4 or not lse.is_contiguous()
                                                         or lse.dtype is not _torch_types["lse"]):
        raise RtpError(RTP_ERR_INVALID_ARG, f"{who}: contiguous fp32 lse [{total}, {n_q}] expected")
    _check(getattr(lib(), who)(layer, q, q_stride, cache, chunk, *heads, out, _ptr(lse), _ptr(ws), _nbytes(ws), _stream(stream)))


def rtp_dense_attn_chunk(layer, q, q_stride, cache, chunk, heads, out, lse, ws, stream=None):
    _chunk_attn("rtp_dense_attn_chunk", layer, q, q_stride, cache, chunk, (heads,), out, lse, ws, stream)


def rtp_dense_attn_chunk_kv4(layer, q, q_stride, cache, chunk, heads, out, lse, ws, stream=None):
    _chunk_attn("rtp_dense_attn_chunk_kv4", layer, q, q_stride, cache, chunk, (heads,), out, lse, ws, stream)


def rtp_local_attn_chunk(layer, q, q_stride, cache, chunk, out, lse, ws, stream=None):
    _chunk_attn("rtp_local_attn_chunk", layer, q, q_stride, cache, chunk, (), out, lse, ws, stream)


def rtp_local_attn_chunk_kv4(layer, q, q_stride, cache, chunk, out, lse, ws, stream=None):
    _chunk_attn("rtp_local_attn_chunk_kv4", layer, q, q_stride, cache, chunk, (), out, lse, ws, stream)
