"""Paged keys and values: the write of new tokens, their attention, and the
eviction by accumulated attention weight.

    ptc_kv_append(k_new, v_new, k, v, page_ids, page_off, tok_off, kv_len)
    out, lse       = ptc_paged_attention(q, k, v, page_ids, page_off, tok_off, kv_len, max_q_len)
    out, lse, mass = ptc_paged_attention(..., mass=mass)
    keep, new_len, new_mass = ptc_kv_evict(k, v, page_ids, page_off, kv_len, mass, dst_page_ids, dst_page_off,
                                           n_keep, n_sink, n_recent, max_kv_len)

``k`` and ``v`` are bfloat16 or float16 CUDA tensors of shape [pages, key heads,
block_size, head_dim] with any strides that are multiples of 8 and a contiguous
last dimension (a cache whose pages hold tokens outermost is passed
transposed).  ``page_ids`` (int32 bits) and ``page_off`` (int64) are the ids of
ptc_assign_ids and the offsets of ptc_hash_blocks, or any other page lists.

With ``status`` (an int32 CUDA tensor of one zero) a call returns without
waiting, for loops over layers and for graph capture; check_status(status)
waits and raises what went wrong.  Without it a call waits and raises itself.
"""
from __future__ import annotations

import ctypes
import math

import torch

PTC_DTYPE_BF16, PTC_DTYPE_FP16 = 0, 1
MAX_HEAD_DIM = 128
_DTYPES = {torch.bfloat16: PTC_DTYPE_BF16, torch.float16: PTC_DTYPE_FP16}


class PagedKv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("page_ids", ctypes.c_void_p), ("page_off", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("n_page_ids", ctypes.c_uint64), ("n_pages", ctypes.c_uint32),
                ("n_req", ctypes.c_uint32), ("block_size", ctypes.c_uint32), ("n_kv_heads", ctypes.c_uint32),
                ("head_dim", ctypes.c_uint32), ("dtype", ctypes.c_int32)]


_Strides = ctypes.c_int64 * 2


def declare(L) -> None:
    """The argument types of the library's calls on paged keys and values."""
    vp, u32, u64, sz, st = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    kv = ctypes.POINTER(PagedKv)
    L.ptc_kv_append_workspace_bytes.restype = sz
    L.ptc_kv_append_workspace_bytes.argtypes = [u32]
    L.ptc_kv_append.restype = st
    L.ptc_kv_append.argtypes = [kv, vp, vp, _Strides, _Strides, vp, u64, vp, sz, vp, vp]
    L.ptc_paged_attention_workspace_bytes.restype = sz
    L.ptc_paged_attention_workspace_bytes.argtypes = [u32, u32, u32, u32, u32, u64]
    L.ptc_paged_attention.restype = st
    L.ptc_paged_attention.argtypes = [kv, vp, _Strides, vp, u64, u32, u32, ctypes.c_float, vp, vp, vp, vp, u64, vp, sz,
                                      vp, vp]
    L.ptc_kv_evict_workspace_bytes.restype = sz
    L.ptc_kv_evict_workspace_bytes.argtypes = [u32, u32, u32]
    L.ptc_kv_evict.restype = st
    L.ptc_kv_evict.argtypes = [kv, vp, u64, u32, u32, u32, u32, vp, vp, u64, vp, vp, vp, u64, vp, sz, vp, vp]


def _pkg():
    import paper_2609_28870_gb300 as ptc
    return ptc


def _want(t: torch.Tensor, dtype, name: str, dev, dims: int = 1) -> None:
    if t.dtype != dtype or t.dim() != dims or t.device != dev:
        raise ValueError(f"{name}: expected a {dims}-dimensional {dtype} tensor on {dev}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")


def _paged(k, v, page_ids, page_off, kv_len) -> PagedKv:
    dev = _pkg()._dev(k)
    if k.dtype not in _DTYPES or v.dtype != k.dtype or k.dim() != 4 or v.shape != k.shape or v.device != dev:
        raise ValueError("k and v: expected bfloat16 or float16 tensors [pages, key heads, block_size, head_dim] of one shape")
    if k.shape[3] != 1 and (k.stride(3) != 1 or v.stride(3) != 1):
        raise ValueError("k and v: expected a contiguous last dimension")
    _want(page_ids, torch.int32, "page_ids", dev)
    _want(page_off, torch.int64, "page_off", dev)
    _want(kv_len, torch.int32, "kv_len", dev)
    if page_off.numel() != kv_len.numel() + 1:
        raise ValueError("page_off: expected one entry more than kv_len")
    ks, vs, shape = k.stride(), v.stride(), k.shape
    return PagedKv(k.data_ptr(), v.data_ptr(), (ks[0], ks[1], ks[2]), (vs[0], vs[1], vs[2]), page_ids.data_ptr(),
                   page_off.data_ptr(), kv_len.data_ptr(), page_ids.numel(), shape[0], kv_len.numel(), shape[2],
                   shape[1], shape[3], _DTYPES[k.dtype])


def _tokens(x, name: str, k, tok_off, heads: int | None = None):
    if x.dtype != k.dtype or x.dim() != 3 or x.shape[2] != k.shape[3] or x.device != k.device or (
            heads is not None and x.shape[1] != heads):
        raise ValueError(f"{name}: expected a {k.dtype} tensor [tokens, heads, {k.shape[3]}] on {k.device}")
    if x.stride(2) != 1:
        raise ValueError(f"{name}: expected a contiguous last dimension")
    return _Strides(x.stride(0), x.stride(1))


def _off(tok_off, kv_len) -> None:
    _want(tok_off, torch.int64, "tok_off", kv_len.device)
    if tok_off.numel() != kv_len.numel() + 1:
        raise ValueError("tok_off: expected one entry more than kv_len")


def _status(status, dev):
    if status is None:
        return None
    if status.dtype != torch.int32 or status.numel() != 1 or status.device != dev:
        raise ValueError("status: expected one int32 on the cache's device")
    return status.data_ptr()


def check_status(status: torch.Tensor, call: str = "ptc") -> None:
    """Waits for the calls that were given ``status`` and raises PtcError if
    one of them failed (and clears the word)."""
    code = int(status.item())
    if code:
        status.zero_()
        raise _pkg().PtcError(call, code)


def ptc_kv_append(k_new, v_new, k, v, page_ids, page_off, tok_off, kv_len, ws: torch.Tensor | None = None,
                  status: torch.Tensor | None = None) -> None:
    """Writes the new tokens' keys and values ([tokens, key heads, head_dim])
    into their requests' pages, as the last tokens of kv_len."""
    p = _pkg()
    kv = _paged(k, v, page_ids, page_off, kv_len)
    _off(tok_off, kv_len)
    ks, vs = _tokens(k_new, "k_new", k, tok_off, k.shape[1]), _tokens(v_new, "v_new", k, tok_off, k.shape[1])
    if v_new.shape != k_new.shape:
        raise ValueError("v_new: expected k_new's shape")
    L = p.lib()
    w = p._workspace(L.ptc_kv_append_workspace_bytes(kv.n_req), k.device, ws)
    rc = L.ptc_kv_append(ctypes.byref(kv), k_new.data_ptr(), v_new.data_ptr(), ks, vs, tok_off.data_ptr(),
                         k_new.shape[0], w.data_ptr(), w.numel(), _status(status, k.device), p._stream(k.device))
    p._check("ptc_kv_append", rc)


def ptc_paged_attention(q, k, v, page_ids, page_off, tok_off, kv_len, max_q_len: int, scale: float | None = None,
                        mass: torch.Tensor | None = None, mass_out: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                        ws: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """Causal attention of new tokens ``q`` [tokens, query heads, head_dim] over
    their requests' pages.  Returns (out, lse), with ``mass`` (the weights
    accumulated so far, float32 [key heads, slots]) or ``mass_out`` (where the
    new sums go; may be ``mass`` itself) also the accumulated weights.  ``scale``
    defaults to head_dim ** -0.5."""
    p = _pkg()
    kv = _paged(k, v, page_ids, page_off, kv_len)
    _off(tok_off, kv_len)
    qs = _tokens(q, "q", k, tok_off)
    dev, T, Hq = k.device, q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty((T, Hq, kv.head_dim), dtype=q.dtype, device=dev)
    elif out.shape != q.shape:
        raise ValueError("out: expected q's shape")
    if lse is None:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    elif lse.shape != q.shape[:2]:
        raise ValueError("lse: expected q's first two dimensions")
    _want(out, q.dtype, "out", dev, 3)
    _want(lse, torch.float32, "lse", dev, 2)
    stride = 0
    if mass is not None or mass_out is not None:
        if mass_out is None:
            mass_out = torch.empty_like(mass)
        _want(mass_out, torch.float32, "mass_out", dev, 2)
        if mass is not None:
            _want(mass, torch.float32, "mass", dev, 2)
            if mass.shape != mass_out.shape:
                raise ValueError("mass: expected mass_out's shape")
        if mass_out.shape[0] != kv.n_kv_heads:
            raise ValueError("mass: expected one row a key head")
        stride = mass_out.shape[1]
    L = p.lib()
    need = L.ptc_paged_attention_workspace_bytes(kv.n_req, Hq, kv.n_kv_heads, kv.head_dim, int(max_q_len), stride)
    w = p._workspace(need, dev, ws)
    rc = L.ptc_paged_attention(ctypes.byref(kv), q.data_ptr(), qs, tok_off.data_ptr(), T, Hq, int(max_q_len),
                               1 / math.sqrt(kv.head_dim) if scale is None else float(scale), out.data_ptr(),
                               lse.data_ptr(), p._ptr(mass), p._ptr(mass_out), stride, w.data_ptr(), w.numel(),
                               _status(status, dev), p._stream(dev))
    p._check("ptc_paged_attention", rc)
    return (out, lse) if mass_out is None else (out, lse, mass_out)


def ptc_kv_evict(k, v, page_ids, page_off, kv_len, mass, dst_page_ids, dst_page_off, n_keep: int, n_sink: int,
                 n_recent: int, max_kv_len: int, ws: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """Cuts every request to n_keep tokens a key head (the first n_sink, the
    last n_recent and the heaviest others) and moves them to the destination
    pages.  Returns (keep int32 [requests, key heads, n_keep], new_len int32,
    new_mass float32 [key heads, destination slots])."""
    p = _pkg()
    kv = _paged(k, v, page_ids, page_off, kv_len)
    dev = k.device
    _want(mass, torch.float32, "mass", dev, 2)
    _want(dst_page_ids, torch.int32, "dst_page_ids", dev)
    _want(dst_page_off, torch.int64, "dst_page_off", dev)
    if dst_page_off.numel() != kv_len.numel() + 1:
        raise ValueError("dst_page_off: expected one entry more than kv_len")
    if mass.shape[0] != kv.n_kv_heads:
        raise ValueError("mass: expected one row a key head")
    if min(n_keep, n_sink, n_recent, max_kv_len) < 0:
        raise ValueError("n_keep, n_sink, n_recent and max_kv_len: expected no negative numbers")
    keep = torch.empty((kv.n_req, kv.n_kv_heads, n_keep), dtype=torch.int32, device=dev)
    new_len = torch.empty(kv.n_req, dtype=torch.int32, device=dev)
    slots = dst_page_ids.numel() * kv.block_size
    new_mass = torch.empty((kv.n_kv_heads, slots), dtype=torch.float32, device=dev)
    L = p.lib()
    w = p._workspace(L.ptc_kv_evict_workspace_bytes(kv.n_req, kv.n_kv_heads, max_kv_len), dev, ws)
    rc = L.ptc_kv_evict(ctypes.byref(kv), mass.data_ptr(), mass.shape[1], n_keep, n_sink, n_recent, max_kv_len,
                        dst_page_ids.data_ptr(), dst_page_off.data_ptr(), dst_page_ids.numel(), keep.data_ptr(),
                        new_len.data_ptr(), new_mass.data_ptr(), slots, w.data_ptr(), w.numel(),
                        _status(status, dev), p._stream(dev))
    p._check("ptc_kv_evict", rc)
    return keep, new_len, new_mass
