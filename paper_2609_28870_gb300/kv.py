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

The calls have no backward pass: inputs that ask for gradients are refused,
unless under torch.no_grad().
"""
from __future__ import annotations

import ctypes
import struct
import sys

import torch

PTC_DTYPE_BF16, PTC_DTYPE_FP16 = 0, 1
MAX_HEAD_DIM, MAX_GROUP = 128, 128
_U32 = 0xFFFFFFFF
_DTYPES = {torch.bfloat16: PTC_DTYPE_BF16, torch.float16: PTC_DTYPE_FP16}

# ptc_paged_kv and two strides, as the C compiler lays them out.  A decode step
# makes one of these calls a layer, so the calls are marshalled in as few steps
# as Python allows.
PAGED_KV = struct.Struct("@PP6qPPPQ5Ii")
_STRIDES = struct.Struct("@2q")


def declare(L) -> None:
    """The argument types of the library's calls on paged keys and values."""
    vp, u32, u64, sz, st = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    packed = ctypes.c_char_p
    L.ptc_kv_append_workspace_bytes.restype = sz
    L.ptc_kv_append_workspace_bytes.argtypes = [u32]
    L.ptc_kv_append.restype = st
    L.ptc_kv_append.argtypes = [packed, vp, vp, packed, packed, vp, u64, vp, sz, vp, vp]
    L.ptc_paged_attention_workspace_bytes.restype = sz
    L.ptc_paged_attention_workspace_bytes.argtypes = [u32, u32, u32, u32, u32, u64]
    L.ptc_paged_attention.restype = st
    L.ptc_paged_attention.argtypes = [packed, vp, packed, vp, u64, u32, u32, ctypes.c_float, vp, vp, vp, vp, u64, vp, sz,
                                      vp, vp]
    L.ptc_kv_evict_workspace_bytes.restype = sz
    L.ptc_kv_evict_workspace_bytes.argtypes = [u32, u32, u32]
    L.ptc_kv_evict.restype = st
    L.ptc_kv_evict.argtypes = [packed, vp, u64, u32, u32, u32, u32, vp, vp, u64, vp, vp, vp, u64, vp, sz, vp, vp]


def _pkg():
    return sys.modules[__package__]


def _want(t: torch.Tensor, dtype, name: str, dev: int, dims: int = 1) -> None:
    if t.dtype is not dtype or t.dim() != dims or t.get_device() != dev:
        raise ValueError(f"{name}: expected a {dims}-dimensional {dtype} tensor on cuda:{dev}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")


def _paged(k, v, page_ids, page_off, kv_len, shape, dev: int) -> bytes:
    """The packed ptc_paged_kv; shape is k's, dev its device's index."""
    if dev < 0:
        raise ValueError("expected a CUDA tensor")
    if k.dtype not in _DTYPES or v.dtype is not k.dtype or len(shape) != 4 or v.shape != shape or v.get_device() != dev:
        raise ValueError("k and v: expected bfloat16 or float16 tensors [pages, key heads, block_size, head_dim] of one shape")
    k0, k1, k2, k3 = k.stride()
    v0, v1, v2, v3 = v.stride()
    if shape[3] != 1 and (k3 != 1 or v3 != 1):
        raise ValueError("k and v: expected a contiguous last dimension")
    _want(page_ids, torch.int32, "page_ids", dev)
    _want(page_off, torch.int64, "page_off", dev)
    _want(kv_len, torch.int32, "kv_len", dev)
    n_req = kv_len.shape[0]
    if page_off.shape[0] != n_req + 1:
        raise ValueError("page_off: expected one entry more than kv_len")
    return PAGED_KV.pack(k.data_ptr(), v.data_ptr(), k0, k1, k2, v0, v1, v2, page_ids.data_ptr(), page_off.data_ptr(),
                         kv_len.data_ptr(), page_ids.shape[0], shape[0], n_req, shape[2], shape[1], shape[3],
                         _DTYPES[k.dtype])


def _tokens(x, name: str, k, dev: int, head_dim: int, heads: int | None = None) -> bytes:
    shape = x.shape
    if x.dtype is not k.dtype or len(shape) != 3 or shape[2] != head_dim or x.get_device() != dev or (
            heads is not None and shape[1] != heads):
        raise ValueError(f"{name}: expected a {k.dtype} tensor [tokens, heads, {head_dim}] on cuda:{dev}")
    a, b, c = x.stride()
    if c != 1:
        raise ValueError(f"{name}: expected a contiguous last dimension")
    return _STRIDES.pack(a, b)


def _no_backward(*tensors) -> None:
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("the calls on paged keys and values have no backward pass: expected inputs that do not "
                                 "require gradients, or torch.no_grad()")


def _off(tok_off, kv_len, dev: int) -> None:
    _want(tok_off, torch.int64, "tok_off", dev)
    if tok_off.shape[0] != kv_len.shape[0] + 1:
        raise ValueError("tok_off: expected one entry more than kv_len")


def _status(status, dev: int):
    if status is None:
        return None
    if status.dtype is not torch.int32 or status.numel() != 1 or status.get_device() != dev:
        raise ValueError("status: expected one int32 on the cache's device")
    return status.data_ptr()


def _room(k, need: int, dev: int, ws):
    if ws is not None and ws.numel() >= need and ws.is_contiguous() and ws.get_device() == dev:
        return ws
    return torch.empty(max(need, 256), dtype=torch.uint8, device=k.device)


def _place(w):
    return (None, 0) if w is None else (w.data_ptr(), w.numel())


def _stream(dev: int) -> int:
    _pkg()._on_current(dev, torch._C._cuda_getDevice())
    return torch._C._cuda_getCurrentRawStream(dev)


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
    p, dev, shape = _pkg(), k.get_device(), k.shape
    kv = _paged(k, v, page_ids, page_off, kv_len, shape, dev)
    _off(tok_off, kv_len, dev)
    ks, vs = _tokens(k_new, "k_new", k, dev, shape[3], shape[1]), _tokens(v_new, "v_new", k, dev, shape[3], shape[1])
    if v_new.shape != k_new.shape:
        raise ValueError("v_new: expected k_new's shape")
    _no_backward(k_new, v_new, k, v)
    L = p.lib()
    w = _room(k, L.ptc_kv_append_workspace_bytes(kv_len.shape[0]), dev, ws) if status is None else None
    rc = L.ptc_kv_append(kv, k_new.data_ptr(), v_new.data_ptr(), ks, vs, tok_off.data_ptr(), k_new.shape[0],
                         *_place(w), _status(status, dev), _stream(dev))
    p._check("ptc_kv_append", rc)


def ptc_paged_attention(q, k, v, page_ids, page_off, tok_off, kv_len, max_q_len: int, scale: float | None = None,
                        mass: torch.Tensor | None = None, mass_out: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                        ws: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """Causal attention of new tokens ``q`` [tokens, query heads, head_dim] over
    their requests' pages.  Returns (out, lse), with ``mass`` (the weights
    accumulated so far, float32 [key heads, slots]) or ``mass_out`` (where the
    new sums go; may be ``mass`` itself) also the accumulated weights, which in
    slots of no request are what they were (zero without ``mass``).  ``scale``
    defaults to head_dim ** -0.5."""
    p, dev, shape = _pkg(), k.get_device(), k.shape
    kv = _paged(k, v, page_ids, page_off, kv_len, shape, dev)
    _off(tok_off, kv_len, dev)
    if not 0 <= max_q_len <= _U32:
        raise ValueError("max_q_len: expected a number of 32 bits, not negative")
    D = shape[3]
    qs = _tokens(q, "q", k, dev, D)
    T, Hq, _ = q.shape
    _no_backward(q, k, v, mass, mass_out, out, lse)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out: expected q's shape")
    else:
        _want(out, q.dtype, "out", dev, 3)
    if lse is None:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
    elif lse.shape != q.shape[:2]:
        raise ValueError("lse: expected q's first two dimensions")
    else:
        _want(lse, torch.float32, "lse", dev, 2)
    slots, m_in, m_out = 0, None, None
    if mass is not None or mass_out is not None:
        if mass_out is None:
            mass_out = torch.empty_like(mass)
        _want(mass_out, torch.float32, "mass_out", dev, 2)
        if mass is not None:
            _want(mass, torch.float32, "mass", dev, 2)
            if mass.shape != mass_out.shape:
                raise ValueError("mass: expected mass_out's shape")
            m_in = mass.data_ptr()
        if mass_out.shape[0] != shape[1]:
            raise ValueError("mass: expected one row a key head")
        slots, m_out = mass_out.shape[1], mass_out.data_ptr()
        # the call writes the slots of page_ids, and without requests none
        first = page_ids.shape[0] * shape[2] if kv_len.shape[0] else 0
        if slots > first and m_in != m_out:
            mass_out[:, first:] = 0 if mass is None else mass[:, first:]
    L = p.lib()
    w = _room(k, L.ptc_paged_attention_workspace_bytes(kv_len.shape[0], Hq, shape[1], D, max_q_len, slots), dev, ws)
    rc = L.ptc_paged_attention(kv, q.data_ptr(), qs, tok_off.data_ptr(), T, Hq, max_q_len,
                               D ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr(), m_in, m_out, slots,
                               w.data_ptr(), w.numel(), _status(status, dev), _stream(dev))
    p._check("ptc_paged_attention", rc)
    return (out, lse) if mass_out is None else (out, lse, mass_out)


def ptc_kv_evict(k, v, page_ids, page_off, kv_len, mass, dst_page_ids, dst_page_off, n_keep: int, n_sink: int,
                 n_recent: int, max_kv_len: int, ws: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """Cuts every request to n_keep tokens a key head (the first n_sink, the
    last n_recent and the heaviest others) and moves them to the destination
    pages.  Returns (keep int32 [requests, key heads, n_keep], new_len int32,
    new_mass float32 [key heads, destination slots], zero where no token was
    moved)."""
    p, dev, shape = _pkg(), k.get_device(), k.shape
    kv = _paged(k, v, page_ids, page_off, kv_len, shape, dev)
    _want(mass, torch.float32, "mass", dev, 2)
    _want(dst_page_ids, torch.int32, "dst_page_ids", dev)
    _want(dst_page_off, torch.int64, "dst_page_off", dev)
    n_req, heads = kv_len.shape[0], shape[1]
    if dst_page_off.shape[0] != n_req + 1:
        raise ValueError("dst_page_off: expected one entry more than kv_len")
    if mass.shape[0] != heads:
        raise ValueError("mass: expected one row a key head")
    if min(n_keep, n_sink, n_recent, max_kv_len) < 0 or max(n_keep, n_sink, n_recent, max_kv_len) > _U32:
        raise ValueError("n_keep, n_sink, n_recent and max_kv_len: expected numbers of 32 bits, none negative")
    _no_backward(k, v, mass)
    keep = torch.empty((n_req, heads, n_keep), dtype=torch.int32, device=k.device)
    new_len = torch.empty(n_req, dtype=torch.int32, device=k.device)
    slots = dst_page_ids.shape[0] * shape[2]
    new_mass = torch.empty((heads, slots), dtype=torch.float32, device=k.device)
    if n_req == 0:
        new_mass.zero_()  # the call has nothing to do
    L = p.lib()
    w = _room(k, L.ptc_kv_evict_workspace_bytes(n_req, heads, max_kv_len), dev, ws) if status is None else None
    rc = L.ptc_kv_evict(kv, mass.data_ptr(), mass.shape[1], n_keep, n_sink, n_recent, max_kv_len,
                        dst_page_ids.data_ptr(), dst_page_off.data_ptr(), dst_page_ids.shape[0], keep.data_ptr(),
                        new_len.data_ptr(), new_mass.data_ptr(), slots, *_place(w), _status(status, dev), _stream(dev))
    p._check("ptc_kv_evict", rc)
    return keep, new_len, new_mass
