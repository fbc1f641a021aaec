"""Paged keys and values in 4 bits: 3.2 times as many tokens of 128 channels in
the same memory, 2.7 times as many of 64.  (Rows are of 64 or of 128 channels:
heads of 80 gain a factor of 2, heads of 24 none, and heads of 16 lose one of 1.5.)

    k4, v4 = (torch.zeros(pages, heads, block_size, kv4_row_bytes(head_dim), dtype=torch.uint8, device="cuda") ...)
    q_out    = ptc_kv4_append(k_new, v_new, k4, v4, page_ids, page_off, tok_off, kv_len, q=q, rope=rope)
    out, lse = ptc_kv4_attention(q_out, k4, v4, page_ids, page_off, tok_off, kv_len, max_q_len)
    k, v     = ptc_kv4_read(k4, v4, page_ids, page_off, tok_off, kv_len, n_tok, head_dim, dtype)

``k4`` and ``v4`` are uint8 CUDA tensors of shape [pages, key heads, block_size,
kv4_row_bytes(head_dim)] with any strides that are multiples of 16 and a
contiguous last dimension.  A row stands for a head's channels in bfloat16 or
float16: 32 of them share a scale and a base, and code c stands for (16 + c) *
scale + base, rounded to that type.  The tensors do not say which: a cache is
written and read with one type.

Page lists, ``status`` and gradients are as in ``kv``, positions as in ``rope``.
"""
from __future__ import annotations

import ctypes

import torch

from .kv import (_DTYPES, _U32, MAX_HEAD_DIM, PAGED_KV, _no_backward, _off, _pkg, _place, _room, _status, _stream,
                 _tokens, _want)
from .rope import _pack, _queries


def declare(L) -> None:
    """The argument types of the library's calls on pages of 4 bits."""
    vp, u32, u64, sz, st = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    packed = ctypes.c_char_p
    L.ptc_kv4_row_bytes.restype = u32
    L.ptc_kv4_row_bytes.argtypes = [u32]
    for name in ("ptc_kv4_append", "ptc_kv4_read"):
        f = getattr(L, name + "_workspace_bytes")
        f.restype = sz
        f.argtypes = [u32]
    L.ptc_kv4_append.restype = st
    L.ptc_kv4_append.argtypes = [packed, packed, vp, packed, vp, packed, u32, vp, vp, packed, packed, vp, u64, vp, sz, vp,
                                 vp]
    L.ptc_kv4_read.restype = st
    L.ptc_kv4_read.argtypes = [packed, vp, u64, vp, vp, vp, sz, vp, vp]
    L.ptc_kv4_attention_workspace_bytes.restype = sz
    L.ptc_kv4_attention_workspace_bytes.argtypes = [u32, u32, u32, u32, u32, u64, u64, u32]
    L.ptc_kv4_attention.restype = st
    L.ptc_kv4_attention.argtypes = [packed, vp, packed, vp, u64, u32, u32, ctypes.c_float, vp, vp, vp, sz, vp, vp]


def kv4_row_bytes(head_dim: int) -> int:
    """Bytes of a row of head_dim channels."""
    if not 16 <= head_dim <= MAX_HEAD_DIM or head_dim % 8:
        raise ValueError(f"head_dim: expected a multiple of 8 from 16 to {MAX_HEAD_DIM}")
    return 48 if head_dim <= 64 else 80


def _paged4(k, v, page_ids, page_off, kv_len, shape, head_dim: int, dtype, dev: int) -> bytes:
    """The packed ptc_paged_kv; shape is k's, dev its device's index."""
    if dev < 0:
        raise ValueError("expected a CUDA tensor")
    if dtype not in _DTYPES:
        raise ValueError("expected a cache of bfloat16 or float16 values")
    row = kv4_row_bytes(head_dim)
    if k.dtype is not torch.uint8 or v.dtype is not torch.uint8 or len(shape) != 4 or v.shape != shape or (
            v.get_device() != dev or shape[3] != row):
        raise ValueError(f"k4 and v4: expected uint8 tensors [pages, key heads, block_size, {row}] of one shape")
    k0, k1, k2, k3 = k.stride()
    v0, v1, v2, v3 = v.stride()
    if k3 != 1 or v3 != 1:
        raise ValueError("k4 and v4: expected a contiguous last dimension")
    _want(page_ids, torch.int32, "page_ids", dev)
    _want(page_off, torch.int64, "page_off", dev)
    _want(kv_len, torch.int32, "kv_len", dev)
    n_req = kv_len.shape[0]
    if page_off.shape[0] != n_req + 1:
        raise ValueError("page_off: expected one entry more than kv_len")
    return PAGED_KV.pack(k.data_ptr(), v.data_ptr(), k0, k1, k2, v0, v1, v2, page_ids.data_ptr(), page_off.data_ptr(),
                         kv_len.data_ptr(), page_ids.shape[0], shape[0], n_req, shape[2], shape[1], head_dim,
                         _DTYPES[dtype])


def ptc_kv4_append(k_new, v_new, k4, v4, page_ids, page_off, tok_off, kv_len, q: torch.Tensor | None = None,
                   rope: torch.Tensor | None = None, pos: torch.Tensor | None = None, interleaved: bool = False,
                   q_out: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                   status: torch.Tensor | None = None):
    """Quantises the new tokens' keys and values ([tokens, key heads, head_dim])
    into their requests' pages, as the last tokens of kv_len.  With ``rope`` the
    keys are turned first, and the queries ``q`` with them: returned as of
    ptc_kv_append_rope, else None."""
    p, dev, shape = _pkg(), k4.get_device(), k4.shape
    D = k_new.shape[-1]
    kv = _paged4(k4, v4, page_ids, page_off, kv_len, shape, D, k_new.dtype, dev)
    _off(tok_off, kv_len, dev)
    ks, vs = _tokens(k_new, "k_new", k_new, dev, D, shape[1]), _tokens(v_new, "v_new", k_new, dev, D, shape[1])
    if v_new.shape != k_new.shape:
        raise ValueError("v_new: expected k_new's shape")
    T = k_new.shape[0]
    if rope is None and (q is not None or pos is not None):
        raise ValueError("q and pos: expected a rope with them")
    angles = None if rope is None else _pack(rope, pos, interleaved, T, D, dev)
    queries, q_out = _queries(q, q_out, k_new, dev, D, T)
    _no_backward(q, k_new, v_new, rope, q_out)
    L = p.lib()
    w = _room(k4, L.ptc_kv4_append_workspace_bytes(kv_len.shape[0]), dev, ws) if status is None else None
    rc = L.ptc_kv4_append(kv, angles, *queries, k_new.data_ptr(), v_new.data_ptr(), ks, vs, tok_off.data_ptr(), T,
                          *_place(w), _status(status, dev), _stream(dev))
    p._check("ptc_kv4_append", rc)
    return q_out


def ptc_kv4_read(k4, v4, page_ids, page_off, tok_off, kv_len, n_tok: int, head_dim: int, dtype=torch.bfloat16,
                 k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                 status: torch.Tensor | None = None):
    """(k, v) [n_tok, key heads, head_dim] of ``dtype``: the values of every
    request's last tokens, as many as tok_off gives it, n_tok in all."""
    p, dev, shape = _pkg(), k4.get_device(), k4.shape
    kv = _paged4(k4, v4, page_ids, page_off, kv_len, shape, head_dim, dtype, dev)
    _off(tok_off, kv_len, dev)
    if not 0 <= n_tok <= 1 << 31:
        raise ValueError("n_tok: expected a number of tokens")
    size = (n_tok, shape[1], head_dim)
    outs = []
    for x, name in ((k_out, "k_out"), (v_out, "v_out")):
        if x is None:
            x = torch.empty(size, dtype=dtype, device=k4.device)
        else:
            _want(x, dtype, name, dev, 3)
            if x.shape != size:
                raise ValueError(f"{name}: expected [n_tok, key heads, head_dim]")
        outs.append(x)
    _no_backward(*outs)
    L = p.lib()
    w = _room(k4, L.ptc_kv4_read_workspace_bytes(kv_len.shape[0]), dev, ws) if status is None else None
    rc = L.ptc_kv4_read(kv, tok_off.data_ptr(), n_tok, outs[0].data_ptr(), outs[1].data_ptr(), *_place(w),
                        _status(status, dev), _stream(dev))
    p._check("ptc_kv4_read", rc)
    return tuple(outs)


def ptc_kv4_attention(q, k4, v4, page_ids, page_off, tok_off, kv_len, max_q_len: int, scale: float | None = None,
                      out: torch.Tensor | None = None, lse: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                      status: torch.Tensor | None = None):
    """Causal attention of new tokens ``q`` [tokens, query heads, head_dim] over
    their requests' pages of 4 bits, which stand for values of q's type.  Returns
    (out, lse); ``scale`` defaults to head_dim ** -0.5."""
    p, dev, shape = _pkg(), k4.get_device(), k4.shape
    D = q.shape[-1]
    kv = _paged4(k4, v4, page_ids, page_off, kv_len, shape, D, q.dtype, dev)
    _off(tok_off, kv_len, dev)
    if not 0 <= max_q_len <= _U32:
        raise ValueError("max_q_len: expected a number of 32 bits, not negative")
    qs = _tokens(q, "q", q, dev, D)
    T, Hq, _ = q.shape
    _no_backward(q, out, lse)
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
    L = p.lib()
    w = _room(k4, L.ptc_kv4_attention_workspace_bytes(kv_len.shape[0], Hq, shape[1], D, max_q_len, T, page_ids.shape[0],
                                                      shape[2]), dev, ws)
    rc = L.ptc_kv4_attention(kv, q.data_ptr(), qs, tok_off.data_ptr(), T, Hq, max_q_len,
                             D ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr(), w.data_ptr(),
                             w.numel(), _status(status, dev), _stream(dev))
    p._check("ptc_kv4_attention", rc)
    return out, lse
