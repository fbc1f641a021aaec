"""Rotary positions: the table of angles, and the write of new tokens with the
rotation on the way.

    freq, factor = rope_frequencies(rot_dim, scaling="parts", factor=8, original=8192)
    rope  = ptc_rope_table(freq.cuda(), n_pos, factor)          # float32 [n_pos, 2 * pairs]
    q_out = ptc_kv_append_rope(q, k_new, v_new, k, v, page_ids, page_off, tok_off, kv_len, rope)

Pair i of a head's channels is (i, pairs + i), or (2 i, 2 i + 1) with
``interleaved``; channels from 2 * pairs on are left as they are.  A token's
position is its place in its context, or its entry of ``pos``.

Caches, page lists, ``status`` and gradients are as in ``kv``.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from .kv import (_STRIDES, _U32, _no_backward, _off, _paged, _pkg, _place, _room, _status, _stream, _tokens,
                 _want)

# ptc_rope, as the C compiler lays it out
ROPE = struct.Struct("@PPIIi0P")
_NO_STRIDES = _STRIDES.pack(0, 0)


def declare(L) -> None:
    """The argument types of the library's calls on rotary positions."""
    vp, u32, u64, sz, st = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    packed = ctypes.c_char_p
    L.ptc_rope_table.restype = st
    L.ptc_rope_table.argtypes = [vp, u32, u32, ctypes.c_float, vp, vp]
    L.ptc_kv_append_rope_workspace_bytes.restype = sz
    L.ptc_kv_append_rope_workspace_bytes.argtypes = [u32]
    L.ptc_kv_append_rope.restype = st
    L.ptc_kv_append_rope.argtypes = [packed, packed, vp, packed, vp, packed, u32, vp, vp, packed, packed, vp, u64, vp, sz,
                                     vp, vp]


def rope_frequencies(rot_dim: int, base: float = 10_000.0, scaling: str = "none", factor: float = 1.0,
                     original: int = 4096, slow: float = 1.0, fast: float = 32.0):
    """(frequencies, table factor): radians a position of the rot_dim / 2 pairs, a
    float64 CPU tensor, and what cosines and sines are multiplied by.

    base ** (-2 i / rot_dim), for contexts of ``factor`` times the ``original``
    positions scaled by

    * "linear": all frequencies divided by factor;
    * "base": the base times factor ** (rot_dim / (rot_dim - 2)), which divides the
      slowest frequency by factor and leaves the fastest;
    * "parts": pairs of at most ``slow`` turns over the original positions divided
      by factor, those of at least ``fast`` left, those between mixed in proportion
      to their turns; cosines and sines are multiplied by 0.1 ln(factor) + 1.

    (Models whose frequencies were mixed in another way, such as in proportion to
    the pair's index between the two bounds, want others: ptc_rope_table takes any.)"""
    if rot_dim < 2 or rot_dim % 2 or not base > 0 or not factor >= 1:
        raise ValueError("rope_frequencies: expected an even rot_dim, a positive base and a factor of at least 1")
    i = torch.arange(0, rot_dim, 2, dtype=torch.float64)
    if scaling == "base":
        if rot_dim == 2:
            raise ValueError("rope_frequencies: scaling by the base needs two pairs at least")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-i / rot_dim)
    if scaling in ("none", "base"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "parts":
        raise ValueError('rope_frequencies: expected a scaling "none", "linear", "base" or "parts"')
    if not (original > 0 and 0 <= slow < fast):
        raise ValueError("rope_frequencies: expected original positions, and fewer slow than fast turns")
    keep = ((original * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1


def _pack(rope, pos, interleaved: bool, n_tok: int, head_dim: int, dev: int) -> bytes:
    _want(rope, torch.float32, "rope", dev, 2)
    n_pos, width = rope.shape
    if width < 2 or width % 2 or width > head_dim or not 0 < n_pos <= _U32:
        raise ValueError(f"rope: expected [positions, 2 * pairs], an even width of at most {head_dim}")
    if pos is not None:
        _want(pos, torch.int32, "pos", dev)
        if pos.shape[0] != n_tok:
            raise ValueError("pos: expected one position a new token")
    return ROPE.pack(rope.data_ptr(), 0 if pos is None else pos.data_ptr(), n_pos, width // 2, 1 if interleaved else 0)


def _queries(q, q_out, like, dev: int, head_dim: int, n_tok: int):
    """q's pointer and strides, q_out's, the number of heads, and q_out."""
    if q is None:
        if q_out is not None:
            raise ValueError("q_out: expected queries with it")
        return (None, _NO_STRIDES, None, _NO_STRIDES, 0), None
    qs = _tokens(q, "q", like, dev, head_dim)
    if q.shape[0] != n_tok:
        raise ValueError("q: expected a row for every new token")
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif q_out.shape != q.shape:
        raise ValueError("q_out: expected q's shape")
    return (q.data_ptr(), qs, q_out.data_ptr(), _tokens(q_out, "q_out", like, dev, head_dim), q.shape[1]), q_out


def ptc_rope_table(freq: torch.Tensor, n_pos: int, factor: float = 1.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """The table of positions 0 .. n_pos - 1: float32 [n_pos, 2 * pairs], the
    cosines of p * freq, then the sines, times ``factor``.  freq: float64 CUDA
    tensor, radians a position.  Returns when the work is enqueued."""
    p, dev = _pkg(), freq.get_device()
    if dev < 0:
        raise ValueError("expected a CUDA tensor")
    _want(freq, torch.float64, "freq", dev)
    if not 0 <= n_pos <= _U32:
        raise ValueError("n_pos: expected a number of 32 bits, not negative")
    shape = (n_pos, 2 * freq.shape[0])
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=freq.device)
    else:
        _want(out, torch.float32, "out", dev, 2)
        if out.shape != shape:
            raise ValueError("out: expected a row a position and two columns a frequency")
    _no_backward(freq, out)
    rc = p.lib().ptc_rope_table(freq.data_ptr(), freq.shape[0], n_pos, factor, out.data_ptr(), _stream(dev))
    p._check("ptc_rope_table", rc)
    return out


def ptc_kv_append_rope(q, k_new, v_new, k, v, page_ids, page_off, tok_off, kv_len, rope, pos: torch.Tensor | None = None,
                       interleaved: bool = False, q_out: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                       status: torch.Tensor | None = None):
    """ptc_kv_append with the new keys turned on the way, and the new tokens'
    queries ``q`` [tokens, query heads, head_dim] with them.  Returns the turned
    queries: ``q_out``, which may be ``q`` itself, or a new tensor; None where q
    is None."""
    p, dev, shape = _pkg(), k.get_device(), k.shape
    kv = _paged(k, v, page_ids, page_off, kv_len, shape, dev)
    _off(tok_off, kv_len, dev)
    D = shape[3]
    ks, vs = _tokens(k_new, "k_new", k, dev, D, shape[1]), _tokens(v_new, "v_new", k, dev, D, shape[1])
    if v_new.shape != k_new.shape:
        raise ValueError("v_new: expected k_new's shape")
    T = k_new.shape[0]
    angles = _pack(rope, pos, interleaved, T, D, dev)
    queries, q_out = _queries(q, q_out, k, dev, D, T)
    _no_backward(q, k_new, v_new, k, v, rope, q_out)
    L = p.lib()
    w = _room(k, L.ptc_kv_append_rope_workspace_bytes(kv_len.shape[0]), dev, ws) if status is None else None
    rc = L.ptc_kv_append_rope(kv, angles, *queries, k_new.data_ptr(), v_new.data_ptr(), ks, vs, tok_off.data_ptr(), T,
                              *_place(w), _status(status, dev), _stream(dev))
    p._check("ptc_kv_append_rope", rc)
    return q_out
