"""Rotations and rows of 4 bits by their definitions, for the tests of the calls
that write and read them."""
import math
from fractions import Fraction

import torch

from tests.kv_util import Cache

BITS = {torch.bfloat16: (8, -133), torch.float16: (11, -24)}  # significant bits, exponent of the smallest step


def once(x, dtype):
    """64 bits to 16 bits in one rounding, to even."""
    bits, least = BITS[dtype]
    step = torch.exp2((torch.frexp(x).exponent - bits).clamp(min=least).double())
    return (torch.round(x / step) * step).to(dtype)


def turned(x, rope, pos, interleaved):
    """Rows [T, heads, D] turned by the table's rows of pos, in 64 bits, rounded once."""
    n = rope.shape[1] // 2
    c, s = rope[pos.long(), :n].double()[:, None], rope[pos.long(), n:].double()[:, None]
    first = torch.arange(n, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    a, b = x[..., first].double(), x[..., second].double()
    y = x.clone()
    y[..., first], y[..., second] = once(a * c - b * s, x.dtype), once(b * c + a * s, x.dtype)
    return y


def row_bytes(D):
    return 48 if D <= 64 else 80


def rows_of(x):
    """Tokens [T, heads, D] as rows of bytes, in 64 bits."""
    T, H, D = x.shape
    Dp = 64 if D <= 64 else 128
    row = torch.zeros(T, H, row_bytes(D), dtype=torch.uint8, device=x.device)
    code = torch.zeros(T, H, Dp, dtype=torch.int64, device=x.device)
    for a in range(0, D, 32):
        part = x[..., a:min(a + 32, D)].double()
        lo, hi = part.amin(-1), part.amax(-1)
        s = once((hi - lo) / 15, x.dtype)
        b = once(lo - 16 * s.double(), x.dtype)
        z = torch.floor((part - b.double()[..., None]) / s.double()[..., None] - 15.5).clamp(0, 15)
        code[..., a:a + part.shape[-1]] = torch.where(s[..., None] == 0, 0.0, z).long()
        at = Dp // 2 + a // 8
        row[..., at:at + 4] = torch.stack([s, b], -1).contiguous().view(torch.uint8)
    e = torch.arange(8, device=x.device)
    word = (code.unflatten(-1, (-1, 8)) << (4 * (e // 2) + 16 * (e % 2))).sum(-1)
    row[..., :Dp // 2] = (word[..., None] >> 8 * torch.arange(4, device=x.device) & 255).to(torch.uint8).flatten(-2)
    return row


def values_of(row, D, dtype):
    """What rows of bytes stand for."""
    Dp = 64 if D <= 64 else 128
    d = torch.arange(D, device=row.device)
    e = d % 8
    code = row[..., 4 * (d // 8) + 2 * (e % 2) + e // 4].long() >> (4 * (e // 2 % 2)) & 15
    p = row[..., Dp // 2:Dp // 2 + Dp // 8].contiguous().view(dtype).double()
    out = (16 + code) * p[..., d // 32 * 2] + p[..., d // 32 * 2 + 1]
    return once(out, dtype)


def group_by_fractions(x, dtype):
    """Codes, scale and base of one group of finite numbers, in exact arithmetic."""
    bits, least = BITS[dtype]

    def rn(f):
        if f == 0:
            return Fraction(0)
        e = math.floor(math.log2(abs(f.numerator)) - math.log2(f.denominator))
        while abs(f) >= Fraction(2) ** (e + 1):
            e += 1
        while abs(f) < Fraction(2) ** e:
            e -= 1
        step = Fraction(2) ** max(e + 1 - bits, least)
        return round(f / step) * step

    x = [Fraction(v) for v in x]
    s = rn((max(x) - min(x)) / 15)
    b = rn(min(x) - 16 * s)
    return [0 if s == 0 else min(15, max(0, math.floor((v - b) / s - Fraction(31, 2)))) for v in x], s, b


class Cache4(Cache):
    """A paged cache of 4 bits with requests in it: keys and vals are what the
    rows stand for.  Slots that hold no token are all ones: codes of 15, NaN."""

    def __init__(self, lens, layout="head", **kw):
        super().__init__(lens, layout=layout, **kw)
        shape = (self.n_pages, self.Hkv, self.B, row_bytes(self.D))
        if layout != "head":
            shape = (shape[0], shape[2], shape[1], shape[3])
        self.k, self.v = (torch.full(shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2))
        if layout != "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for r in range(len(lens)):
            K, V = rows_of(self.keys[r]), rows_of(self.vals[r])
            self.put(r, K, V)
            self.keys[r], self.vals[r] = values_of(K, self.D, self.dt), values_of(V, self.D, self.dt)



def check_attention4(c, scale=None, **kw):
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import close, reference
    got = ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), scale=scale, **kw)
    out, lse, _, out_tol, lse_tol, _ = reference(c, scale)
    close(got[0], out, out_tol)
    close(got[1], lse, lse_tol)
    return got
