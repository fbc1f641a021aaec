"""A paged cache with requests in it, and the operators' definitions in 64
bits, for the tests of the calls on paged keys and values."""
import math

import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
# half a unit in the last place, relative: 8 and 11 significant bits
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Cache:
    """Requests of (new, total) tokens.  Slots that hold no token are NaN."""

    def __init__(self, lens, Hq=4, Hkv=2, D=64, B=16, dtype="bf16", layout="head", spare=1, shared=0, seed=0, q_scale=1.5,
                 extra_pages=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = DT[dtype]
        self.lens, self.Hq, self.Hkv, self.D, self.B, self.dt = lens, Hq, Hkv, D, B, dt
        self.new, self.total = [m for m, _ in lens], [n for _, n in lens]
        count = [-(-n // B) + spare for n in self.total]
        S = shared // B
        own = [c - S if r else c for r, c in enumerate(count)]
        self.n_pages = sum(own) + extra_pages
        perm = torch.randperm(self.n_pages, generator=g, device="cuda").to(torch.int32)
        ids, at = [], 0
        for r, c in enumerate(own):
            mine = perm[at:at + c]
            at += c
            ids.append(torch.cat([ids[0][:S], mine]) if r and S else mine)
        self.lists = ids
        self.page_ids = torch.cat(ids) if ids else torch.zeros(0, dtype=torch.int32, device="cuda")
        off = lambda x: torch.tensor([0] + list(x), dtype=torch.int64).cumsum(0).cuda()
        self.page_off, self.tok_off = off(count), off(self.new)
        self.kv_len = torch.tensor(self.total, dtype=torch.int32, device="cuda")
        shape = (self.n_pages, Hkv, B, D) if layout == "head" else (self.n_pages, B, Hkv, D)
        self.k = torch.full(shape, math.nan, dtype=dt, device="cuda")
        self.v = torch.full(shape, math.nan, dtype=dt, device="cuda")
        if layout != "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.keys, self.vals = [], []
        for r, n in enumerate(self.total):
            K = torch.randn(n, Hkv, D, generator=g, device="cuda").to(dt)
            V = torch.randn(n, Hkv, D, generator=g, device="cuda").to(dt)
            if r and S:
                K[:shared], V[:shared] = self.keys[0][:shared], self.vals[0][:shared]
            self.put(r, K, V)
            self.keys.append(K)
            self.vals.append(V)
        self.q = (torch.randn(sum(self.new), Hq, D, generator=g, device="cuda") * q_scale).to(dt)
        self.slots = sum(count) * B
        self.g = g

    def table(self):
        return self.k, self.v, self.page_ids, self.page_off

    def where(self, r, n):
        j = torch.arange(n, device="cuda")
        return self.lists[r].long()[j // self.B], j % self.B

    def put(self, r, K, V):
        page, slot = self.where(r, K.shape[0])
        self.k[page, :, slot] = K
        self.v[page, :, slot] = V

    def request(self, r):
        """Queries, keys and values of a request in 64 bits, heads first."""
        a, b = int(self.tok_off[r]), int(self.tok_off[r + 1])
        return self.q[a:b].double().transpose(0, 1), self.keys[r].double().transpose(0, 1), self.vals[r].double().transpose(0, 1)


def reference(c, scale=None, mass=None):
    """(out, lse, mass, and the bounds of their errors) by the definition.

    A score is a sum of D products of 16-bit numbers, exact in 32 bits, added
    in 32 bits: its error is below D * 2^-23 * scale * sum |q k|, far more than
    what any order of the sum makes (and as much again for chopped sums).
    exp2 and log2 of the hardware are good to 2^-21 of their result, and to
    2^-21 absolute.  The weights meet the values rounded to the cache's type,
    and the result is rounded once more."""
    scale = c.D ** -0.5 if scale is None else scale
    u = UNIT[c.dt]
    T = c.q.shape[0]
    out = torch.zeros(T, c.Hq, c.D, dtype=torch.float64, device="cuda")
    lse = torch.full((T, c.Hq), -math.inf, dtype=torch.float64, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    m_out = torch.zeros(c.Hkv, c.slots, dtype=torch.float64, device="cuda")
    m_tol = torch.zeros_like(m_out)
    G = c.Hq // c.Hkv
    for r, (m, n) in enumerate(c.lens):
        base = int(c.page_off[r]) * c.B
        if mass is not None:
            m_out[:, base:base + n] = mass[:, base:base + n].double()
        if m == 0 or n == 0:
            continue
        a = int(c.tok_off[r])
        q, k, v = c.request(r)
        for h in range(c.Hq):
            kh, vh = k[h // G], v[h // G]
            s = q[h] @ kh.T * scale
            err = (q[h].abs() @ kh.abs().T).amax(1) * scale * c.D * 2.0 ** -23 + 2.0 ** -20
            sees = torch.arange(n, device="cuda")[None] < (n - m + 1 + torch.arange(m, device="cuda"))[:, None]
            s = torch.where(sees, s, -math.inf)
            some = sees.any(1)
            z = torch.logsumexp(s, 1)
            w = torch.where(some[:, None], torch.exp(s - z[:, None]), 0.0)
            out[a:a + m, h] = w @ vh
            lse[a:a + m, h] = z
            size = w @ vh.abs()
            out_tol[a:a + m, h] = (u + 2 * err[:, None]) * 1.01 * size + u * (w @ vh).abs() + n * 2.0 ** -30 * vh.abs().amax()
            lse_tol[a:a + m, h] = err + 2.0 ** -20 * (1 + torch.where(some, z, 0.0).abs())
            m_out[h // G, base:base + n] += w.sum(0)
            e = 2 * err + 2.0 ** -20 * (2 + torch.where(some, z, 0.0).abs())
            m_tol[h // G, base:base + n] += (w * e[:, None]).sum(0) * 1.01 + m * 2.0 ** -60
    return out, lse, m_out, out_tol, lse_tol, m_tol + m_out.abs() * 2.0 ** -20


def close(got, want, tol):
    got = got.double()
    gone = torch.isinf(want)
    assert torch.equal(got[gone], want[gone])
    d = torch.where(gone, 0.0, got - want).abs()
    assert not torch.isnan(d).any(), "NaN"
    over = d - torch.where(gone, 0.0, tol)
    assert (over <= 0).all(), f"off by {float(d.max()):.3g}, {float(over.max()):.3g} over the bound at {int(over.argmax())}"


def check_attention(c, mass=None, scale=None, **kw):
    import paper_2609_28870_gb300 as ptc
    more = {} if mass is None else {"mass": mass}
    got = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), scale=scale, **more, **kw)
    out, lse, m, ot, lt, mt = reference(c, scale, mass)
    close(got[0], out, ot)
    close(got[1], lse, lt)
    if mass is not None:
        at = torch.zeros(c.slots, dtype=torch.bool, device="cuda")
        at[int(c.page_off[0]) * c.B:int(c.page_off[-1]) * c.B] = True
        close(got[2][:, at], m[:, at], mt[:, at])
    return got
