"""ptc_kv_append and ptc_kv_evict: exact, on every layout, with ties, zeros,
NaN and infinities among the weights, at lengths around the limits; refusals;
and the three calls together with the block ids of a trace as page lists."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


def bits(x):
    import torch
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("lens", [[(1, 1)], [(1, 17), (1, 16), (1, 500)], [(40, 40), (0, 9), (0, 0), (33, 70), (1, 5)],
                                  [(700, 900), (300, 300)]])
@pytest.mark.parametrize("B,D,Hkv,layout", [(16, 128, 2, "head"), (16, 64, 8, "token"), (1, 16, 1, "head"),
                                            (12, 40, 3, "token"), (256, 96, 5, "head")])
def test_append(lens, B, D, Hkv, layout):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache(lens, Hq=Hkv, Hkv=Hkv, D=D, B=B, layout=layout)
    want_k, want_v = c.k.clone(), c.v.clone()
    k_new = torch.cat([k[n - m:] for k, (m, n) in zip(c.keys, lens)])
    both = torch.stack([k_new, torch.cat([v[n - m:] for v, (m, n) in zip(c.vals, lens)])], 1)  # strides: one buffer
    for r, (m, n) in enumerate(lens):
        page, slot = c.where(r, n)
        c.k[page[n - m:], :, slot[n - m:]] = math.nan
        c.v[page[n - m:], :, slot[n - m:]] = math.nan
    ptc.ptc_kv_append(both[:, 0], both[:, 1], *c.table(), c.tok_off, c.kv_len)
    assert torch.equal(bits(c.k), bits(want_k)) and torch.equal(bits(c.v), bits(want_v))


def test_append_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(2, 40), (3, 20)], Hq=2)
    x = torch.zeros(5, 2, 64, dtype=c.dt, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    i64 = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")
    before = bits(c.k).clone()

    def refused(*a):
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_kv_append(*a)
        assert e.value.name == "PTC_ERR_INVALID_ARG"

    ids = c.page_ids.clone()
    ids[:] = c.n_pages
    refused(x, x, c.k, c.v, ids, c.page_off, c.tok_off, c.kv_len)
    refused(x, x, *c.table(), i64([0, 6, 5]), c.kv_len)
    refused(x, x, *c.table(), i64([0, 2, 2]), i32([1, 1]))
    assert torch.equal(bits(c.k), before)
    refused(x, x, *c.table(), c.tok_off, i32([40, 2]))       # fewer tokens than new ones
    refused(x, x, *c.table(), c.tok_off, i32([40, 900]))     # more than the pages hold
    with pytest.raises(ValueError):
        ptc.ptc_kv_append(x[:, :1], x, *c.table(), c.tok_off, c.kv_len)
    with pytest.raises(ValueError):
        ptc.ptc_kv_append(x.half(), x, *c.table(), c.tok_off, c.kv_len)


# ---------------------------------------------------------------- evict
def chosen(w, n, n_keep, n_sink, n_recent):
    """The kept positions by the definition, on the host."""
    if n <= n_keep:
        return list(range(n))
    w = np.asarray(w[:n], dtype=np.float64)
    mid = range(n_sink, n - n_recent)
    key = lambda j: (0, -w[j], j) if not np.isnan(w[j]) else (1, 0, j)
    best = sorted(mid, key=key)[: n_keep - n_sink - n_recent]
    return sorted(set(range(n_sink)) | set(best) | set(range(n - n_recent, n)))


def evict(c, mass, n_keep, n_sink, n_recent, max_len=None, spare=1):
    """Runs the call into new pages behind c's and checks all of it."""
    import torch
    import paper_2609_28870_gb300 as ptc
    want = [[chosen(mass[h, int(c.page_off[r]) * c.B:].tolist()[:n], n, n_keep, n_sink, n_recent) for h in range(c.Hkv)]
            for r, n in enumerate(c.total)]
    kept = [min(n, n_keep) for n in c.total]
    count = [-(-b // c.B) + spare for b in kept]
    first, more = c.n_pages, sum(count)
    grow = lambda x: torch.cat([x, torch.full((more,) + tuple(x.shape[1:]), 7, dtype=x.dtype, device="cuda")])
    k, v = grow(c.k), grow(c.v)
    if not c.k.is_contiguous():
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    ids = (first + torch.randperm(more, generator=c.g, device="cuda")).to(torch.int32)
    off = torch.tensor([0] + count, dtype=torch.int64).cumsum(0).cuda()
    src_k, src_v = bits(k[:first]).clone(), bits(v[:first]).clone()
    keep, new_len, new_mass = ptc.ptc_kv_evict(k, v, c.page_ids, c.page_off, c.kv_len, mass, ids, off, n_keep, n_sink,
                                               n_recent, max(c.total) if max_len is None else max_len)
    assert new_len.tolist() == kept
    assert torch.equal(bits(k[:first]), src_k) and torch.equal(bits(v[:first]), src_v)
    exp_k, exp_v = torch.full_like(k[first:], 7), torch.full_like(v[first:], 7)
    exp_m = torch.zeros_like(new_mass)
    for r, b in enumerate(kept):
        for h in range(c.Hkv):
            got = keep[r, h].tolist()
            assert got[:b] == want[r][h], (r, h)
            assert got[b:] == [-1] * (n_keep - b)
            i = torch.arange(b, device="cuda")
            src = torch.tensor(want[r][h], dtype=torch.long, device="cuda")
            page, slot = ids.long()[int(off[r]) + i // c.B] - first, i % c.B
            exp_k[page, h, slot] = c.keys[r][src, h]
            exp_v[page, h, slot] = c.vals[r][src, h]
            exp_m[h, int(off[r]) * c.B + i] = mass[h, int(c.page_off[r]) * c.B + src]
    assert torch.equal(bits(k[first:]), bits(exp_k)) and torch.equal(bits(v[first:]), bits(exp_v))
    assert torch.equal(bits(new_mass), bits(exp_m))
    return k, v, ids, off, new_len, new_mass


def weights(c, kind):
    import torch
    w = torch.exp(2 * torch.randn(c.Hkv, c.slots, generator=c.g, device="cuda"))
    pick = torch.rand(c.Hkv, c.slots, generator=c.g, device="cuda")
    if kind == "zeros":
        w[pick < 0.9] = 0
        w[pick < 0.4] = -0.0
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "ties":
        w = (pick * 4).floor()
    elif kind == "odd":
        for at, x in ((0.1, math.nan), (0.2, math.inf), (0.3, -math.inf), (0.4, -1.5), (0.5, 1e-42), (0.55, -math.nan)):
            w[(pick < at) & (pick >= at - 0.1)] = x
    elif kind == "close":  # values that differ in their last bits only
        w = (torch.full_like(w, 1.0).view(torch.int32) + (pick * 5).to(torch.int32)).view(torch.float32)
    return w


@pytest.mark.parametrize("kind", ["spread", "zeros", "equal", "ties", "odd", "close"])
@pytest.mark.parametrize("keep", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 4, 16), (64, 64, 0), (64, 0, 64), (64, 10, 54),
                                  (100, 0, 0), (333, 1, 2), (1024, 4, 64)])
def test_evict(kind, keep):
    from tests.kv_util import Cache
    c = Cache([(0, n) for n in (1, 63, 64, 65, 100, 1023, 1024, 1025, 2500, 0)], Hkv=2, Hq=2, D=64)
    evict(c, weights(c, kind), *keep)


@pytest.mark.parametrize("B,D,Hkv,layout,dtype", [(1, 16, 1, "head", "bf16"), (7, 24, 3, "token", "fp16"),
                                                  (16, 128, 8, "token", "bf16"), (256, 80, 2, "head", "fp16")])
def test_evict_layouts(B, D, Hkv, layout, dtype):
    from tests.kv_util import Cache
    c = Cache([(0, 300), (0, 90), (0, 1000)], Hq=Hkv, Hkv=Hkv, D=D, B=B, layout=layout, dtype=dtype)
    evict(c, weights(c, "spread"), 100, 3, 20)


@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict_long(kind):
    from tests.kv_util import Cache
    c = Cache([(0, 131_072), (0, 40_000), (0, 5000)], Hq=2, Hkv=2, D=16)
    evict(c, weights(c, kind), 8000, 16, 1024)


def test_evict_bound_above_the_lengths():
    from tests.kv_util import Cache
    c = Cache([(0, 300), (0, 90)], Hq=2)
    evict(c, weights(c, "spread"), 100, 3, 20, max_len=100_000)


def test_evict_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(0, 300), (0, 90)], Hq=2, extra_pages=40)
    mass = weights(c, "spread")
    used = c.page_ids.tolist()
    free = torch.tensor([p for p in range(c.n_pages) if p not in used], dtype=torch.int32, device="cuda")[:14]
    off = torch.tensor([0, 7, 14], dtype=torch.int64, device="cuda")

    def refused(n_keep, n_sink, n_recent, max_len=300, ids=free, dst=off, w=mass, src=c.page_ids):
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_kv_evict(c.k, c.v, src, c.page_off, c.kv_len, w, ids, dst, n_keep, n_sink, n_recent, max_len)
        assert e.value.name == "PTC_ERR_INVALID_ARG"

    refused(0, 0, 0)
    refused(100, 60, 41)
    refused(100, 4, 10, max_len=299)
    refused(113, 4, 10)                                           # seven pages hold 112
    refused(100, 4, 10, dst=torch.tensor([0, 7, 15], dtype=torch.int64, device="cuda"))
    refused(100, 4, 10, ids=free + c.n_pages)
    refused(100, 4, 10, src=c.page_ids + c.n_pages)
    refused(100, 4, 10, w=mass[:, :-1].contiguous())
    with pytest.raises(ValueError):
        ptc.ptc_kv_evict(c.k, c.v, c.page_ids, c.page_off, c.kv_len, mass.double(), free, off, 100, 4, 10, 300)
    with pytest.raises(ValueError):
        ptc.ptc_kv_evict(c.k, c.v, c.page_ids, c.page_off, c.kv_len, mass, free, off, 100, -1, 10, 300)
    keep, new_len, _ = ptc.ptc_kv_evict(c.k, c.v, c.page_ids, c.page_off, c.kv_len, mass, free, off, 100, 4, 10, 300)
    assert new_len.tolist() == [100, 90]


# ---------------------------------------------------------------- together
def test_attention_over_an_evicted_cache():
    """What is kept is a paged cache again: attention over it is attention
    over the kept tokens."""
    import torch
    from tests.kv_util import Cache, check_attention
    c = Cache([(0, 900), (0, 70), (0, 300)], Hq=8, Hkv=2, D=128)
    k, v, ids, off, new_len, new_mass = evict(c, weights(c, "spread"), 128, 4, 32)
    lens = [(1, int(n)) for n in new_len]
    d = Cache(lens, Hq=8, Hkv=2, D=128)
    d.k, d.v, d.page_ids, d.page_off, d.n_pages = k, v, ids, off, k.shape[0]
    d.lists = [ids[int(a):int(b)] for a, b in zip(off[:-1], off[1:])]
    d.keys, d.vals, d.slots = [], [], new_mass.shape[1]
    for r, (_, n) in enumerate(lens):
        page, slot = d.where(r, n)
        d.keys.append(k[page, :, slot])
        d.vals.append(v[page, :, slot])
    check_attention(d, mass=new_mass)


def test_example_replays_a_trace():
    """examples/serve_trace.py: block ids as page lists, append, attention and
    eviction over a small trace, checked inside against a dense computation."""
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "serve_trace.py"), "--requests", "12", "--check"],
                       capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "checked" in r.stdout
