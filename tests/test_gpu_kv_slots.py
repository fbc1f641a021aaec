"""Slots of weights that belong to no request of the call: a page list may be
longer than the requests' part of it, before and behind, and the weights longer
than the page list.  There the accumulated weights are what they were, and after
an eviction zero, so that a list that grows into them goes on from there."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


def within(c, first, more):
    """The cache's lists inside a longer one: `first` pages before, `more` behind."""
    import torch
    pad = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")
    return torch.cat([pad(first), c.page_ids, pad(more)]), c.page_off + first


LENS = [[(1, 100), (1, 40)], [(60, 300), (0, 30), (1, 9)], [(0, 50)]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("first,more,wide", [(3, 0, 0), (0, 5, 0), (2, 70, 0), (90, 1, 0), (0, 0, 24), (1, 1, 9)])
@pytest.mark.parametrize("B", [16, 6])
def test_attention(lens, first, more, wide, B):
    """`wide`: slots of the weights behind those of the page list."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache(lens, Hq=8, Hkv=2, D=64, B=B)
    ids, off = within(c, first, more)
    n, a, b = ids.numel() * B + wide, first * B, first * B + c.slots
    mass = torch.rand(2, n, generator=c.g, device="cuda")
    call = lambda **k: ptc.ptc_paged_attention(c.q, c.k, c.v, ids, off, c.tok_off, c.kv_len, max(c.new), **k)[2]
    torch.full((2, n), math.nan, device="cuda")  # what the allocator hands out next
    fresh = call(mass=mass)
    assert torch.equal(fresh[:, :a], mass[:, :a]) and torch.equal(fresh[:, b:], mass[:, b:])
    # the requests' slots are those of a call on their own list
    alone = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), mass=mass[:, a:b].contiguous())[2]
    assert torch.equal(fresh[:, a:b], alone)
    for given in (torch.full_like(mass, math.nan), mass.clone()):
        kept = given if torch.equal(given, mass) else mass
        assert call(mass=kept, mass_out=given) is given and torch.equal(given, fresh)
    none = call(mass_out=torch.full_like(mass, math.nan))
    assert not none[:, :a].any() and not none[:, b:].any()


def test_attention_without_requests():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([], Hkv=2)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    mass = torch.rand(2, 64, device="cuda")
    torch.full((2, 64), math.nan, device="cuda")
    _, _, got = ptc.ptc_paged_attention(c.q, c.k, c.v, ids, c.page_off, c.tok_off, c.kv_len, 0, mass=mass)
    assert got is not mass and torch.equal(got, mass)


@pytest.mark.parametrize("first,more", [(3, 0), (0, 5), (2, 70)])
def test_eviction(first, more):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(0, 300), (0, 90)], Hq=2, extra_pages=40)
    used = set(c.page_ids.tolist())
    free = torch.tensor([p for p in range(c.n_pages) if p not in used], dtype=torch.int32, device="cuda")[:14]
    pad = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")
    ids = torch.cat([pad(first), free, pad(more)])
    off = first + torch.tensor([0, 7, 14], dtype=torch.int64, device="cuda")
    mass = torch.rand(c.Hkv, c.slots, generator=c.g, device="cuda") + 1
    call = lambda i, o: ptc.ptc_kv_evict(c.k, c.v, c.page_ids, c.page_off, c.kv_len, mass, i, o, 100, 4, 10, 300)
    want = call(free, off - first)[2]
    torch.full((c.Hkv, ids.numel() * c.B), math.nan, device="cuda")
    got = call(ids, off)[2]
    a, b = first * c.B, (first + 14) * c.B
    assert torch.equal(got[:, a:b], want)
    assert not got[:, :a].any() and not got[:, b:].any()


def test_eviction_without_requests():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([], Hkv=2)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    torch.full((2, 64), math.nan, device="cuda")
    keep, new_len, got = ptc.ptc_kv_evict(c.k, c.v, c.page_ids, c.page_off, c.kv_len, torch.zeros(2, 0, device="cuda"), ids,
                                          c.page_off, 4, 1, 1, 10)
    assert keep.shape == (0, 2, 4) and new_len.shape == (0,) and got.shape == (2, 64) and not got.any()
