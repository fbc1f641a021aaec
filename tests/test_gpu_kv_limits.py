"""The calls on paged keys and values at the ends of their ranges: slices of the
eviction that shared memory does not hold, the largest head group, more
requests than a CTA looks at, pages past 32-bit offsets, broadcast inputs."""
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


@pytest.mark.parametrize("kind", ["spread", "zeros", "close"])
def test_evict_from_weights_read_in_every_pass(kind):
    """400,000 tokens: slices of 50,000, more than shared memory holds."""
    from tests.kv_util import Cache
    from tests.test_gpu_kv import evict, weights
    c = Cache([(0, 400_000), (0, 3), (0, 20_000)], Hq=1, Hkv=1, D=16, B=64)
    evict(c, weights(c, kind), 6000, 5, 100)


def test_evict_and_append_many_requests():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    from tests.test_gpu_kv import bits, evict, weights
    c = Cache([(0, 1 + (13 * r) % 90) for r in range(1300)], Hq=2, Hkv=2, D=16)
    evict(c, weights(c, "ties"), 40, 3, 10)
    lens = [((5 * r) % 4, 4 + (13 * r) % 90) for r in range(1300)]
    c = Cache(lens, Hq=2, Hkv=2, D=16)
    k_new = torch.cat([k[n - m:] for k, (m, n) in zip(c.keys, lens)])
    v_new = torch.cat([v[n - m:] for v, (m, n) in zip(c.vals, lens)])
    want_k, want_v = bits(c.k).clone(), bits(c.v).clone()
    for r, (m, n) in enumerate(lens):
        page, slot = c.where(r, n)
        c.k[page[n - m:], :, slot[n - m:]] = math.nan
        c.v[page[n - m:], :, slot[n - m:]] = math.nan
    ptc.ptc_kv_append(k_new, v_new, *c.table(), c.tok_off, c.kv_len)
    assert torch.equal(bits(c.k), want_k) and torch.equal(bits(c.v), want_v)


def test_append_and_evict_past_32_bit_offsets():
    import torch
    import paper_2609_28870_gb300 as ptc
    far, H, B, D = 300_000, 4, 16, 128
    k = torch.zeros((far + 80, H, B, D), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    ids = far + torch.arange(40, dtype=torch.int32, device="cuda")
    i64 = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    n = 600
    kn = torch.randn(n, H, D, device="cuda").half()
    vn = torch.randn(n, H, D, device="cuda").half()
    ptc.ptc_kv_append(kn, vn, k, v, ids, i64([0, 40]), i64([0, n]), i32([n]))
    rows = lambda x, first: x[far + first:].transpose(1, 2).reshape(-1, H, D)
    assert torch.equal(rows(k, 0)[:n], kn) and torch.equal(rows(v, 0)[:n], vn)
    mass = torch.rand(H, 40 * B, device="cuda")
    keep, new_len, _ = ptc.ptc_kv_evict(k, v, ids, i64([0, 40]), i32([n]), mass, ids + 40, i64([0, 40]), 100, 1, 2, n)
    got_k, got_v = rows(k, 40), rows(v, 40)
    for h in range(H):
        kept = keep[0, h].long()
        assert torch.equal(got_k[:100, h], kn[kept, h]) and torch.equal(got_v[:100, h], vn[kept, h])


@pytest.mark.parametrize("group", [127, 128])
def test_the_largest_head_groups(group):
    from tests.test_gpu_paged_attention import cache, check
    check(cache([(1, 260), (3, 140), (40, 300)], Hq=group, Hkv=1, D=64), with_mass=True)


def test_broadcast_inputs_are_refused():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(3, 50)], Hq=4, Hkv=4)
    one = torch.zeros(3, 1, 64, dtype=c.dt, device="cuda")
    with pytest.raises(ptc.PtcError) as e:
        ptc.ptc_paged_attention(one.expand(3, 4, 64), *c.table(), c.tok_off, c.kv_len, 3)
    assert e.value.name == "PTC_ERR_INVALID_ARG"
    with pytest.raises(ptc.PtcError) as e:
        ptc.ptc_kv_append(one.expand(3, 4, 64), one.expand(3, 4, 64), *c.table(), c.tok_off, c.kv_len)
    assert e.value.name == "PTC_ERR_INVALID_ARG"


def test_dimensions_of_one_may_have_any_stride():
    """One token, one head, one page: strides that are never used."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, close, reference
    c = Cache([(1, 9)], Hq=1, Hkv=1, B=16, D=64, spare=0, extra_pages=0)
    odd = lambda x, s: torch.as_strided(x, x.shape, s)
    k, v = odd(c.k.contiguous(), (3, 5, 64, 1)), odd(c.v.contiguous(), (0, 7, 64, 1))
    q = odd(c.q.contiguous(), (1, 3, 1))
    out, lse = ptc.ptc_paged_attention(q, k, v, c.page_ids, c.page_off, c.tok_off, c.kv_len, 1)
    want = reference(c)
    close(out, want[0], want[3])
    close(lse, want[1], want[4])


def test_weights_with_rows_between_both_ways():
    """16 rows a request keep their scores, 17 have them computed again; the
    sums agree to their rounding."""
    from tests.test_gpu_paged_attention import cache, check
    for m in (4, 5):
        check(cache([(m, 700), (1, 129), (0, 40), (m, m)], Hq=8, Hkv=2, D=128), with_mass=True)
