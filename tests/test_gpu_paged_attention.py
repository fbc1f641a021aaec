"""ptc_paged_attention against its definition in 64 bits: chunks, single
tokens and both mixed, head groups, widths, page sizes, layouts and types;
masks that leave rows empty; what lies in slots that hold no token; the
accumulated weights; streams, graphs and refusals."""
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


def cache(*a, **k):
    from tests.kv_util import Cache
    return Cache(*a, **k)


def check(c, with_mass=False, **k):
    import torch
    from tests.kv_util import check_attention
    mass = None
    if with_mass:
        mass = torch.rand(c.Hkv, c.slots, generator=c.g, device="cuda")
        for r, (m, n) in enumerate(c.lens):
            a, b = int(c.page_off[r]) * c.B, int(c.page_off[r + 1]) * c.B
            mass[:, a + max(n - m, 0):b] = 0
    return check_attention(c, mass, **k)


LENS = {
    "one": [(1, 1)],
    "decode": [(1, 5), (1, 128), (1, 129), (1, 1000), (1, 127)],
    "few": [(2, 300), (5, 5), (31, 64), (33, 500)],
    "chunk": [(200, 200), (129, 400)],
    "edges": [(127, 127), (128, 128), (129, 129), (255, 255), (256, 256), (257, 257), (64, 320), (63, 319), (65, 321)],
    "mixed": [(1, 700), (300, 300), (0, 40), (1, 1), (0, 0), (70, 1500), (2, 2)],
    "empty rows": [(5, 2), (4, 0), (300, 10), (1, 0), (200, 150), (40, 41)],
}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (7, 1), (6, 2), (15, 3)])
def test_lengths_and_groups(lens, heads):
    check(cache(LENS[lens], Hq=heads[0], Hkv=heads[1], D=64), with_mass=True)


@pytest.mark.parametrize("D", [16, 24, 40, 64, 72, 80, 96, 104, 120, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_widths(D, dtype):
    check(cache([(1, 333), (150, 270), (3, 3)], D=D, dtype=dtype), with_mass=True)


@pytest.mark.parametrize("B", [1, 2, 7, 8, 12, 16, 24, 32, 48, 64, 100, 128, 200, 256, 384, 512])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_page_sizes(B, layout):
    check(cache([(1, 777), (140, 600), (2, 3)], D=128, B=B, layout=layout), with_mass=True)


@pytest.mark.parametrize("group", [1, 2, 3, 8, 16, 31, 64, 100])
def test_head_groups(group):
    check(cache([(1, 260), (3, 140), (9, 9), (50, 300)], Hq=2 * group, Hkv=2, D=128), with_mass=True)


def test_long_contexts_split_over_the_gpu():
    check(cache([(1, 40_000)], Hq=8, Hkv=2, D=128), with_mass=True)
    check(cache([(3, 20_001), (1, 12_345)], Hq=8, Hkv=1, D=128, dtype="fp16"), with_mass=True)
    check(cache([(130, 9000)], Hq=4, Hkv=1, D=128), with_mass=True)


def test_many_requests():
    lens = [(1 + (7 * r) % 3, 20 + (37 * r) % 400) for r in range(1500)]
    check(cache(lens, Hq=4, Hkv=2, D=64), with_mass=True)


def test_long_chunk():
    check(cache([(1500, 2300), (700, 700)], Hq=8, Hkv=2, D=128), with_mass=True)


def test_shared_prefix_pages():
    check(cache([(1, 500), (1, 333), (40, 400), (1, 257)], Hq=8, Hkv=2, D=128, shared=256), with_mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("q_scale", [0.0, 1e-3, 20.0])
def test_flat_and_peaked_scores(dtype, q_scale):
    """All scores alike, and scores whose largest takes all the weight."""
    check(cache([(1, 900), (130, 500)], Hq=4, Hkv=2, D=128, dtype=dtype, q_scale=q_scale), with_mass=True)


def test_rising_scores():
    """The running maximum rises with every key."""
    import torch
    c = cache([(1, 2000), (140, 900)], Hq=4, Hkv=2, D=64)
    for r, n in enumerate(c.total):
        ramp = torch.linspace(-1, 1, n, device="cuda")[:, None, None]
        c.keys[r] = (ramp * 3 + 0.01 * c.keys[r].float()).to(c.dt)
        c.put(r, c.keys[r], c.vals[r])
    c.q = c.q.abs()
    check(c, with_mass=True)


def test_scale_is_used():
    check(cache([(1, 100), (60, 100)]), scale=0.37)


def test_query_strides_and_outputs_given():
    import torch
    c = cache([(1, 100), (60, 150)], Hq=6, Hkv=3, D=40)
    wide = torch.full((c.q.shape[0], 9, 56), math.nan, dtype=c.dt, device="cuda")
    wide[:, 2:8, 8:48] = c.q
    c.q = wide[:, 2:8, 8:48]
    out = torch.empty(c.q.shape, dtype=c.dt, device="cuda")
    lse = torch.empty(c.q.shape[:2], dtype=torch.float32, device="cuda")
    got = check(c, out=out, lse=lse)
    assert got[0] is out and got[1] is lse


def test_pages_past_32_bit_offsets():
    """Elements of the last pages lie beyond 2^32 bytes and 2^31 elements."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import close, reference
    c = cache([(1, 400), (150, 300)], Hq=4, Hkv=2, D=128, B=16)
    far = 600_000
    k = torch.empty((far + c.n_pages, 2, 16, 128), dtype=c.dt, device="cuda")
    v = torch.empty_like(k)
    k[far:], v[far:] = c.k, c.v
    out, lse = ptc.ptc_paged_attention(c.q, k, v, c.page_ids + far, c.page_off, c.tok_off, c.kv_len, 150)
    want = reference(c)
    close(out, want[0], want[3])
    close(lse, want[1], want[4])


def test_mass_starts_from_nothing_and_in_place():
    import torch
    import paper_2609_28870_gb300 as ptc
    c = cache([(1, 300), (129, 200), (0, 50), (0, 0)], Hq=8, Hkv=2)
    call = lambda **k: ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 129, **k)
    fresh = torch.full((c.Hkv, c.slots), math.nan, device="cuda")
    _, _, a = call(mass_out=fresh)
    assert a is fresh
    zero = torch.zeros_like(fresh)
    _, _, b = call(mass=zero, mass_out=zero)
    assert b is zero and torch.equal(a, b)
    _, _, two = call(mass=b.clone())
    assert torch.allclose(two, 2 * b, rtol=1e-6, atol=0)


def test_same_bytes_twice_and_on_another_stream():
    import torch
    import paper_2609_28870_gb300 as ptc
    c = cache([(1, 9000), (300, 1500), (7, 7)], Hq=8, Hkv=2, D=128)
    mass = torch.rand(c.Hkv, c.slots, device="cuda")
    run = lambda **k: ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 300, mass=mass, **k)
    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        second = run(status=status)
        ptc.check_status(status)
    for x, y in zip(first, second):
        assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))


def test_graph_replay_reads_new_lengths():
    """A captured call follows the lengths and pages of the replay."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import close, reference
    c = cache([(1, 500), (1, 900)], Hq=8, Hkv=2, D=128)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(ptc.lib().ptc_paged_attention_workspace_bytes(2, 8, 2, 128, 1, 0), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(c.q)
    lse = torch.empty(c.q.shape[:2], dtype=torch.float32, device="cuda")
    run = lambda: ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 1, out=out, lse=lse, ws=ws, status=status)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens in ([(1, 500), (1, 900)], [(1, 77), (1, 640)]):
        c.lens, c.total = lens, [n for _, n in lens]
        c.kv_len.copy_(torch.tensor(c.total, dtype=torch.int32))
        full = (list(c.keys), list(c.vals))
        c.keys, c.vals = [k[:n] for k, n in zip(c.keys, c.total)], [v[:n] for v, n in zip(c.vals, c.total)]
        out.zero_()
        graph.replay()
        ptc.check_status(status)
        want = reference(c)
        close(out, want[0], want[3])
        close(lse, want[1], want[4])
        c.keys, c.vals = full


def test_nothing_to_do():
    import torch
    import paper_2609_28870_gb300 as ptc
    c = cache([(0, 40), (0, 0)])
    out, lse = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 0)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    c = cache([])
    ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 0)
    torch.cuda.synchronize()


def test_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    c = cache([(1, 100), (60, 100)], D=64)
    args = lambda **o: [o.get(x, getattr(c, x)) for x in ("q", "k", "v", "page_ids", "page_off", "tok_off", "kv_len")]

    def refused(*a, name="PTC_ERR_INVALID_ARG", **k):
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_paged_attention(*a, **k)
        assert e.value.name == name

    i64 = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    refused(*args(), 59)                                            # a chunk longer than max_q_len
    refused(*args(tok_off=i64([0, 62, 61])), 62)                    # offsets that fall
    refused(*args(tok_off=i64([0, 1, 60])), 60)                     # tokens left over
    refused(*args(tok_off=i64([1, 1, 61])), 60)
    refused(*args(kv_len=i32([100, 10_000])), 60)                   # more tokens than pages
    refused(*args(page_off=i64([0, 9, 8])), 60)
    refused(*args(page_off=i64([0, 8, 1 << 40])), 60)
    bad = c.page_ids.clone()
    bad[3] = c.n_pages
    refused(*args(page_ids=bad), 60)                                # a page that the cache does not have
    bad[3] = -1
    refused(*args(page_ids=bad), 60)
    for scale in (0.0, -1.0, math.inf, math.nan):
        refused(*args(), 60, scale=scale)
    refused(*args(q=c.q[:, :3].contiguous()), 60)                   # 3 query heads on 2 key heads
    odd = torch.zeros(c.q.shape[0] * 4 * 64 + 1, dtype=c.dt, device="cuda")[1:].view(-1, 4, 64)
    refused(*args(q=odd), 60)                                       # 2-byte alignment
    refused(*args(), 60, ws=None, mass=torch.zeros(2, c.slots - c.B, device="cuda"))
    wide = torch.zeros(c.n_pages, 2, 16, 68, dtype=c.dt, device="cuda")[..., :64]
    refused(*args(k=wide), 60)                                      # strides that are no multiple of 8
    for o in (dict(q=c.q.float()), dict(v=c.v[:-1]), dict(k=c.k.half()), dict(page_ids=c.page_ids.long()),
              dict(kv_len=c.kv_len[:1])):
        with pytest.raises(ValueError):
            ptc.ptc_paged_attention(*args(**o), 60)
    # stream-ordered: the word takes the code, later calls leave it, the data stays usable
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ptc.ptc_paged_attention(*args(page_ids=bad), 60, status=status)
    ptc.ptc_paged_attention(*args(), 60, status=status)
    with pytest.raises(ptc.PtcError):
        ptc.check_status(status)
    ptc.check_status(status)
    check(c)
