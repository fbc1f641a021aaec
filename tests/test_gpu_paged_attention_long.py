"""ptc_paged_attention of requests of many new tokens, which pairs of CTAs take
through the same keys, against the definition in 64 bits: lengths about the
limit from which they do and about the ends of their tiles, alone and beside
requests that are not theirs, contexts split over pairs, page sizes, types."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


def check(lens, **k):
    import torch
    from tests.kv_util import Cache, check_attention
    c = Cache(lens, **k)
    mass = torch.rand(c.Hkv, c.slots, generator=c.g, device="cuda")
    for r, (m, n) in enumerate(c.lens):
        a, b = int(c.page_off[r]) * c.B, int(c.page_off[r + 1]) * c.B
        mass[:, a + max(n - m, 0):b] = 0
    return check_attention(c, mass)


@pytest.mark.parametrize("m", [255, 256, 257, 288, 319, 320, 321, 384, 385, 511, 512, 513, 700])
def test_lengths_about_the_limit_and_the_tiles(m):
    """Four heads a group: halves of 32 tokens, tiles of 64, of a pair 128."""
    check([(m, m)], Hq=8, Hkv=2)
    check([(m, m + 77)], Hq=4, Hkv=1, D=128)


@pytest.mark.parametrize("group,m", [(1, 1030), (2, 600), (3, 400), (5, 260), (7, 200), (16, 100), (31, 60), (64, 40),
                                     (100, 20), (128, 9), (128, 33)])
def test_head_groups(group, m):
    check([(m, m + 300), (m + 1, m + 1)], Hq=2 * group, Hkv=2, D=64)


@pytest.mark.parametrize("lens", [
    [(1, 500), (300, 300), (1, 90), (400, 2000), (0, 10), (64, 64), (2, 700)],
    [(300, 900), (1, 1), (0, 0), (0, 0), (257, 257)],
    [(0, 3), (1, 1000), (290, 290)],
    [(20, 20), (260, 100), (300, 0), (256, 256), (330, 331)],
])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_beside_requests_that_are_not_the_pairs(lens, dtype):
    check(lens, Hq=8, Hkv=2, D=128, dtype=dtype)


@pytest.mark.parametrize("B", [7, 8, 16, 24, 48, 64, 128, 192, 512])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_page_sizes(B, layout):
    check([(300, 777), (1, 400)], Hq=4, Hkv=1, D=128, B=B, layout=layout)


@pytest.mark.parametrize("D", [16, 40, 64, 72, 120])
def test_widths(D):
    check([(270, 1000), (5, 40)], Hq=4, Hkv=1, D=D)


def test_long_contexts_split_over_pairs():
    check([(257, 30_000)], Hq=4, Hkv=1, D=128)
    check([(1025, 9000)], Hq=2, Hkv=2, D=128, dtype="fp16")
    check([(300, 12_000), (1, 8000), (280, 5000)], Hq=8, Hkv=2, D=64)


def test_a_limit_above_the_lengths():
    """max_q_len promises more tokens than any request has."""
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, close, reference
    for lens in ([(200, 300)], [(200, 300), (100, 100)], [(300, 300), (5, 9)]):
        c = Cache(lens, Hq=8, Hkv=2, D=128)
        out, lse = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 5000)
        want = reference(c)
        close(out, want[0], want[3])
        close(lse, want[1], want[4])


def test_captured_and_replayed():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, close, reference
    c = Cache([(300, 1200), (1, 700), (513, 513)], Hq=8, Hkv=2, D=128)
    want = reference(c)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty(c.q.shape, dtype=c.dt, device="cuda")
    lse = torch.empty(c.q.shape[:2], dtype=torch.float32, device="cuda")
    run = lambda: ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 513, out=out, lse=lse, status=status)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        out.zero_()
        lse.zero_()
        g.replay()
        torch.cuda.synchronize()
        close(out, want[0], want[3])
        close(lse, want[1], want[4])
    ptc.check_status(status, "attention")


# From here on the requests have at least eight query tiles (of 256 rows) on
# average and more than 64 columns, without which no pair is formed.


@pytest.mark.parametrize("m", [1, 63, 64, 65, 127, 128, 129, 191, 192, 193])
def test_ends_of_a_pairs_last_tile(m):
    """Four heads a group: a pair's tile is 128 tokens."""
    check([(1024 + m, 1024 + m)], Hq=4, Hkv=1, D=128)
    check([(512 + m, 512 + m + 1000)], Hq=8, Hkv=2, D=96, dtype="fp16")


@pytest.mark.parametrize("group,m", [(1, 2100), (2, 1100), (3, 700), (5, 450), (7, 300), (16, 140), (31, 70), (64, 37),
                                     (100, 20), (128, 17), (128, 40)])
def test_pairs_by_head_groups(group, m):
    check([(m, m + 300), (m + 1, m + 1)], Hq=2 * group, Hkv=2, D=128)


@pytest.mark.parametrize("lens", [
    [(1500, 1500), (1, 500), (255, 300), (256, 256), (257, 900), (1100, 1101)],
    [(0, 0), (1400, 3000), (0, 10), (200, 200)],
    [(1, 1000), (2000, 2000), (3, 4)],
    [(1300, 100), (900, 0), (700, 701), (60, 400)],
    [(600, 600)] * 7,
])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_pairs_beside_other_requests(lens, dtype):
    """Requests of up to four query tiles, empty ones and rows that see no key."""
    check(lens, Hq=8, Hkv=2, D=128, dtype=dtype)


@pytest.mark.parametrize("B", [8, 16, 24, 32, 40, 48, 64, 96, 128, 192, 256, 512])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_pairs_by_page_sizes(B, layout):
    check([(700, 1777), (520, 520)], Hq=4, Hkv=1, D=128, B=B, layout=layout)


@pytest.mark.parametrize("B", [7, 12, 100])
def test_pages_without_tensor_copies(B):
    check([(700, 1777)], Hq=4, Hkv=1, D=128, B=B)


@pytest.mark.parametrize("D", [72, 80, 104, 120])
def test_pairs_by_widths(D):
    check([(600, 1000), (520, 4000)], Hq=4, Hkv=1, D=D)


def test_pairs_over_many_requests():
    """More requests than the plan keeps in shared memory, all of them pairs';
    every 37th and the last are compared."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, close, reference
    c = Cache([(17 + r % 5, 20 + r % 40) for r in range(1200)], Hq=128, Hkv=1, D=72)
    out, lse = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 21)
    assert torch.isfinite(out).all() and not torch.isnan(lse).any()
    some = [r for r in range(1200) if r % 37 == 0 or r == 1199]
    c.lens = [x if r in some else (0, 0) for r, x in enumerate(c.lens)]
    want = reference(c)
    rows = torch.cat([torch.arange(int(c.tok_off[r]), int(c.tok_off[r + 1])) for r in some]).cuda()
    close(out[rows], want[0][rows], want[3][rows])
    close(lse[rows], want[1][rows], want[4][rows])


def test_pairs_with_pages_that_the_cache_does_not_have():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(600, 900)], Hq=4, Hkv=1, D=128)
    ids = c.page_ids.clone()
    ids[3] = c.n_pages
    with pytest.raises(ptc.PtcError):
        ptc.ptc_paged_attention(c.q, c.k, c.v, ids, c.page_off, c.tok_off, c.kv_len, 600)
    short = c.tok_off.clone()
    short[0] = 1
    with pytest.raises(ptc.PtcError):
        ptc.ptc_paged_attention(c.q, *c.table()[:2], c.page_ids, c.page_off, short, c.kv_len, 600)
    out, _ = ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, 600)
    assert torch.isfinite(out).all()
