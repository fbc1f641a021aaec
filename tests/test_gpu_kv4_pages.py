"""Attention over pages of 4 bits: ids of pages that the cache does not have are
refused wherever a token needs them, the one with all bits set among them; pages
that nothing needs are not worked on."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


# Requests (new, total), and page sizes.  By 4 query heads a key head: requests of few
# rows, of more, and (from 512 new tokens on, pages of 16) over a copy in 16 bits.
CALLS = {
    "few": ([(1, 100), (3, 50), (1, 1)], 16),
    "few, pages of 12": ([(1, 100), (3, 50), (1, 1)], 12),
    "few, long": ([(1, 5000)], 16),
    "few, pages of 256": ([(8, 700)], 256),
    "tiles": ([(40, 300), (1, 50)], 16),
    "tiles, pages of 12": ([(40, 300), (1, 50)], 12),
    "copy": ([(520, 700), (1, 50)], 16),
}


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "fp16")])
@pytest.mark.parametrize("name", CALLS)
def test_pages_that_the_cache_does_not_have(name, D, dtype):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, check_attention4
    lens, B = CALLS[name]
    c = Cache4(lens, Hq=8, Hkv=2, D=D, B=B, dtype=dtype)
    good, status = c.page_ids.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    off = c.page_off.tolist()
    for r, n in enumerate(c.total):
        needed = -(-n // B)
        for i in range(needed) if needed < 30 else (0, 1, needed // 2, needed - 2, needed - 1):
            for bad in (c.n_pages, -1, -2, -2 ** 31):
                c.page_ids.copy_(good)
                c.page_ids[off[r] + i] = bad
                ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), status=status)
                assert int(status) == 1, f"request {r}, page {i}, id {bad}"
                status.zero_()
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new))
        assert e.value.name == "PTC_ERR_INVALID_ARG"
    # ids behind a request's tokens are not needed
    c.page_ids.copy_(good)
    for r, n in enumerate(c.total):
        c.page_ids[off[r] + -(-n // B):off[r + 1]] = -1
    check_attention4(c)


@pytest.mark.parametrize("D", [128, 64])
def test_a_chunk_beside_requests_without_new_tokens(D):
    """The copy in 16 bits at the workspace's end (keys, then values, a page an entry of
    the lists) has the pages of requests with new tokens, and those alone; what the
    others' lists hold does not matter."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, check_attention4
    c = Cache4([(0, 400), (600, 700), (0, 90), (1, 50), (0, 0), (0, 33)], Hq=8, Hkv=2, D=D)
    n, page, off = c.page_ids.shape[0], 2 * c.B * 2 * D, c.page_off.tolist()
    size = lambda B: ptc.lib().ptc_kv4_attention_workspace_bytes(6, 8, 2, D, 600, 601, n, B)
    need, copy = size(16), -(-n * page // 256) * 256
    assert need == size(12) + -(-4 * n // 256) * 256 + 2 * copy  # (there is no copy of pages of 12)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    check_attention4(c, ws=ws)
    made = [(x[:n * page].view(n, page) != 255).any(1).cpu() for x in (ws[need - 2 * copy:need - copy], ws[need - copy:])]
    want = torch.zeros(n, dtype=torch.bool)
    for r, (m, total) in enumerate(c.lens):
        if m:
            want[off[r]:off[r] + -(-total // c.B)] = True
    assert all(torch.equal(x, want) for x in made)
    for r, (m, _) in enumerate(c.lens):
        if not m:
            c.page_ids[off[r]:off[r + 1]] = -1
    check_attention4(c, ws=ws)


def test_a_cache_without_slots_is_refused():
    import torch
    import paper_2609_28870_gb300 as ptc
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    i64 = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    k, v = (torch.zeros(3, 2, 0, 80, dtype=torch.uint8, device="cuda") for _ in range(2))
    for T in (1, 4096):
        q = torch.zeros(T, 8, 128, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_kv4_attention(q, k, v, i32([0, 1]), i64([0, 2]), i64([0, T]), i32([T]), T)
        assert e.value.name == "PTC_ERR_INVALID_ARG"
