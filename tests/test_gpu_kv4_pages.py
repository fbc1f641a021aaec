"""Attention over pages of 4 bits: ids of pages that the cache does not have are
refused wherever a token needs them, the one with all bits set among them."""
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
