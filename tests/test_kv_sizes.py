"""Sizes of ptc_paged_attention whose products would wrap around 64 bits are
refused on the host, before any CUDA call."""
from tests.test_kv_abi import FAKE, L, OVERFLOW, paged, strides  # noqa: F401


def attend(L, slots, max_q=1, heads=8, **o):
    return L.ptc_paged_attention(paged(**o), FAKE, strides(), FAKE, 3, heads, max_q, 0.1, FAKE, FAKE, None, FAKE, slots,
                                 FAKE, 1 << 40, None, None)


def test_a_stride_of_the_weights_that_wraps(L):  # noqa: F811
    # with one key head the stride is of no row, so any array could have it; the
    # scores of few rows are kept at this stride
    assert attend(L, (1 << 62) + 320, heads=4, n_kv_heads=1) == OVERFLOW
    assert attend(L, (1 << 61) + 320) == OVERFLOW
    assert attend(L, (1 << 64) - 1, heads=1, n_kv_heads=1) == OVERFLOW
    assert attend(L, (1 << 40) + 1, max_q=100) == OVERFLOW


def test_a_page_count_that_wraps(L):  # noqa: F811
    for pages, B in ((1 << 60, 16), ((1 << 60) + 1, 16), (1 << 55, 512), ((1 << 38) + 1, 1)):
        assert L.ptc_paged_attention(paged(n_page_ids=pages, block_size=B), FAKE, strides(), FAKE, 3, 8, 1, 0.1, FAKE, FAKE,
                                     None, None, 0, FAKE, 1 << 40, None, None) == OVERFLOW
