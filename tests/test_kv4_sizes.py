"""Workspace sizes of the calls on pages of 4 bits, asked for before a cache is
checked: any numbers have one."""
import itertools

import pytest

import paper_2609_28870_gb300 as ptc


@pytest.fixture(scope="module")
def L():
    from paper_2609_28870_gb300 import build
    build.build()
    return ptc.lib()


@pytest.mark.parametrize("bad", [dict(block_size=0), dict(head_dim=0), dict(n_kv_heads=0), dict(n_q_heads=0),
                                 dict(block_size=1 << 31, n_kv_heads=1 << 31, n_q_heads=1 << 31, max_q_len=1 << 31),
                                 dict(block_size=0, n_tok=(1 << 64) - 1, n_page_ids=(1 << 64) - 1)], ids=str)
def test_attention_workspace_of_sizes_that_no_cache_has(L, bad):
    size = dict(n_req=1, n_q_heads=8, n_kv_heads=2, head_dim=128, max_q_len=4096, n_tok=4096, n_page_ids=300, block_size=16)
    copied = L.ptc_kv4_attention_workspace_bytes(*size.values())
    size.update(bad)
    assert 0 < L.ptc_kv4_attention_workspace_bytes(*size.values()) < copied  # no room for a copy


def test_attention_workspace_at_the_ends_of_every_argument(L):
    u32, u64 = (0, 1, 0xFFFFFFFE), (0, 1 << 20, (1 << 64) - 1)
    for a in itertools.product(u32, u32, u32, (0, 128), u32, u64, u64, (0, 16, 0xFFFFFFF8)):
        L.ptc_kv4_attention_workspace_bytes(*a)
