"""Counts that 32 bits do not hold are refused by the binding: the C calls take
them as 32-bit numbers, and a wrapped one would be a different question.  No
GPU is needed: the library is a recorder and the tensors' device is faked."""
import pytest
import torch

import paper_2609_28870_gb300 as ptc
from tests.test_current_device import current, lib, on1, paged  # noqa: F401


@pytest.mark.parametrize("max_q_len", [-1, 1 << 32, (1 << 32) + 1])
def test_max_q_len(monkeypatch, lib, max_q_len):  # noqa: F811
    t, tok, n, x = paged()
    current(monkeypatch, 1)
    with pytest.raises(ValueError, match="max_q_len"):
        ptc.ptc_paged_attention(x, *t, tok, n, max_q_len)
    assert lib.calls == []
    for fine in (0, 1, (1 << 32) - 1):
        ptc.ptc_paged_attention(x, *t, tok, n, fine)


@pytest.mark.parametrize("which", ["n_sink", "n_recent", "max_kv_len"])
@pytest.mark.parametrize("value", [-1, 1 << 32, (1 << 32) + 1])
def test_eviction(monkeypatch, lib, which, value):  # noqa: F811
    t, tok, n, x = paged()
    current(monkeypatch, 1)
    args = dict(n_keep=4, n_sink=1, n_recent=1, max_kv_len=16)
    with pytest.raises(ValueError, match="max_kv_len"):
        ptc.ptc_kv_evict(*t, n, on1(torch.zeros(1, 16)), t[2], t[3], **{**args, which: value})
    assert lib.calls == []
    ptc.ptc_kv_evict(*t, n, on1(torch.zeros(1, 16)), t[2], t[3], **args)
    assert lib.calls == ["ptc_kv_evict"]
