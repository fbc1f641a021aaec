"""A workspace that the caller gives is used only where it is as many bytes as
it says: an expanded tensor has more elements than memory."""
import pytest
import torch

import paper_2609_28870_gb300 as ptc
from paper_2609_28870_gb300 import kv

NEED = 4096


def room(ws):
    return [ptc._workspace(NEED, torch.device("cpu"), ws), kv._room(torch.zeros(1), NEED, -1, ws)]


@pytest.mark.parametrize("ws", [torch.empty(1, dtype=torch.uint8).expand(2 * NEED),
                                torch.empty(64, dtype=torch.uint8).expand(2 * NEED // 64, 64),
                                torch.empty(4 * NEED, dtype=torch.uint8)[::2]], ids=["one", "rows", "strided"])
def test_a_workspace_with_strides_is_not_used(ws):
    for w in room(ws):
        assert w.data_ptr() != ws.data_ptr()
        assert w.is_contiguous() and w.numel() >= NEED and w.untyped_storage().nbytes() >= NEED


def test_a_workspace_that_is_large_enough_is_used():
    ws = torch.empty(NEED, dtype=torch.uint8)
    for w in room(ws):
        assert w.data_ptr() == ws.data_ptr()
