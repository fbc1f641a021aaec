"""The calls on paged keys and values have no backward pass: inputs that ask for
gradients are refused, not detached without a word.  No GPU is needed: the
library is a recorder and the tensors' device is faked."""
import pytest
import torch

import paper_2609_28870_gb300 as ptc
from tests.test_current_device import current, lib, on1, paged  # noqa: F401

KV = ("k", "v")
INPUTS = {"ptc_kv_append": ("k_new", "v_new") + KV, "ptc_paged_attention": ("q", "mass") + KV,
          "ptc_kv_evict": ("mass",) + KV}


def call(name, grad):
    (k, v, ids, off), tok, n, x = paged()
    ask = lambda t, what: on1(t.detach().requires_grad_()) if what == grad else t
    mass, k, v = ask(on1(torch.zeros(1, 16)), "mass"), ask(k, "k"), ask(v, "v")
    if name == "ptc_kv_append":
        return ptc.ptc_kv_append(ask(x, "k_new"), ask(x, "v_new"), k, v, ids, off, tok, n)
    if name == "ptc_paged_attention":
        return ptc.ptc_paged_attention(ask(x, "q"), k, v, ids, off, tok, n, 1, mass=mass)
    return ptc.ptc_kv_evict(k, v, ids, off, n, mass, ids, off, 4, 1, 1, 16)


@pytest.mark.parametrize("name,grad", [(n, g) for n in INPUTS for g in INPUTS[n]])
def test_inputs_that_ask_for_gradients(monkeypatch, lib, name, grad):  # noqa: F811
    current(monkeypatch, 1)
    with pytest.raises(ValueError, match="no backward pass"):
        call(name, grad)
    assert lib.calls == []
    with torch.no_grad():
        call(name, grad)
    assert lib.calls == [name]


@pytest.mark.parametrize("name", INPUTS)
def test_inputs_that_do_not(monkeypatch, lib, name):  # noqa: F811
    current(monkeypatch, 1)
    call(name, None)
    assert lib.calls == [name]
