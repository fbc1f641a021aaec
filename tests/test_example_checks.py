"""The checks inside examples/serve_trace.py tell a right result from one with a
key missed, a key too many, a wrong slot or a wrong head.  The mistakes are
planted in plain torch on the CPU."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("serve_trace", os.path.join(ROOT, "examples", "serve_trace.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def made(ex, m, n, seed):
    g = torch.Generator().manual_seed(seed)
    draw = lambda t, h: torch.randn(t, h, ex.D, generator=g).to(torch.bfloat16)
    return draw(m, ex.HQ), draw(n, ex.HKV), draw(n, ex.HKV)


def rounded(ex, q, k, v, mask=0, swap=None, head=0):
    """Attention with weights and outputs rounded as a kernel does it.  mask: keys
    more (or fewer) than causal; swap: two slots whose values are exchanged; head:
    by how many key heads the values are off."""
    G, m, n = ex.HQ // ex.HKV, q.shape[0], k.shape[0]
    q, k, v = (x.float().transpose(0, 1) for x in (q, k, v))
    v = v.roll(head, 0)
    if swap:
        a, b = swap
        v = v.clone()
        v[:, [a, b]] = v[:, [b, a]]
    k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = q @ k.transpose(1, 2) * ex.D ** -0.5
    s = s.masked_fill(torch.arange(n) > torch.arange(n - m, n)[:, None] + mask, float("-inf"))
    e = torch.exp(s - s.amax(2, keepdim=True))
    out = e.to(torch.bfloat16).float() @ v / e.sum(2, keepdim=True)
    w = e / e.sum(2, keepdim=True)
    return out.to(torch.bfloat16).transpose(0, 1), w.sum(1).view(ex.HKV, G, n).sum(1)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 40), (1, 3000), (70, 70), (64, 2000)])
def test_right_results_pass(ex, m, n):
    x = made(ex, m, n, m + n)
    want, off, w, w_off = ex.dense(*x)
    out, got = rounded(ex, *x)
    ex.compare("right", out, want, off)
    ex.compare_weights("right", got, w, w_off)


@pytest.mark.parametrize("m,n", [(1, 40), (1, 3000), (64, 2000)])
@pytest.mark.parametrize("wrong", [dict(mask=-1), dict(swap=(5, 17)), dict(head=1)], ids=str)
def test_wrong_outputs_do_not(ex, m, n, wrong):
    x = made(ex, m, n, m + n)
    want, off, w, w_off = ex.dense(*x)
    out, got = rounded(ex, *x, **wrong)
    with pytest.raises(AssertionError):
        ex.compare("wrong", out, want, off)
    if "mask" in wrong:
        with pytest.raises(AssertionError):
            ex.compare_weights("wrong", got, w, w_off)


def test_a_key_too_many(ex):
    x = made(ex, 64, 2000, 9)
    want, off, w, w_off = ex.dense(*x)
    out, got = rounded(ex, *x, mask=1)
    with pytest.raises(AssertionError):
        ex.compare("wrong", out, want, off)
    with pytest.raises(AssertionError):
        ex.compare_weights("wrong", got, w, w_off)


def test_what_an_eviction_keeps(ex):
    w = [9.0, 0.5, 3.0, 3.0, 7.0, 3.0, 0.0, 1.0]
    assert ex.heaviest(w, 8, 1, 1) == list(range(8))
    assert ex.heaviest(w, 4, 1, 1) == [0, 2, 4, 7]   # of equal weights the earlier one
    assert ex.heaviest(w, 5, 0, 2) == [0, 2, 4, 6, 7]
