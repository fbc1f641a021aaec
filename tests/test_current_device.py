"""Kernels are launched on the thread's current device, so a call whose tensors
lie on another one is refused before anything is launched.  No GPU is needed:
the device indices are faked, and the library is a recorder."""
from types import SimpleNamespace

import pytest
import torch

import paper_2609_28870_gb300 as ptc


class On1(torch.Tensor):
    """A CPU tensor that says it lies on cuda:1."""

    def get_device(self):
        return 1


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *a: 256
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(ptc, "lib", lambda: r)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: SimpleNamespace(cuda_stream=0))
    return r


def current(monkeypatch, index):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: index)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: index)


def on1(x):
    return x.as_subclass(On1)


def paged():
    i64 = lambda v: on1(torch.tensor(v, dtype=torch.int64))
    i32 = lambda v: on1(torch.tensor(v, dtype=torch.int32))
    kv = lambda: on1(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16))
    return (kv(), kv(), i32([0]), i64([0, 1])), i64([0, 1]), i32([1]), on1(torch.zeros(1, 1, 64, dtype=torch.bfloat16))


CALLS = {
    "ptc_kv_append": lambda t, off, n, x: ptc.ptc_kv_append(x, x, *t, off, n),
    "ptc_paged_attention": lambda t, off, n, x: ptc.ptc_paged_attention(x, *t, off, n, 1),
    "ptc_kv_evict": lambda t, off, n, x: ptc.ptc_kv_evict(*t, n, on1(torch.zeros(1, 16)), t[2], t[3], 4, 1, 1, 16),
}


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_paged_keys_and_values(monkeypatch, lib, name):
    t, off, n, x = paged()
    current(monkeypatch, 0)
    with pytest.raises(ValueError, match="current device"):
        CALLS[name](t, off, n, x)
    assert lib.calls == []
    current(monkeypatch, 1)
    CALLS[name](t, off, n, x)
    assert lib.calls == [name]


def test_the_other_calls(monkeypatch, lib):
    """All of them take their stream from the tensors' device."""
    current(monkeypatch, 0)
    with pytest.raises(ValueError, match="current device"):
        ptc._stream(torch.device("cuda", 1))
    assert ptc._stream(torch.device("cuda", 0)) == 0


@pytest.mark.parametrize("plan", [ptc.PipelinePlan, ptc.HostPipelinePlan, ptc.TraceStatsPlan])
def test_a_plan_made_on_another_device(monkeypatch, lib, plan):
    """A plan is run where it was made."""
    ran = []
    p = plan.__new__(plan)
    p.device, p._fn, p._args = torch.device("cuda", 1), lambda: ran.append(1) or 0, ()
    current(monkeypatch, 0)
    with pytest.raises(ValueError, match="current device"):
        p.run()
    assert ran == []
    current(monkeypatch, 1)
    p.run()
    assert ran == [1]
