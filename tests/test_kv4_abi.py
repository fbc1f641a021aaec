"""The calls on rotary positions and pages of 4 bits without a GPU: the binding
packs ptc_rope as a C compiler lays it out, bad arguments are refused before any
CUDA call, by the library and by the binding, and frequencies are scaled by their
definitions."""
import math
import os
import struct
import subprocess

import pytest
import torch

import paper_2609_28870_gb300 as ptc
from tests.test_current_device import current, lib, on1  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, OVERFLOW, WORKSPACE = 1, 3, 4
FAKE = 4096  # never dereferenced: the checks below fail first


@pytest.fixture(scope="module")
def L():
    from paper_2609_28870_gb300 import build
    build.build()
    return ptc.lib()


def paged(**o):
    from paper_2609_28870_gb300 import kv
    d = dict(k=FAKE, v=FAKE, ks=(8 * 16 * 48, 16 * 48, 48), vs=(8 * 16 * 48, 16 * 48, 48), page_ids=FAKE, page_off=FAKE,
             kv_len=FAKE, n_page_ids=20, n_pages=40, n_req=3, block_size=16, n_kv_heads=8, head_dim=64, dtype=0)
    d.update(o)
    return kv.PAGED_KV.pack(d["k"], d["v"], *d["ks"], *d["vs"], d["page_ids"], d["page_off"], d["kv_len"],
                            d["n_page_ids"], d["n_pages"], d["n_req"], d["block_size"], d["n_kv_heads"], d["head_dim"],
                            d["dtype"])


def rope(table=FAKE, pos=0, n_pos=100, n_freq=32, inter=0):
    from paper_2609_28870_gb300 import rope as r
    return r.ROPE.pack(table, pos, n_pos, n_freq, inter)


def strides(a=512, b=64):
    return struct.pack("@2q", a, b)


def test_rope_layout_matches_binding(tmp_path):
    from paper_2609_28870_gb300 import rope as r
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ptc.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", offsetof(ptc_rope, {f}));\n'
                             for f in ("table", "pos", "n_pos", "n_freq", "interleaved"))
                   + '  printf("%zu\\n", sizeof(ptc_rope));\n  return 0;\n}\n')
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [0, 8, 16, 20, 24, r.ROPE.size]


def test_row_bytes(L):
    for D in range(16, 129, 8):
        row = 48 if D <= 64 else 80
        assert L.ptc_kv4_row_bytes(D) == ptc.kv4_row_bytes(D) == row
    for bad in (0, 8, 60, 136):
        with pytest.raises(ValueError):
            ptc.kv4_row_bytes(bad)


def test_table_refusals(L):
    assert L.ptc_rope_table(FAKE, 0, 10, 1.0, FAKE, None) == INVALID
    assert L.ptc_rope_table(FAKE, 65, 10, 1.0, FAKE, None) == INVALID
    for factor in (math.inf, math.nan):
        assert L.ptc_rope_table(FAKE, 8, 10, factor, FAKE, None) == INVALID
    assert L.ptc_rope_table(None, 8, 10, 1.0, FAKE, None) == INVALID
    assert L.ptc_rope_table(FAKE + 4, 8, 10, 1.0, FAKE, None) == INVALID
    assert L.ptc_rope_table(FAKE, 8, 10, 1.0, FAKE + 8, None) == INVALID
    assert L.ptc_rope_table(FAKE, 8, 10, 1.0, None, None) == INVALID
    assert L.ptc_rope_table(None, 8, 0, 1.0, None, None) == 0


BAD_CACHES = [dict(dtype=2), dict(block_size=0), dict(block_size=513), dict(n_kv_heads=0), dict(head_dim=8),
              dict(head_dim=60), dict(head_dim=136), dict(page_off=0), dict(kv_len=0), dict(page_ids=0), dict(k=FAKE + 8),
              dict(v=0), dict(ks=(0, 768, 48)), dict(ks=(6144, 768, 40)), dict(vs=(6144, -768, 48)), dict(vs=(6144, 768, 0)),
              dict(ks=(6152, 768, 48))]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=[str(b) for b in BAD_CACHES])
def test_a_bad_cache_is_refused_by_every_call(L, bad):
    kv = paged(**bad)
    s = strides()
    assert L.ptc_kv4_append(kv, rope(), FAKE, s, FAKE, s, 8, FAKE, FAKE, s, s, FAKE, 5, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_kv4_read(kv, FAKE, 5, FAKE, FAKE, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_kv4_attention(kv, FAKE, s, FAKE, 5, 8, 5, 0.1, FAKE, FAKE, FAKE, 1 << 30, None, None) == INVALID


@pytest.mark.parametrize("four", [False, True])
def test_write_refusals(L, four):
    fn = L.ptc_kv4_append if four else L.ptc_kv_append_rope
    cache = {} if four else dict(ks=(8192, 1024, 64), vs=(8192, 1024, 64))

    def call(r=rope(), q=FAKE, qs=strides(), qo=FAKE, qos=strides(), heads=8, k=FAKE, v=FAKE, ks=strides(), vs=strides(),
             off=FAKE, n=5, ws=FAKE, ws_bytes=1 << 20, **o):
        return fn(paged(**cache, **o), r, q, qs, qo, qos, heads, k, v, ks, vs, off, n, ws, ws_bytes, None, None)

    for bad in (rope(table=0), rope(table=FAKE + 4), rope(n_freq=0), rope(n_freq=33), rope(inter=2), rope(inter=-1),
                rope(n_pos=0)):
        assert call(r=bad) == INVALID
    assert call(r=None) == INVALID  # queries, or turned keys, without a table
    for bad in (dict(q=0), dict(q=FAKE + 2), dict(qo=0), dict(k=0), dict(v=FAKE + 8), dict(off=None), dict(qs=None),
                dict(qos=None), dict(ks=None), dict(vs=None), dict(qs=strides(512, 60)), dict(qos=strides(-512)),
                dict(ks=strides(0)), dict(vs=strides(512, 4)), dict(n_req=0),
                dict(qos=strides(1024))):  # in place with other strides
        assert call(**bad) == INVALID, bad
    assert call(n=(1 << 31) + 1) == OVERFLOW
    assert call(ws=None) == WORKSPACE and call(ws_bytes=16) == WORKSPACE
    assert call(n=0) == 0


def test_read_and_attention_refusals(L):
    kv, s = paged(), strides()
    assert L.ptc_kv4_read(kv, None, 5, FAKE, FAKE, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_kv4_read(kv, FAKE, 5, FAKE + 2, FAKE, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_kv4_read(kv, FAKE, 5, FAKE, 0, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_kv4_read(kv, FAKE, 5, FAKE, FAKE, None, 0, None, None) == WORKSPACE
    assert L.ptc_kv4_read(kv, FAKE, (1 << 31) + 1, FAKE, FAKE, FAKE, 1 << 20, None, None) == OVERFLOW
    assert L.ptc_kv4_read(paged(n_req=0), FAKE, 5, FAKE, FAKE, FAKE, 1 << 20, None, None) == INVALID

    def call(n_tok=5, heads=8, max_q=5, scale=0.1, q=FAKE, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 30, qs=s, off=FAKE, **o):
        return L.ptc_kv4_attention(paged(**o), q, qs, off, n_tok, heads, max_q, scale, out, lse, ws, ws_bytes, None, None)

    for scale in (0.0, -1.0, math.inf, math.nan, 3e38):
        assert call(scale=scale) == INVALID
    for bad in (dict(heads=12), dict(heads=0), dict(heads=8 * 129), dict(q=0), dict(q=FAKE + 2), dict(out=0), dict(lse=None),
                dict(off=None), dict(qs=None), dict(qs=strides(512, 4)), dict(n_req=0)):
        assert call(**bad) == INVALID, bad
    assert call(n_tok=1 << 31) == OVERFLOW and call(n_pages=1 << 31) == OVERFLOW
    assert call(n_page_ids=1 << 38) == OVERFLOW
    assert call(ws=None) == WORKSPACE and call(ws_bytes=0) == WORKSPACE
    assert call(n_req=0, n_tok=0) == 0
    assert L.ptc_kv4_attention_workspace_bytes(3, 8, 8, 64, 5, 15, 20, 16) % 256 == 0
    # many rows a request: room for the pages in 16 bits, unless they are no multiple of 8 slots or more than 1 GB
    plain = L.ptc_kv4_attention_workspace_bytes(1, 8, 2, 128, 4096, 50, 300, 16)
    assert L.ptc_kv4_attention_workspace_bytes(1, 8, 2, 128, 4096, 4096, 300, 16) >= plain + 300 * 16 * 2 * 128 * 4
    assert L.ptc_kv4_attention_workspace_bytes(1, 8, 2, 128, 4096, 4096, 400, 12) == plain
    assert L.ptc_kv4_attention_workspace_bytes(1, 8, 2, 128, 4096, 4096, 1 << 17, 16) == plain


def cached():
    i64 = lambda v: on1(torch.tensor(v, dtype=torch.int64))
    i32 = lambda v: on1(torch.tensor(v, dtype=torch.int32))
    c4 = lambda: on1(torch.zeros(2, 1, 16, 48, dtype=torch.uint8))
    c16 = lambda: on1(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16))
    tail = i32([0]), i64([0, 1])
    return (c4(), c4(), *tail), (c16(), c16(), *tail), (i64([0, 1]), i32([1])), on1(torch.zeros(1, 1, 64, dtype=torch.bfloat16)), \
        on1(torch.ones(4, 64))


CALLS = {
    "ptc_kv_append_rope": lambda t4, t, n, x, r: ptc.ptc_kv_append_rope(None, x, x, *t, *n, r),
    "ptc_kv4_append": lambda t4, t, n, x, r: ptc.ptc_kv4_append(x, x, *t4, *n),
    "ptc_kv4_read": lambda t4, t, n, x, r: ptc.ptc_kv4_read(*t4, *n, 1, 64, k_out=x, v_out=x),
    "ptc_kv4_attention": lambda t4, t, n, x, r: ptc.ptc_kv4_attention(x, *t4, *n, 1, out=x, lse=on1(torch.zeros(1, 1))),
    "ptc_rope_table": lambda t4, t, n, x, r: ptc.ptc_rope_table(on1(torch.ones(2, dtype=torch.float64)), 1,
                                                                out=on1(torch.zeros(1, 4))),
}


@pytest.mark.parametrize("call", CALLS)
def test_calls_on_another_device_are_refused(lib, monkeypatch, call):  # noqa: F811
    import paper_2609_28870_gb300.kv4 as kv4
    import paper_2609_28870_gb300.rope as r
    for m in (kv4, r):  # workspaces cannot be made on the device that is not there
        monkeypatch.setattr(m, "_room", lambda k, need, dev, ws: torch.empty(max(need, 256), dtype=torch.uint8))
    current(monkeypatch, 0)
    with pytest.raises(ValueError, match="device"):
        CALLS[call](*cached())
    assert lib.calls == []
    current(monkeypatch, 1)
    CALLS[call](*cached())
    assert lib.calls == [call]


@pytest.mark.parametrize("call", ["ptc_kv_append_rope", "ptc_kv4_append", "ptc_kv4_attention"])
def test_gradients_are_refused(lib, monkeypatch, call):  # noqa: F811
    current(monkeypatch, 1)
    t4, t, n, x, r = cached()
    x.requires_grad_()
    with pytest.raises(ValueError, match="backward"):
        CALLS[call](t4, t, n, x, r)
    assert lib.calls == []


def test_frequencies():
    f, factor = ptc.rope_frequencies(8, base=10_000.0)
    assert factor == 1.0 and f.dtype == torch.float64
    assert torch.allclose(f, torch.tensor([1, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(ptc.rope_frequencies(8, scaling="linear", factor=4)[0], f / 4)
    b, _ = ptc.rope_frequencies(8, scaling="base", factor=4)
    assert float(b[0]) == 1.0 and math.isclose(float(b[-1]), 0.001 / 4, rel_tol=1e-12)
    p, factor = ptc.rope_frequencies(64, scaling="parts", factor=16, original=2048)
    g, _ = ptc.rope_frequencies(64)
    turns = 2048 * g / (2 * math.pi)
    assert torch.equal(p[turns >= 32], g[turns >= 32]) and torch.allclose(p[turns <= 1], g[turns <= 1] / 16, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert between.any() and ((p < g) & (p > g / 16))[between].all() and (p.diff() < 0).all()
    assert math.isclose(factor, 0.1 * math.log(16) + 1)
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, base=-1), dict(rot_dim=8, factor=0.5),
                dict(rot_dim=8, scaling="other"), dict(rot_dim=2, scaling="base"),
                dict(rot_dim=8, scaling="parts", slow=4, fast=2)):
        with pytest.raises(ValueError):
            ptc.rope_frequencies(**bad)
