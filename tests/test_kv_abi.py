"""The calls on paged keys and values without a GPU: the binding packs
ptc_paged_kv as a C compiler lays it out, bad arguments are refused before any
CUDA call, and workspaces have the sizes their documentation gives."""
import os
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, OVERFLOW, WORKSPACE = 1, 3, 4
FAKE = 4096  # never dereferenced: the checks below fail first

FIELDS = ["k", "v", "k_stride", "v_stride", "page_ids", "page_off", "kv_len", "n_page_ids", "n_pages", "n_req",
          "block_size", "n_kv_heads", "head_dim", "dtype"]


@pytest.fixture(scope="module")
def L():
    from paper_2609_28870_gb300 import build
    build.build()
    import paper_2609_28870_gb300 as ptc
    return ptc.lib()


def paged(**o):
    from paper_2609_28870_gb300 import kv
    d = dict(k=FAKE, v=FAKE, ks=(8 * 16 * 64, 16 * 64, 64), vs=(8 * 16 * 64, 16 * 64, 64), page_ids=FAKE, page_off=FAKE,
             kv_len=FAKE, n_page_ids=20, n_pages=40, n_req=3, block_size=16, n_kv_heads=8, head_dim=64, dtype=0)
    d.update(o)
    return kv.PAGED_KV.pack(d["k"], d["v"], *d["ks"], *d["vs"], d["page_ids"], d["page_off"], d["kv_len"],
                            d["n_page_ids"], d["n_pages"], d["n_req"], d["block_size"], d["n_kv_heads"], d["head_dim"],
                            d["dtype"])


def strides(a=512, b=64):
    return struct.pack("@2q", a, b)


def test_paged_kv_layout_matches_binding(tmp_path):
    from paper_2609_28870_gb300 import kv
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ptc.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", offsetof(ptc_paged_kv, {f}));\n' for f in FIELDS)
                   + '  printf("%zu\\n", sizeof(ptc_paged_kv));\n  return 0;\n}\n')
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want, at = [], 0
    for size, count in [(8, 1), (8, 1), (8, 3), (8, 3), (8, 1), (8, 1), (8, 1), (8, 1)] + [(4, 1)] * 6:
        want.append(at)
        at += size * count
    assert got == want + [kv.PAGED_KV.size]


BAD_CACHES = [dict(dtype=2), dict(dtype=-1), dict(block_size=0), dict(block_size=513), dict(n_kv_heads=0),
              dict(head_dim=8), dict(head_dim=60), dict(head_dim=136), dict(page_off=0), dict(kv_len=0), dict(page_ids=0),
              dict(k=FAKE + 2), dict(v=0), dict(ks=(0, 1024, 64)), dict(ks=(8192, 1024, 60)), dict(vs=(8192, -1024, 64)),
              dict(vs=(8192, 1024, 0))]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=[str(b) for b in BAD_CACHES])
def test_a_bad_cache_is_refused_by_every_call(L, bad):
    kv = paged(**bad)
    assert L.ptc_kv_append(kv, FAKE, FAKE, strides(), strides(), FAKE, 5, FAKE, 1 << 20, None, None) == INVALID
    assert L.ptc_paged_attention(kv, FAKE, strides(), FAKE, 5, 8, 5, 0.1, FAKE, FAKE, None, None, 0, FAKE, 1 << 30, None,
                                 None) == INVALID
    assert L.ptc_kv_evict(kv, FAKE, 320, 8, 1, 1, 100, FAKE, FAKE, 9, FAKE, FAKE, FAKE + 4096, 144, FAKE, 1 << 20, None,
                          None) == INVALID


def test_attention_refusals(L):
    def call(n_tok=5, heads=8, max_q=5, scale=0.1, q=FAKE, out=FAKE, lse=FAKE, m_in=None, m_out=None, slots=0, ws=FAKE,
             ws_bytes=1 << 30, s=strides(), off=FAKE, **o):
        return L.ptc_paged_attention(paged(**o), q, s, off, n_tok, heads, max_q, scale, out, lse, m_in, m_out, slots, ws,
                                     ws_bytes, None, None)

    inf = float("inf")
    for scale in (0.0, -1.0, inf, -inf, float("nan"), 3e38):
        assert call(scale=scale) == INVALID
    assert call(heads=12) == INVALID and call(heads=0) == INVALID
    assert call(heads=8 * 129) == INVALID                      # more than PTC_MAX_GROUP query heads a key head
    assert call(q=FAKE + 4) == INVALID and call(out=None) == INVALID and call(lse=None) == INVALID
    assert call(s=strides(512, 60)) == INVALID and call(s=strides(0, 64)) == INVALID
    assert call(off=None) == INVALID and call(n_req=0) == INVALID
    assert call(m_out=FAKE, slots=319) == INVALID              # fewer slots than pages hold
    assert call(m_in=FAKE) == INVALID                          # weights so far, but no place for new ones
    assert call(n_tok=1 << 31) == OVERFLOW and call(n_tok=1 << 29) == OVERFLOW
    assert call(n_pages=1 << 31) == OVERFLOW
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE and call(ws_bytes=1000) == WORKSPACE


def test_append_and_evict_refusals(L):
    def append(n_tok=5, ws=FAKE, ws_bytes=1 << 20, kn=FAKE, s=strides(), **o):
        return L.ptc_kv_append(paged(**o), kn, FAKE, s, strides(), FAKE, n_tok, ws, ws_bytes, None, None)

    assert append(kn=None) == INVALID and append(kn=FAKE + 8) == INVALID and append(s=strides(512, 4)) == INVALID
    assert append(n_req=0) == INVALID and append(n_tok=1 << 32) == OVERFLOW
    assert append(ws=None) == WORKSPACE and append(ws_bytes=16) == WORKSPACE
    assert append(n_tok=0) == 0                                 # nothing to do

    def evict(keep=8, sink=1, recent=1, longest=100, mass=FAKE, slots=320, dst=FAKE, new=FAKE + 4096, new_slots=144,
              out=FAKE, ws=FAKE, ws_bytes=1 << 20, **o):
        return L.ptc_kv_evict(paged(**o), mass, slots, keep, sink, recent, longest, dst, FAKE, 9, out, FAKE, new, new_slots,
                              ws, ws_bytes, None, None)

    assert evict(keep=0) == INVALID and evict(sink=4, recent=5) == INVALID
    assert evict(sink=0xFFFFFFFF, recent=9) == INVALID          # the sum does not wrap
    assert evict(mass=None) == INVALID and evict(new=None) == INVALID and evict(out=None) == INVALID
    assert evict(new=FAKE) == INVALID                           # the new weights over the old
    assert evict(slots=319) == INVALID and evict(new_slots=143) == INVALID and evict(dst=None) == INVALID
    assert evict(n_req=70_000) == INVALID
    assert evict(keep=(1 << 30) + 1) == OVERFLOW and evict(longest=(1 << 31) + 1) == OVERFLOW
    assert evict(ws=None) == WORKSPACE
    assert evict(n_req=0) == 0


def test_workspaces(L):
    w = L.ptc_paged_attention_workspace_bytes
    base = w(4, 32, 8, 128, 1, 0)
    assert base % 256 == 0 and base > 0
    # scores of requests of at most 16 rows are kept for the weights: 4 bytes a row, slot and key head
    slots = 1 << 20
    assert w(4, 32, 8, 128, 1, slots) - base == 4 * 4 * 8 * slots
    assert w(4, 32, 8, 128, 4, slots) - base == 16 * 4 * 8 * slots
    assert w(4, 32, 8, 128, 5, slots) == base
    assert L.ptc_kv_append_workspace_bytes(9) <= 4096 and L.ptc_kv_evict_workspace_bytes(9, 8, 1 << 20) <= 4096
