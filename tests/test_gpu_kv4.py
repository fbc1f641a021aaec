"""Pages of 4 bits: rows equal to the definition's bit for bit (in 64 bits, and in
exact arithmetic where numbers of all sizes meet), values read back, attention over
them at lengths around tiles' and pages' ends; refusals; the calls together."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


SHAPES = [(16, 128, 4, 2, "head", "bf16"), (16, 64, 8, 8, "token", "fp16"), (1, 16, 1, 1, "head", "bf16"),
          (12, 40, 6, 3, "token", "bf16"), (256, 96, 5, 5, "head", "fp16"), (8, 80, 4, 1, "token", "bf16"),
          (24, 120, 2, 2, "head", "bf16")]
LENS = [[(1, 1)], [(1, 17), (1, 16), (1, 500)], [(40, 40), (0, 9), (0, 0), (33, 70), (1, 5)], [(700, 900), (300, 300)]]


# ---------------------------------------------------------------- append and read
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("B,D,Hq,Hkv,layout,dtype", SHAPES)
@pytest.mark.parametrize("rot", [0, 1, 2])
def test_append_and_read(lens, B, D, Hq, Hkv, layout, dtype, rot):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, rows_of, turned, values_of
    c = Cache4(lens, Hq=Hq, Hkv=Hkv, D=D, B=B, layout=layout, dtype=dtype)
    T = sum(c.new)
    g = torch.Generator(device="cuda").manual_seed(7)
    both = torch.randn(T, 2, Hkv, D, generator=g, device="cuda").to(c.dt)
    k_new, v_new = both[:, 0], both[:, 1]
    rope, at = None, torch.cat([torch.arange(n - m, n) for m, n in lens]).cuda()
    keys = k_new
    if rot:
        rope = ptc.ptc_rope_table(ptc.rope_frequencies(D if rot == 1 else 10)[0].cuda(), 1000)
        keys = turned(k_new, rope, at, rot == 2)
    K, V = rows_of(keys), rows_of(v_new)
    want_k, want_v = c.k.clone(), c.v.clone()
    row = 0
    for r, (m, n) in enumerate(lens):
        page, slot = c.where(r, n)
        want_k[page[n - m:], :, slot[n - m:]] = K[row:row + m]
        want_v[page[n - m:], :, slot[n - m:]] = V[row:row + m]
        row += m
    q = ptc.ptc_kv4_append(k_new, v_new, *c.table(), c.tok_off, c.kv_len, q=c.q if rot else None, rope=rope,
                           interleaved=rot == 2)
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v)
    assert q is None if not rot else torch.equal(q, turned(c.q, rope, at, rot == 2))
    k, v = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, T, D, c.dt)
    assert torch.equal(k, values_of(K, D, c.dt)) and torch.equal(v, values_of(V, D, c.dt))
    # a value is half a step off at most, and the base's rounding, half a unit of at most 32 steps'
    # last place: 1/16 of a step (fp16: less); then its own rounding
    for x, y in ((keys, k), (v_new, v)):
        u = torch.finfo(c.dt).eps / 2
        for a in range(0, D, 32):
            p = x[..., a:a + 32].double()
            step = (p.amax(-1) - p.amin(-1)) / 15 * (1 + u)
            # the scale's rounding moves the last code by 15 u steps, which the clamp adds
            off = (p - y[..., a:a + 32].double()).abs().amax(-1) - u * p.abs().amax(-1) * (1 + u)
            assert (off <= step * (0.5 + 32 * u + 15 * u)).all()


def test_rows_in_exact_arithmetic():
    """Groups of numbers on the borders of codes, of sizes that no 32-bit sum holds
    together, constant ones, subnormals and the largest."""
    import random
    import torch
    import paper_2609_28870_gb300 as ptc
    from fractions import Fraction
    from tests.kv4_util import Cache4, group_by_fractions
    for dtype in ("bf16", "fp16"):
        c = Cache4([(96, 96)], Hq=4, Hkv=4, D=128, dtype=dtype, seed=5)
        rng = random.Random(11)
        x = torch.randn(96, 4, 4, 32, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
        low, high = (-120, 100) if dtype == "bf16" else (-22, 12)
        for t in range(96):
            for h in range(4):
                for i in range(4):
                    kind, y = rng.randrange(8), x[t, h, i]
                    if kind == 0:  # a ladder of half steps
                        y[:] = torch.arange(32) * 2.0 ** rng.randint(-6, 3) * 0.5 + rng.randint(-40, 40) * 2.0 ** -3
                    elif kind == 1:  # all sizes
                        y *= torch.exp2(torch.tensor([float(rng.randint(low, high)) for _ in range(32)]))
                    elif kind == 2:
                        y[:] = y[0]
                    elif kind == 3:
                        y *= 2.0 ** low
                    elif kind == 4:  # a few large, the rest tiny
                        y[2:] *= 2.0 ** rng.randint(-20, -8)
                    elif kind == 5:
                        y[:] = torch.tensor([float(rng.choice([-15, -7.5, 0, 7.5, 15, 3.25])) for _ in range(32)])
                    elif kind == 6:  # far from zero
                        y += rng.choice([-1, 1]) * 2.0 ** rng.randint(2, 9)
        x = x.to(c.dt).reshape(96, 4, 128)
        ptc.ptc_kv4_append(x.cuda(), x.cuda(), *c.table(), c.tok_off, c.kv_len)
        assert torch.equal(c.k[c.lists[0][:6].long()], c.v[c.lists[0][:6].long()])
        got = c.k[c.lists[0][:6].long()].transpose(1, 2).reshape(96, 4, 80).cpu()
        params = got[..., 64:].contiguous().view(c.dt).double()
        for t in range(96):
            for h in range(4):
                for i in range(4):
                    codes, s, b = group_by_fractions(x[t, h, 32 * i:32 * i + 32].double().tolist(), c.dt)
                    assert Fraction(float(params[t, h, 2 * i])) == s and Fraction(float(params[t, h, 2 * i + 1])) == b
                    mine = []
                    for d in range(32 * i, 32 * i + 32):
                        word = int.from_bytes(bytes(got[t, h, 4 * (d // 8):4 * (d // 8) + 4].tolist()), "little")
                        mine.append(word >> (4 * (d % 8 // 2) + 16 * (d % 2)) & 15)
                    assert mine == codes, (dtype, t, h, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_groups_that_are_not_finite_read_as_nan(dtype):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4
    c = Cache4([(8, 8)], Hq=1, Hkv=1, D=128, dtype=dtype)
    x = torch.randn(8, 1, 128, device="cuda").to(c.dt)
    bad = {0: (3, math.nan), 1: (40, math.inf), 2: (70, -math.inf), 3: (127, math.nan)}
    for t, (d, value) in bad.items():
        x[t, 0, d] = value
    x[4, 0, 0], x[4, 0, 1] = torch.finfo(c.dt).max, -torch.finfo(c.dt).max
    x[5, 0, 32:64] = math.inf
    ptc.ptc_kv4_append(x, x, *c.table(), c.tok_off, c.kv_len)
    k, v = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, 8, 128, c.dt)
    gone = torch.isnan(k[:, 0].view(8, 4, 32)).cpu()
    want = torch.zeros(8, 4, dtype=torch.bool)
    for t, i in ((0, 0), (1, 1), (2, 2), (3, 3), (4, 0), (5, 1)):
        want[t, i] = True
    assert torch.equal(gone.all(-1), want) and torch.equal(gone.any(-1), want) and torch.equal(k.isnan(), v.isnan())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_groups_next_to_the_largest_number(dtype):
    """Scale and base are finite, while a value less the base may pass 32 bits."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, rows_of
    c = Cache4([(64, 64)], Hq=1, Hkv=1, D=128, dtype=dtype)
    top = torch.finfo(c.dt).max
    ends = [(a, b) for a in (0.0, 0.01, 0.25, 0.5) for b in (0.52, 0.53, 0.8, 0.92) if b - 16 * (b - a) / 15 > -0.9]
    gen = torch.Generator().manual_seed(4)
    x = torch.rand(64, 4, 32, generator=gen, dtype=torch.float64)
    for t in range(64):
        for i in range(4):
            lo, hi = ends[(4 * t + i) % len(ends)]
            x[t, i, 0], x[t, i, 1] = 0, 1
            x[t, i] = (lo + (hi - lo) * x[t, i]) * top
    x = x.to(c.dt).view(64, 1, 128).cuda()
    ptc.ptc_kv4_append(x, x, *c.table(), c.tok_off, c.kv_len)
    want = rows_of(x)
    for kept in c.table()[:2]:
        got = kept[c.lists[0][:4].long()].transpose(1, 2).reshape(64, 1, 80)
        assert torch.equal(got.cpu(), want.cpu())
    k, _ = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, 64, 128, c.dt)
    assert torch.isfinite(k).all()


@pytest.mark.parametrize("D", [64, 120])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_reading_rows_of_any_bytes(dtype, D):
    """Scales and bases of every size and sign, subnormal and infinite ones, NaN."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, once
    c = Cache4([(300, 300)], Hq=2, Hkv=2, D=D, dtype=dtype)
    c.k.copy_(torch.randint(0, 256, c.k.shape, generator=torch.Generator().manual_seed(9), dtype=torch.uint8))
    k, _ = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, 300, D, c.dt)
    page, slot = c.where(0, 300)
    row = c.k[page, :, slot].cpu()
    word = row[..., :D // 2].contiguous().view(torch.int32).long()
    e = torch.arange(8)
    code = (word[..., None] >> (4 * (e // 2) + 16 * (e % 2)) & 15).flatten(-2)
    Dp = 64 if D <= 64 else 128
    p = row[..., Dp // 2:Dp // 2 + Dp // 8].contiguous().view(c.dt).double()[..., torch.arange(D)[:, None] // 32 * 2 + torch.arange(2)]
    x, y = (16 + code) * p[..., 0], p[..., 1]  # x is exact
    z = x + y
    u = z - x
    lost = (x - (z - u)) + (y - u)
    # a bit that 64 bits lose makes the last one odd, so that the rounding to 16 still sees it
    odd = (z.view(torch.int64) & 1) == 1
    z = torch.where((lost != 0) & ~odd, torch.nextafter(z, torch.copysign(torch.full_like(z, math.inf), lost)), z)
    fine = torch.isfinite(p).all(-1)
    want = torch.where(fine, once(torch.where(fine, z, 0.0), c.dt).double(), x + y)
    got = k.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and int(fine.sum()) > 0.8 * fine.numel()
    assert torch.equal(got.nan_to_num(1.0, math.inf, -math.inf), want.nan_to_num(1.0, math.inf, -math.inf))


def test_append_and_read_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4
    c = Cache4([(2, 40), (3, 20)], Hq=2)
    x = torch.ones(5, 2, 64, dtype=c.dt, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    i64 = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")
    k, v, ids, off = c.table()
    before = c.k.clone()

    def refused(what, **o):
        with pytest.raises(what) as e:
            ptc.ptc_kv4_append(o.get("x", x), o.get("x", x), o.get("k", k), o.get("v", v), o.get("ids", ids),
                               o.get("off", off), o.get("tok", c.tok_off), o.get("n", c.kv_len))
        with pytest.raises(what) as f:
            ptc.ptc_kv4_read(o.get("k", k), o.get("v", v), o.get("ids", ids), o.get("off", off), o.get("tok", c.tok_off),
                             o.get("n", c.kv_len), 5, 64, o.get("x", x).dtype)
        return what is not ptc.PtcError or e.value.status == f.value.status == 1

    for o in (dict(k=k[..., :40]), dict(k=k.view(torch.int8)), dict(v=v[:-1]), dict(k=k.float()), dict(x=x.float()),
              dict(off=off[:-1]), dict(n=c.kv_len.long()), dict(ids=ids.long()), dict(tok=c.tok_off[:-1])):
        assert refused(ValueError, **o)
    assert refused(ptc.PtcError, n=i32([40, 2]))           # more new tokens than tokens
    assert refused(ptc.PtcError, n=i32([40, 49]))          # more tokens than pages
    assert refused(ptc.PtcError, tok=i64([0, 3, 4]))       # offsets that do not end at the tokens
    assert refused(ptc.PtcError, tok=i64([1, 2, 5]))
    assert refused(ptc.PtcError, off=i64([0, 9, 100]))
    bad = ids.clone()
    bad[2] = c.n_pages
    c.k.copy_(before)
    assert refused(ptc.PtcError, ids=bad)                  # the page of request 0's new tokens
    page, slot = c.where(1, 20)
    untouched = torch.ones(c.n_pages, 16, dtype=torch.bool, device="cuda")
    untouched[page[17:], slot[17:]] = False
    same = (c.k == before).all(-1).all(1)
    assert same[untouched].all() and not same[~untouched].any()
    with pytest.raises(ValueError):
        ptc.ptc_kv4_append(x, x, k, v, ids, off, c.tok_off, c.kv_len, q=x)  # queries without a rope
    with pytest.raises(ValueError):
        ptc.ptc_kv4_append(x.requires_grad_(), x, k, v, ids, off, c.tok_off, c.kv_len)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("lens", LENS + [[(1, 128), (1, 129), (1, 127), (1, 3000)], [(3, 1000), (2, 15), (8, 8)],
                                         [(5, 3), (1, 0), (40, 10), (200, 130)], [(130, 130), (257, 700), (1, 400)]])
@pytest.mark.parametrize("B,D,Hq,Hkv,layout,dtype", SHAPES)
def test_attention(lens, B, D, Hq, Hkv, layout, dtype):
    from tests.kv4_util import Cache4, check_attention4
    check_attention4(Cache4(lens, Hq=Hq, Hkv=Hkv, D=D, B=B, layout=layout, dtype=dtype))


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 17, 24, 32, 33, 64, 128])
@pytest.mark.parametrize("new", [1, 2, 3, 5])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_few_rows(group, new, D):
    from tests.kv4_util import Cache4, check_attention4
    check_attention4(Cache4([(new, 300), (1, 90), (new, new), (0, 40)], Hq=2 * group, Hkv=2, D=D, seed=group))


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 2047, 2049, 40_000])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_one_token_at_every_length(n, dtype):
    from tests.kv4_util import Cache4, check_attention4
    check_attention4(Cache4([(1, n)], Hq=8, Hkv=2, D=128, dtype=dtype, seed=n))


def test_scores_that_rise():
    """Every key outweighs all before it, so the maximum moves all the time; and falls."""
    import torch
    from tests.kv4_util import Cache4, check_attention4, rows_of, values_of
    for sign in (1, -1):
        for m in (1, 200):
            c = Cache4([(m, 900)], Hq=4, Hkv=1, D=64)
            ramp = torch.linspace(-4, 4, 900, device="cuda")[:, None, None] * sign
            K = rows_of((c.keys[0].float() * 0.1 + ramp).to(c.dt))
            c.put(0, K, rows_of(c.vals[0]))
            c.keys[0] = values_of(K, 64, c.dt)
            c.vals[0] = values_of(rows_of(c.vals[0]), 64, c.dt)
            c.q = (c.q.float() * 0.1 + 2).to(c.dt)
            check_attention4(c)


def test_attention_shares_pages_and_scale():
    from tests.kv4_util import Cache4, check_attention4
    check_attention4(Cache4([(1, 700), (3, 650), (40, 800), (1, 512)], Hq=8, Hkv=2, D=128, shared=512), scale=0.3)


def test_many_requests():
    from tests.kv4_util import Cache4, check_attention4
    check_attention4(Cache4([(1 + r % 3, 5 + 7 * r % 190) for r in range(1200)], Hq=2, Hkv=1, D=64))


@pytest.mark.parametrize("B,D,layout,dtype", [(16, 128, "head", "bf16"), (24, 64, "token", "fp16"), (8, 80, "token", "bf16"),
                                              (12, 128, "head", "bf16"), (256, 120, "head", "fp16")])
def test_attention_of_many_rows(B, D, layout, dtype):
    """Requests of thousands of rows: over a copy of the pages in 16 bits
    (where pages have a multiple of 8 slots).  List entries behind a request's
    tokens may name no page; one that is needed may not."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, check_attention4
    c = Cache4([(40, 700), (33, 33), (90, 2000)], Hq=128, Hkv=1, D=D, B=B, layout=layout, dtype=dtype, spare=2)
    for r, n in enumerate(c.total):
        c.page_ids[int(c.page_off[r + 1]) - 1] = -1
    check_attention4(c)
    c.page_ids[int(c.page_off[1])] = c.n_pages
    with pytest.raises(ptc.PtcError) as e:
        ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, 90)
    assert e.value.status == 1
    c = Cache4([(128, 40), (64, 0), (200, 130)], Hq=64, Hkv=1, D=D, B=B, layout=layout, dtype=dtype)
    check_attention4(c)  # tokens that see no key


def joined(c):
    """The cache's keys and values in one buffer, a page's keys before its values."""
    import torch
    both = torch.stack([c.k, c.v], 1).contiguous()
    c.k, c.v = both[:, 0], both[:, 1]
    return c


@pytest.mark.parametrize("lens", [[(1, 700), (3, 41)], [(200, 900), (1, 30)], [(700, 700)]])
@pytest.mark.parametrize("B,D,Hq", [(16, 128, 8), (12, 64, 8)])
def test_keys_and_values_in_one_buffer(lens, B, D, Hq):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, check_attention4
    c = joined(Cache4(lens, Hq=Hq, Hkv=2, D=D, B=B))
    check_attention4(c)
    T = sum(c.new)
    k, v = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, T, D, c.dt)
    assert torch.equal(k, torch.cat([x[n - m:] for x, (m, n) in zip(c.keys, lens)]))
    assert torch.equal(v, torch.cat([x[n - m:] for x, (m, n) in zip(c.vals, lens)]))
    was = c.k.clone(), c.v.clone()
    ptc.ptc_kv4_append(k, v, *c.table(), c.tok_off, c.kv_len)  # values, quantised again, are other values near them
    again = ptc.ptc_kv4_read(*c.table(), c.tok_off, c.kv_len, T, D, c.dt)
    step = 2 / 15 * k.abs().amax()
    assert float((again[0] - k).abs().max()) <= step and float((again[1] - v).abs().max()) <= 2 / 15 * v.abs().amax()
    rest = torch.ones(c.n_pages, B, dtype=torch.bool, device="cuda")
    for r, (m, n) in enumerate(lens):
        page, slot = c.where(r, n)
        rest[page[n - m:], slot[n - m:]] = False
    for now, before in zip((c.k, c.v), was):
        assert torch.equal(now.transpose(1, 2)[rest], before.transpose(1, 2)[rest])


def test_two_calls_at_once():
    """On two streams, each with its own workspace; and one workspace for calls in turn."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4
    cs = [Cache4([(1, 5000), (1, 900)], Hq=8, Hkv=2, D=128, seed=1), Cache4([(300, 2000), (5, 70)], Hq=8, Hkv=2, D=128, seed=2)]
    call = lambda c, **k: ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), **k)
    want = [call(c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    status = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in cs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, c in enumerate(cs):
            with torch.cuda.stream(streams[i]):
                got[i].append(call(c, status=status[i]))
    torch.cuda.synchronize()
    ws = torch.full((1 << 27,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        for i, c in enumerate(cs):
            got[i].append(call(c, ws=ws))
    for w, g, s in zip(want, got, status):
        ptc.check_status(s)
        for x in g:
            assert torch.equal(x[0], w[0]) and torch.equal(x[1], w[1])


@pytest.mark.parametrize("lens,Hq,Hkv", [([(300, 900), (1, 77), (130, 130)], 4, 2), ([(600, 3000)], 8, 1), ([(40, 400)], 8, 8)])
@pytest.mark.parametrize("D,B", [(128, 16), (64, 12)])
def test_given_up_waits_then_right_results(lens, Hq, Hkv, D, B):
    """The tile kernel's waits give up where nothing comes, without a fault; the
    calls after that are right.  (Requests of few rows wait for nothing.)"""
    import time
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, check_attention4
    c = Cache4(lens, Hq=Hq, Hkv=Hkv, D=D, B=B)
    check_attention4(c)
    torch.cuda.synchronize()
    L = ptc.lib()
    L.ptc_test_wait_polls(ptc.PTC_TEST_WAIT_ATTENTION + 2000)
    try:
        began = time.perf_counter()
        with pytest.raises(ptc.PtcError) as e:
            ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new))
        assert e.value.name == "PTC_ERR_TIMEOUT" and time.perf_counter() - began < 1.0
    finally:
        L.ptc_test_wait_polls(0)
    for _ in range(2):
        check_attention4(c)


def test_attention_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4
    c = Cache4([(2, 40), (3, 20)], Hq=4)
    k, v, ids, off = c.table()
    for bad in (c.q.float(), c.q[..., :44], c.q.transpose(1, 2)):
        with pytest.raises(ValueError):
            ptc.ptc_kv4_attention(bad, k, v, ids, off, c.tok_off, c.kv_len, 3)
    with pytest.raises(ptc.PtcError):
        ptc.ptc_kv4_attention(c.q[:, :3], k, v, ids, off, c.tok_off, c.kv_len, 3)
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(ptc.PtcError):
            ptc.ptc_kv4_attention(c.q, k, v, ids, off, c.tok_off, c.kv_len, 3, scale=scale)
    with pytest.raises(ptc.PtcError):
        ptc.ptc_kv4_attention(c.q, k, v, ids, off, c.tok_off, c.kv_len, 2)  # a request has three
    bad = ids.clone()
    bad[1] = c.n_pages
    with pytest.raises(ptc.PtcError):
        ptc.ptc_kv4_attention(c.q, k, v, bad, off, c.tok_off, c.kv_len, 3)
    with pytest.raises(ValueError):
        ptc.ptc_kv4_attention(c.q.requires_grad_(), k, v, ids, off, c.tok_off, c.kv_len, 3)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_captured_decode_loop(dtype):
    """Prompts written and attended, then tokens one by one out of a captured
    graph on a stream of its own, against the same in 64 bits."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4, rows_of, turned, values_of
    from tests.kv_util import close, reference
    steps, prompts = 6, [37, 128, 5]
    c = Cache4([(n, n) for n in prompts], Hq=8, Hkv=2, D=128, dtype=dtype, spare=2)
    rope = ptc.ptc_rope_table(ptc.rope_frequencies(128, scaling="parts", factor=4)[0].cuda(), 200)
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda T, H: torch.randn(T, H, 128, generator=g, device="cuda").to(c.dt)
    keys, vals = [None] * 3, [None] * 3

    def grow(k, v, lens, at):
        row = 0
        for r, m in enumerate(lens):
            K = values_of(rows_of(turned(k[row:row + m], rope, at[row:row + m], False)), 128, c.dt)
            V = values_of(rows_of(v[row:row + m]), 128, c.dt)
            keys[r] = K if keys[r] is None else torch.cat([keys[r], K])
            vals[r] = V if vals[r] is None else torch.cat([vals[r], V])
            row += m

    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = draw(170, 8), draw(170, 2), draw(170, 2)
    at = torch.cat([torch.arange(n) for n in prompts]).cuda()
    q_rot = ptc.ptc_kv4_append(k, v, *c.table(), c.tok_off, c.kv_len, q=q, rope=rope, status=status)
    got = ptc.ptc_kv4_attention(q_rot, *c.table(), c.tok_off, c.kv_len, 128, status=status)
    grow(k, v, prompts, at)
    c.q, c.keys, c.vals = turned(q, rope, at, False), keys, vals
    want = reference(c)
    close(got[0], want[0], want[3])
    close(got[1], want[1], want[4])

    one = torch.arange(4, dtype=torch.int64, device="cuda")
    qs, ks, vs = draw(3, 8), draw(3, 2), draw(3, 2)
    q_out, out, lse = torch.empty_like(qs), torch.empty_like(qs), torch.empty(3, 8, device="cuda")
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")

    def step():
        c.kv_len += 1
        ptc.ptc_kv4_append(ks, vs, *c.table(), one, c.kv_len, q=qs, rope=rope, q_out=q_out, status=status)
        ptc.ptc_kv4_attention(q_out, *c.table(), one, c.kv_len, 1, out=out, lse=lse, ws=ws, status=status)

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    lens_was = c.kv_len.clone()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        c.kv_len.copy_(lens_was)
        with torch.cuda.graph(graph, stream=stream):
            step()
        for s in range(steps):
            qs.copy_(draw(3, 8)), ks.copy_(draw(3, 2)), vs.copy_(draw(3, 2))
            graph.replay()
            at = torch.tensor([n + s for n in prompts], device="cuda")
            grow(ks, vs, [1, 1, 1], at)
            c.q, c.lens, c.tok_off = turned(qs, rope, at, False), [(1, n + s + 1) for n in prompts], one
            want = reference(c)
            close(out, want[0], want[3])
            close(lse, want[1], want[4])
    stream.synchronize()
    ptc.check_status(status)
    assert c.kv_len.tolist() == [n + steps for n in prompts]


@pytest.mark.parametrize("new", [96, 512])
def test_captured_chunks_share_a_workspace(new):
    """Graphs of a chunk (over codes; over the copy in 16 bits) and of single tokens, with one
    workspace, replayed in turn while lengths, offsets and pages change under them; offsets that are
    not sound are refused by the replay and leave the outputs; the next one works again."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import Cache4
    big = Cache4([(new, 1500), (new, new)], Hq=8, Hkv=2, D=128, seed=1)
    small = Cache4([(1, 700), (1, 33), (0, 5)], Hq=8, Hkv=2, D=128, seed=2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = [(torch.empty_like(c.q), torch.empty(c.q.shape[:2], device="cuda")) for c in (big, small)]
    need = ptc.lib().ptc_kv4_attention_workspace_bytes(2, 8, 2, 128, new, 2 * new, big.page_ids.shape[0], 16)
    plain = ptc.lib().ptc_kv4_attention_workspace_bytes(2, 8, 2, 128, new, 2 * new, big.page_ids.shape[0], 12)
    assert (need > plain) == (new == 512)

    def call(c, o, **kw):
        return ptc.ptc_kv4_attention(c.q, *c.table(), c.tok_off, c.kv_len, new if c is big else 1, out=o[0], lse=o[1], **kw)

    stream, graphs = torch.cuda.Stream(), []
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c, o in zip((big, small), outs):
            call(c, o, ws=ws, status=status)
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                call(c, o, ws=ws, status=status)
        turns = [([new, new], [1500, new]), ([new - 31, new], [1469, new]), ([new, 0], [1111, 9]), ([new, new], [new, 1500])]
        for m, n in turns:
            lens = big.kv_len
            off = torch.tensor([0, m[0], m[0] + m[1]], dtype=torch.int64)
            if m[0] + m[1] != 2 * new:  # rows behind the last sequence: not sound
                big.tok_off.copy_(off)
                for o in outs[0]:
                    o.fill_(7.0)
                graphs[0].replay()
                stream.synchronize()
                assert int(status) != 0 and all(bool((o == 7.0).all()) for o in outs[0])
                status.zero_()
                off = torch.tensor([0, new, 2 * new], dtype=torch.int64)
                m, n = [new, new], [1500, new]
            big.tok_off.copy_(off)
            if n[1] > new:  # the lists swapped: the first has few tokens, the second many
                c0, c1 = (x.clone() for x in big.lists)
                both = torch.cat([c1, c0])
                big.page_ids.copy_(both)
                big.page_off.copy_(torch.tensor([0, len(c1), len(c1) + len(c0)]))
            lens.copy_(torch.tensor(n, dtype=torch.int32))
            for g in (0, 1, 0):
                graphs[g].replay()
            got = [[x.clone() for x in o] for o in outs]
            want = [call(c, (torch.empty_like(c.q), torch.empty(c.q.shape[:2], device="cuda"))) for c in (big, small)]
            stream.synchronize()
            for x, y in zip(got, want):
                assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and bool(torch.isfinite(x[0]).all())
            ptc.check_status(status)


def test_example_over_pages_of_4_bits():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "serve_trace.py"), "--requests", "12", "--steps", "3",
                        "--bits", "4", "--check"], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "every step checked against 64 bits" in r.stdout
