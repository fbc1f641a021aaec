"""ptc_rope_table and ptc_kv_append_rope against their definitions in 64 bits:
angles of near and far positions; rotations rounded once, so equal bit for bit;
both layouts of pairs, parts of a head, in place, given positions; refusals."""
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


def bits(x):
    import torch
    return x.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


@pytest.mark.parametrize("pairs", [1, 3, 8, 40, 64])
@pytest.mark.parametrize("n_pos", [1, 77, 5000, 200_003])
@pytest.mark.parametrize("factor", [1.0, 1.375])
def test_table(pairs, n_pos, factor):
    """An angle's remainder is within an eighth of a turn, 0.785, with a relative
    error of four roundings, 2^-23: 9.4e-8.  Its function adds 1.3e-8 and two
    roundings of 2^-25, the factor one: below 1.8e-7 in all, and 2^-22 is 2.4e-7."""
    import torch
    import paper_2609_28870_gb300 as ptc
    f, _ = ptc.rope_frequencies(2 * pairs, scaling="none")
    f = (f * 1.1).cuda()
    got = ptc.ptc_rope_table(f, n_pos, factor)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    want = factor * torch.cat([angle.cos(), angle.sin()], 1)
    assert got.shape == want.shape and got.dtype == torch.float32
    assert float((got.double() - want).abs().max()) <= factor * 2 ** -22


def test_table_of_odd_frequencies():
    """Negative ones, none at all, many turns a position, and ones that are not finite."""
    import torch
    import paper_2609_28870_gb300 as ptc
    f = torch.tensor([-0.25, 0.0, 1000.0, math.inf, math.nan, 1e-12, 2 * math.pi], dtype=torch.float64, device="cuda")
    got = ptc.ptc_rope_table(f, 300)
    angle = torch.arange(300, dtype=torch.float64, device="cuda")[:, None] * f
    want = torch.cat([angle.cos(), angle.sin()], 1)
    fine = [0, 1, 2, 5, 6, 7, 8, 9, 12, 13]
    assert float((got[:, fine].double() - want[:, fine]).abs().max()) <= 2 ** -22
    assert torch.isnan(got[:, [3, 4, 10, 11]]).all()
    out = torch.full((300, 14), 7.0, device="cuda")
    assert ptc.ptc_rope_table(f, 300, out=out) is out and torch.equal(out.nan_to_num(), got.nan_to_num())
    assert ptc.ptc_rope_table(f, 0).shape == (0, 14)


LENS = [[(1, 1)], [(1, 17), (1, 16), (1, 500)], [(40, 40), (0, 9), (0, 0), (33, 70), (1, 5)], [(700, 900), (300, 300)]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("B,D,Hq,Hkv,layout,dtype", [(16, 128, 8, 2, "head", "bf16"), (16, 64, 8, 8, "token", "fp16"),
                                                     (1, 16, 3, 1, "head", "bf16"), (12, 40, 6, 3, "token", "bf16"),
                                                     (256, 96, 5, 5, "head", "fp16")])
@pytest.mark.parametrize("part", ["all", "half", "odd"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rope(lens, B, D, Hq, Hkv, layout, dtype, part, interleaved):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import turned
    from tests.kv_util import Cache
    c = Cache(lens, Hq=Hq, Hkv=Hkv, D=D, B=B, layout=layout, dtype=dtype)
    rot = {"all": D, "half": D // 2 // 8 * 8, "odd": 2 * (D // 2 - 3) - 4}[part]
    rope = ptc.ptc_rope_table(ptc.rope_frequencies(rot)[0].cuda(), 1500, 1.25)
    at = torch.cat([torch.arange(n - m, n) for m, n in lens]).cuda()
    k_new = torch.cat([k[n - m:] for k, (m, n) in zip(c.keys, lens)])
    both = torch.stack([k_new, torch.cat([v[n - m:] for v, (m, n) in zip(c.vals, lens)])], 1)  # strides: one buffer
    want_k, want_v = c.k.clone(), c.v.clone()
    keys = turned(k_new, rope, at, interleaved)
    row = 0
    for r, (m, n) in enumerate(lens):
        page, slot = c.where(r, n)
        want_k[page[n - m:], :, slot[n - m:]] = keys[row:row + m]
        row += m
        c.k[page[n - m:], :, slot[n - m:]] = math.nan
        c.v[page[n - m:], :, slot[n - m:]] = math.nan
    q_was = c.q.clone()
    q = ptc.ptc_kv_append_rope(c.q, both[:, 0], both[:, 1], *c.table(), c.tok_off, c.kv_len, rope, interleaved=interleaved)
    want_q = turned(q_was, rope, at, interleaved)
    assert torch.equal(bits(c.q), bits(q_was)) and torch.equal(bits(q), bits(want_q))
    assert torch.equal(bits(c.k), bits(want_k)) and torch.equal(bits(c.v), bits(want_v))
    # in place, out of a wider buffer, at given positions (angle 0: as they are)
    wide = torch.zeros(c.q.shape[0], Hq, D + 8, dtype=c.dt, device="cuda")
    wide[..., :D] = q_was
    pos = (1499 - at).int()
    same = ptc.ptc_kv_append_rope(wide[..., :D], both[:, 0], both[:, 1], *c.table(), c.tok_off, c.kv_len, rope, pos=pos,
                                  interleaved=interleaved, q_out=wide[..., :D])
    assert same.data_ptr() == wide.data_ptr() and not wide[..., D:].any()
    assert torch.equal(bits(wide[..., :D]), bits(turned(q_was, rope, pos, interleaved)))
    # no queries
    assert ptc.ptc_kv_append_rope(None, both[:, 0], both[:, 1], *c.table(), c.tok_off, c.kv_len, rope) is None


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rotation_is_rounded_once(dtype):
    """Half a million channels whose turned values lie on or beside the middle of
    two 16-bit numbers, sums that cancel, subnormals, zeros and values that are not finite."""
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv4_util import turned
    from tests.kv_util import Cache
    T, D = 1000, 128
    c = Cache([(T, T)], Hq=4, Hkv=1, D=D, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    rope = torch.randn(T, D, generator=g, device="cuda")
    rope[::3] = torch.round(rope[::3] * 8) / 8  # products with few bits: sums on a border
    rope[1::7] = rope[1::7].to(c.dt).float() * (1 + 2.0 ** -12)
    q = c.q.clone()
    q[::5, :, :64] = q[::5, :, 64:]
    q[::4] *= torch.exp2(torch.randint(-14, 8, (1, 4, D), generator=g, device="cuda").float()).to(c.dt)
    q[7] = 0
    q[8, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 0.0], device="cuda")
    q[9] = torch.finfo(c.dt).tiny * torch.randn(4, D, generator=g, device="cuda").to(c.dt)
    got = ptc.ptc_kv_append_rope(q, c.keys[0], c.vals[0], *c.table(), c.tok_off, c.kv_len, rope)
    want = turned(q, rope, torch.arange(T, device="cuda"), False)
    a, b = q[8, :, :64].double(), q[8, :, 64:].double()  # (the reference's rounding is for finite numbers)
    cs, sn = rope[8, :64].double(), rope[8, 64:].double()
    full = torch.cat([a * cs - b * sn, b * cs + a * sn], -1)
    gone = ~torch.isfinite(full)
    assert torch.equal(got[8][gone].nan_to_num(1, 2, 3), full[gone].to(c.dt).nan_to_num(1, 2, 3)) and int(gone.sum()) == 6
    want[8][gone], got[8][gone] = 0, 0
    assert torch.equal(got, want)  # (a zero's sign may differ)


def test_refusals():
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache
    c = Cache([(2, 40), (3, 20)], Hq=2)
    x = torch.ones(5, 2, 64, dtype=c.dt, device="cuda")
    rope = torch.ones(40, 64, device="cuda")
    call = (x, x, *c.table(), c.tok_off, c.kv_len)
    for bad in (rope.double(), rope[:, :63], rope[:, ::2], torch.ones(40, 66, device="cuda"), rope[:0], rope.cpu(), rope[0]):
        with pytest.raises(ValueError):
            ptc.ptc_kv_append_rope(x, *call, bad)
    for bad in (torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda")):
        with pytest.raises(ValueError):
            ptc.ptc_kv_append_rope(x, *call, rope, pos=bad)
    with pytest.raises(ValueError):
        ptc.ptc_kv_append_rope(x[:4], *call, rope)
    with pytest.raises(ValueError):
        ptc.ptc_kv_append_rope(x, *call, rope, q_out=x[:, :1])
    with pytest.raises(ValueError):
        ptc.ptc_kv_append_rope(None, *call, rope, q_out=x)
    with pytest.raises(ValueError):  # a table that asks for gradients
        ptc.ptc_kv_append_rope(x, *call, rope.clone().requires_grad_())
    # a table too short for one request's tokens: the others are written
    before = bits(c.k).clone()
    q_out = torch.full_like(x, 5)
    with pytest.raises(ptc.PtcError) as e:
        ptc.ptc_kv_append_rope(x, *call, rope[:39], q_out=q_out)
    assert e.value.status == 1
    changed = (bits(c.k) != before).any(-1).any(1).nonzero().tolist()
    want = [[int(c.lists[0][2]), 6]] + [[int(c.lists[1][j // 16]), j % 16] for j in (17, 18, 19)]
    assert sorted(changed) == sorted(want)
    assert (q_out[1] == 5).all() and not (q_out[[0, 2, 3, 4]] == 5).all()
    # positions at the last row and past it
    pos = torch.tensor([39, 0, 40, 39, -1], dtype=torch.int32, device="cuda")
    q_out.fill_(5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ptc.ptc_kv_append_rope(torch.ones_like(x), *call, rope, pos=pos, q_out=q_out, status=status)
    assert int(status) == 1 and (q_out[[2, 4]] == 5).all() and not (q_out[[0, 1, 3]] == 5).any()
