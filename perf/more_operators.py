"""The calls that the operators of rotated and of 4-bit caches are measured on:
the table of rotary angles, the write of new tokens into their pages with the
rotation on the way (pages of 16 bits, pages of 4 bits), tokens read back from
pages of 4 bits, and attention over such pages.

A request's context is a list of pages, as in the calls over 16-bit pages.  A
token's row in a 4-bit page is 48 bytes for heads of up to 64 channels and 80
for up to 128: words of eight 4-bit codes, then a word (scale, base) for every
32 channels; code c stands for (16 + c) * scale + base, rounded to the 16-bit
type of the cache.  Lengths are drawn from the case alone, so that every seed
has the same work; the seed decides where the pages lie and what they hold.

With `own` false, `run` computes the plain form from elementary torch
operations; with `own` true it calls the package.
"""
import math
import random

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
_BITS = {torch.bfloat16: (8, -133), torch.float16: (11, -24)}  # significant bits, exponent of the smallest step


def listed():
    return [
        # The angles of a model of short contexts, a quarter of a head's 128
        # channels rotated: made once when a server starts.
        _table("table short", n_pos=4096, rot=32),
        # The angles of an agentic context, scaled by frequency parts.
        _table("table long", n_pos=131_072, rot=128, scaled="parts"),
        # A decode step's queries, keys and values of 64 requests, one layer.
        _append("rotate tokens", "append", n=64, past=(10, 8000), new=(1, 1)),
        # The chunks of a prefill step, one layer: neighbouring channels
        # paired, half of each head rotated, pages with the token outermost.
        _append("rotate chunks", "append", n=16, past=(0, 4000), new=(100, 8192), layout="token", inter=True, rot=64),
        # The same two into 4-bit pages, and the new tokens' values read back.
        _append("quantise tokens", "append4", n=64, past=(10, 8000), new=(1, 1), moved=True),
        _append("quantise chunks", "append4", n=16, past=(0, 4000), new=(100, 8192)),
        # Contexts taken out of their 4-bit pages, as an eviction or a move to
        # a cache of 16 bits needs them.
        _read("read contexts", n=8, total=(700, 30_000)),
        # One conversation's next token over a short context: latency.
        _attend("one token", n=1, past=(1012, 1012), new=(1, 1)),
        # A decode batch of 64 conversations that share a system prompt of
        # 1,024 tokens; contexts about the chat workload's median of 3,386.
        _attend("decode batch", n=64, past=(1100, 12_000), new=(1, 1), shared=1024),
        # Agents decoding over 32K to 131,072 tokens (the agentic cap).
        _attend("decode long", n=12, past=(32_768, 131_071), new=(1, 1), Hkv=4),
        # One engine step of continuous batching: chunks of 1 to 2,048 new
        # tokens (some requests decode) over ragged contexts.
        _attend("mixed step", n=24, past=(1, 12_000), new=(1, 2048), Hq=16, D=64, dtype="fp16", layout="token"),
        # A chunk of 4,096 tokens deep in an agentic context.
        _attend("long chunk", n=1, past=(28_701, 28_701), new=(4096, 4096)),
    ]


def _table(name, n_pos, rot, scaled="none"):
    return {"name": name, "kind": "table", "n_pos": n_pos, "rot": rot, "scaled": scaled}


def _append(name, kind, n, past, new, Hq=32, Hkv=8, D=128, B=16, dtype="bf16", layout="head", rot=0, inter=False,
            moved=False, lens=1):
    return {"name": name, "kind": kind, "n": n, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0],
            "new_hi": new[1], "Hq": Hq, "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": 0,
            "rot": rot or D, "inter": inter, "moved": moved, "lens": lens}


def _read(name, n, total, Hkv=8, D=128, B=16, dtype="bf16", layout="head", lens=1):
    return {"name": name, "kind": "read", "n": n, "past_lo": 0, "past_hi": 0, "new_lo": total[0], "new_hi": total[1],
            "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": 0, "lens": lens}


def _attend(name, n, past, new, Hq=32, Hkv=8, D=128, B=16, dtype="bf16", layout="head", shared=0, lens=1):
    return {"name": name, "kind": "attend", "n": n, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0],
            "new_hi": new[1], "Hq": Hq, "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": shared,
            "lens": lens}


def _log_int(rng, lo, hi):
    return int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** rng.random())) - 1


def draw(rng):
    """One more case: a kind, then sizes spread over the logarithm of their
    range, cut until they cost no more than the largest listed case."""
    kind = rng.choice(["table", "append", "append4", "append4", "read", "decode", "decode", "chunk", "mixed"])
    big = max(_cost(c) for c in listed())
    while True:
        n = _log_int(rng, 1, 128)
        Hkv = rng.choice([1, 2, 4, 8, 8, 16])
        D = rng.choice([64, 128, 128, 96, 80])
        B = rng.choice([16, 16, 16, 32, 64, 256, 24, 12])
        same = dict(Hkv=Hkv, D=D, B=B, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                    layout=rng.choice(["head", "token"]), lens=rng.randrange(1 << 30))
        hi = _log_int(rng, 30, 131_071)
        past = (_log_int(rng, 1, hi), hi)
        G = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16]) if Hkv <= 8 else rng.choice([1, 2, 4])
        if kind == "table":
            case = _table("", _log_int(rng, 1, 262_144), 2 * rng.choice([8, 16, 32, 40, 48, 64, rng.randint(1, 64)]),
                          rng.choice(["none", "linear", "parts"]))
        elif kind in ("append", "append4"):
            top = _log_int(rng, 1, 8192)
            case = _append("", kind, n, past, (rng.choice([1, top]), top), Hq=G * Hkv, inter=rng.random() < 0.4,
                           moved=rng.random() < 0.3, rot=rng.choice([D, D, D // 2, 16, 2 * rng.randint(1, D // 2)]),
                           **same)
        elif kind == "read":
            case = _read("", n, (max(past[0], 1), hi), **same)
        else:
            same.update(Hq=G * Hkv, shared=rng.choice([0, 0, past[0] // B * B]))
            if kind == "decode":
                new = (1, rng.choice([1, 1, 1, 3, 5]))
            else:
                top = _log_int(rng, 8, 4096)
                new = (top if kind == "chunk" and rng.random() < 0.5 else _log_int(rng, 1, top), top)
                if kind == "mixed":
                    new = (1, top)
            case = _attend("", n, past, new, **same)
        if _cost(case) <= big and _state_bytes(case) <= 12e9:
            del case["name"]
            return case


# ------------------------------------------------------------------ sizes
def _lengths(case):
    """(new, total) tokens of every request; the first has the longest of both."""
    rng = random.Random(case["lens"])
    new, past = [case["new_hi"]], [case["past_hi"]]
    for _ in range(case["n"] - 1):
        new.append(_log_int(rng, case["new_lo"], case["new_hi"]))
        past.append(_log_int(rng, case["past_lo"], case["past_hi"]))
    return new, [p + m for p, m in zip(past, new)]


def _pages(case):
    """Pages of every request, how many of them the requests share, and the
    number of different pages."""
    _, total = _lengths(case)
    B = case["B"]
    count = [-(-t // B) for t in total]
    shared = case["shared"] // B if case["n"] > 1 else 0
    return count, shared, sum(count) - shared * (case["n"] - 1)


def _padded(D):
    return 64 if D <= 64 else 128


def _row_bytes(D):
    return 48 if D <= 64 else 80


def _state_bytes(case):
    if case["kind"] == "table":
        return 4 * case["n_pos"] * case["rot"]
    rows = _pages(case)[2] * case["B"] * case["Hkv"]
    tokens = 4 * sum(_lengths(case)[0]) * case["Hkv"] * case["D"]
    return 2 * rows * (2 * case["D"] if case["kind"] == "append" else _row_bytes(case["D"])) + tokens


def _pairs(case):
    """Query and key pairs that the causal mask leaves, for one query head."""
    new, total = _lengths(case)
    return sum(m * t - m * (m - 1) // 2 for m, t in zip(new, total))


def work(case):
    if case["kind"] == "table":
        return {"bytes": 4 * case["n_pos"] * case["rot"] + 4 * case["rot"], "flops": 0}
    new, total = _lengths(case)
    Hkv, D, T, n = case["Hkv"], case["D"], sum(new), case["n"]
    count, shared, _ = _pages(case)
    tables = 4 * sum(count) + 8 * (n + 1) + 12 * n
    row = 4 * Hkv * D  # a token's key and value, 16 bits each
    groups = -(-D // 32)
    row4 = 2 * Hkv * (4 * (-(-D // 8)) + 4 * groups)  # and in a 4-bit page
    if case["kind"] in ("append", "append4"):
        # the queries in and out, keys and values in, the angles, the rows written
        size = T * (4 * case["Hq"] * D + row + 4 * case["rot"]) + tables
        if case["kind"] == "append":
            return {"bytes": size + T * row, "flops": 3 * T * (case["Hq"] + Hkv) * case["rot"]}
        return {"bytes": size + T * (row4 + row), "flops": T * (3 * (case["Hq"] + Hkv) * case["rot"] + 6 * Hkv * D)}
    if case["kind"] == "read":
        return {"bytes": T * (row4 + row) + tables, "flops": 4 * T * Hkv * D}
    Hq = case["Hq"]
    cached = sum(total) - shared * case["B"] * (n - 1)
    return {"bytes": cached * row4 + 4 * T * Hq * D + 4 * T * Hq + tables, "flops": 4 * _pairs(case) * Hq * D}


def _cost(case):
    """About the microseconds of a pass at a few TB/s and half a PFLOP/s."""
    w = work(case)
    return w["bytes"] / 4e6 + w["flops"] / 5e8


# ------------------------------------------------------------------ inputs
def _frequencies(case):
    """Radians a position of the pairs of channels, in 64 bits, and the factor
    on cosines and sines; "parts" leaves fast pairs as they are, stretches slow
    ones over 32 times the positions and mixes those between."""
    f = 10_000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
    scaled = case.get("scaled", "none")
    if scaled == "linear":
        return f / 4, 1.0
    if scaled == "parts":
        turns = 4096 * f / (2 * math.pi)
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        return f * keep + f / 32 * (1 - keep), 0.1 * math.log(32) + 1
    return f, 1.0


def _randn(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if math.prod(shape) < 1 << 28 else dtype)
    return (x * scale).to(dtype)


def _pack(codes):
    """Codes [..., channels] to bytes [..., channels / 2]: a little-endian word
    of eight channels, the even ones in its low half."""
    c = codes.unflatten(-1, (-1, 8))
    return torch.stack([c[..., a] | c[..., a + 2] << 4 for a in (0, 4, 1, 5)], -1).flatten(-2)


def _cache4(g, shape, dtype, D, spread):
    """Rows of 4-bit pages [pages, heads, slots, bytes] as keys or values leave
    them: codes about the middle, scales about 0.27."""
    P, Dp = shape[:3], _padded(D)
    x = torch.zeros(*P, _row_bytes(D), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 28) // (P[1] * P[2] * Dp))
    used = torch.arange(Dp, device="cuda") < D
    groups = torch.arange(0, Dp, 32, device="cuda") < D
    size = 0.27 * torch.exp(spread * torch.randn(Dp // 32, generator=g, device="cuda"))
    for a in range(0, P[0], step):
        part = x[a:a + step]
        c = torch.randn(*part.shape[:3], Dp, generator=g, device="cuda").mul_(3.2).add_(7.5).round_().clamp_(0, 15)
        part[..., :Dp // 2] = _pack(c.mul_(used).to(torch.uint8))
        z = torch.randn(*part.shape[:3], Dp // 32, 2, generator=g, device="cuda")
        s = (size * torch.exp(0.15 * z[..., 0])).to(dtype)
        b = ((0.3 * z[..., 1] - 23.5) * s.float()).to(dtype)
        words = torch.stack([s, b], -1) * groups[:, None]
        part[..., Dp // 2:Dp // 2 + Dp // 8] = words.flatten(-2).contiguous().view(torch.uint8)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "table":
        f, factor = _frequencies(case)
        # the pairs' frequencies differ between models by their base
        f = f * float(torch.empty(1).uniform_(0.5, 1.0, generator=torch.Generator().manual_seed(seed)))
        return {"case": case, "freq": f.cuda(), "factor": factor}
    new, total = _lengths(case)
    count, shared, pages = _pages(case)
    n, Hkv, D, B, dtype = case["n"], case["Hkv"], case["D"], case["B"], _DTYPE[case["dtype"]]
    # where the pages lie: the pages of a cache in use, in no order
    where = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    ids, at = [], shared
    for c in count:
        s = min(shared, c)
        ids += [where[:s], where[at:at + c - s]]
        at += c - s
    shape = (pages, Hkv, B) if case["layout"] == "head" else (pages, B, Hkv)
    if case["kind"] == "append":
        caches = [torch.zeros(*shape, D, dtype=dtype, device="cuda") for _ in range(2)]
    elif case["kind"] == "append4":
        caches = [torch.zeros(*shape, _row_bytes(D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        caches = [_cache4(g, shape, dtype, D, spread) for spread in (0.3, 0.1)]
    if case["layout"] == "token":
        caches = [x.transpose(1, 2) for x in caches]

    def offsets(sizes):
        return torch.tensor([0] + sizes, dtype=torch.int64).cumsum(0).cuda()

    state = {"case": case, "new": new, "total": total, "count": count, "k": caches[0], "v": caches[1],
             "page_ids": torch.cat(ids), "page_off": offsets(count), "tok_off": offsets(new),
             "kv_len": torch.tensor(total, dtype=torch.int32, device="cuda"),
             "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if case["kind"] in ("append", "append4"):
        # keys whose channels differ in size, as rotary keys' do
        chan = torch.exp(0.4 * torch.randn(D, generator=g, device="cuda")).to(dtype)
        state["q"] = _randn(g, (sum(new), case["Hq"], D), dtype)
        state["k_new"] = _randn(g, (sum(new), Hkv, D), dtype).mul_(chan)
        state["v_new"] = _randn(g, (sum(new), Hkv, D), dtype)
        # positions of contexts that an eviction has cut run ahead of their slots
        ahead = [0] * n
        if case["moved"]:
            rng = random.Random(case["lens"] + 1)
            ahead = [rng.randint(0, 2000) for _ in total]
            state["pos"] = torch.cat([torch.arange(t - m, t) + a for t, m, a in zip(total, new, ahead)]).int().cuda()
        f, factor = _frequencies(case)
        angle = torch.arange(max(t + a for t, a in zip(total, ahead)), dtype=torch.float64, device="cuda")[:, None] * f.cuda()
        state["rope"] = torch.cat([angle.cos(), angle.sin()], 1).mul_(factor).float()
    elif case["kind"] == "attend":
        state["q"] = _randn(g, (sum(new), case["Hq"], D), dtype, 1.5)
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2609_28870_gb300 as ptc
    case = s["case"]
    if case["kind"] == "table":
        return ptc.ptc_rope_table(s["freq"], case["n_pos"], s["factor"])
    table = (s["k"], s["v"], s["page_ids"], s["page_off"])
    if case["kind"] == "append":
        q = ptc.ptc_kv_append_rope(s["q"], s["k_new"], s["v_new"], *table, s["tok_off"], s["kv_len"], s["rope"],
                                   pos=s.get("pos"), interleaved=case["inter"], status=s["status"])
        return q, s["k"], s["v"]
    D, dtype, T = case["D"], _DTYPE[case["dtype"]], sum(s["new"])
    if case["kind"] == "append4":
        q = ptc.ptc_kv4_append(s["k_new"], s["v_new"], *table, s["tok_off"], s["kv_len"], q=s["q"], rope=s["rope"],
                               pos=s.get("pos"), interleaved=case["inter"], status=s["status"])
        return q, *ptc.ptc_kv4_read(*table, s["tok_off"], s["kv_len"], T, D, dtype, status=s["status"])
    if case["kind"] == "read":
        return ptc.ptc_kv4_read(*table, s["tok_off"], s["kv_len"], T, D, dtype, status=s["status"])
    return ptc.ptc_kv4_attention(s["q"], *table, s["tok_off"], s["kv_len"], max_q_len=max(s["new"]), status=s["status"])


def _run_plain(s):
    return {"table": _plain_table, "append": _plain_append, "append4": _plain_append4, "read": _plain_read,
            "attend": _plain_attend}[s["case"]["kind"]](s)


def _plain_table(s):
    angle = torch.arange(s["case"]["n_pos"], dtype=torch.float64, device="cuda")[:, None] * s["freq"]
    return torch.cat([angle.cos(), angle.sin()], 1).mul_(s["factor"]).float()


def _round(x, dtype):
    """64 bits to 16 bits in one step, ties to even."""
    bits, least = _BITS[dtype]
    step = torch.exp2((torch.frexp(x).exponent - bits).clamp_(min=least).double())
    return torch.round(x / step).mul_(step).to(dtype)


def _places(s):
    """Page, slot and position in its request's context of every new token."""
    B, T = s["case"]["B"], sum(s["new"])
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(s["tok_off"], t, right=True) - 1
    at = s["kv_len"][r] - s["tok_off"][r + 1] + t
    return s["page_ids"][s["page_off"][r] + at // B].long(), at % B, at


def _rotate(x, rows, inter):
    """Rotated tokens [T, heads, D] by their rows of cosines and sines; 64 bits
    for values next to a rounding's border."""
    half = rows.shape[1] // 2
    c, s = rows[:, None, :half].double(), rows[:, None, half:].double()
    y, turned = x.clone(), x[..., :2 * half].double()
    a, b = (turned[..., ::2], turned[..., 1::2]) if inter else (turned[..., :half], turned[..., half:])
    u, w = _round(a * c - b * s, x.dtype), _round(b * c + a * s, x.dtype)
    y[..., :2 * half] = torch.stack([u, w], -1).flatten(-2) if inter else torch.cat([u, w], -1)
    return y


def _plain_append(s):
    page, slot, at = _places(s)
    rows = s["rope"][s.get("pos", at).long()]
    s["k"][page, :, slot] = _rotate(s["k_new"], rows, s["case"]["inter"])
    s["v"][page, :, slot] = s["v_new"]
    return _rotate(s["q"], rows, s["case"]["inter"]), s["k"], s["v"]


def _quantise(x):
    """Rows of 4-bit pages of tokens [T, heads, D]; 64 bits for codes next to a
    border."""
    D, dtype = x.shape[-1], x.dtype
    Dp = _padded(D)
    last = x[..., -1:].expand(*x.shape[:-1], -D % 32)  # a short group's smallest and largest are its own
    y = torch.cat([x, last], -1).unflatten(-1, (-1, 32)).double()
    lo, hi = y.amin(-1), y.amax(-1)
    scale = _round((hi - lo) / 15, dtype)
    base = _round(lo - 16 * scale.double(), dtype)
    b, sc = base.double()[..., None], scale.double()[..., None]
    c = torch.floor((y - b) / sc - 15.5).clamp_(0, 15)
    c = torch.where(sc == 0, 0.0, c).flatten(-2)[..., :D].to(torch.uint8)
    row = torch.zeros(*x.shape[:-1], _row_bytes(D), dtype=torch.uint8, device="cuda")
    row[..., :Dp // 2] = _pack(torch.nn.functional.pad(c, (0, Dp - D)))
    words = torch.stack([scale, base], -1).flatten(-2).contiguous().view(torch.uint8)
    row[..., Dp // 2:Dp // 2 + words.shape[-1]] = words
    return row


def _values(rows, D, dtype):
    """What rows [..., bytes] stand for, in 32 bits; the codes and scales have few
    enough bits for the product to be exact."""
    Dp = _padded(D)
    w = rows[..., :Dp // 2].unflatten(-1, (-1, 4))
    codes = torch.stack([w[..., 0] & 15, w[..., 2] & 15, w[..., 0] >> 4, w[..., 2] >> 4,
                         w[..., 1] & 15, w[..., 3] & 15, w[..., 1] >> 4, w[..., 3] >> 4], -1).flatten(-2)
    words = rows[..., Dp // 2:Dp // 2 + Dp // 8].contiguous().view(dtype).unflatten(-1, (-1, 2)).float()
    x = codes.unflatten(-1, (-1, 32)).float().add_(16).mul_(words[..., :1]).add_(words[..., 1:])
    return x.flatten(-2)[..., :D].to(dtype)


def _plain_read(s):
    page, slot, _ = _places(s)
    D, dtype = s["case"]["D"], _DTYPE[s["case"]["dtype"]]
    return _values(s["k"][page, :, slot], D, dtype), _values(s["v"][page, :, slot], D, dtype)


def _plain_append4(s):
    page, slot, at = _places(s)
    rows = s["rope"][s.get("pos", at).long()]
    s["k"][page, :, slot] = _quantise(_rotate(s["k_new"], rows, s["case"]["inter"]))
    s["v"][page, :, slot] = _quantise(s["v_new"])
    return _rotate(s["q"], rows, s["case"]["inter"]), *_plain_read(s)


def _context(cache, ids, n, D, dtype):
    """A request's keys or values out of its pages: [heads, n, D] in 32 bits."""
    x = cache[ids].transpose(0, 1)
    return _values(x.reshape(x.shape[0], -1, x.shape[3])[:, :n], D, dtype).float()


def _plain_attend(s):
    case = s["case"]
    Hq, Hkv, D, dtype = case["Hq"], case["Hkv"], case["D"], _DTYPE[case["dtype"]]
    G, scale = Hq // Hkv, 1 / math.sqrt(D)
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    t0 = p0 = 0
    for m, t, c in zip(s["new"], s["total"], s["count"]):
        ids = s["page_ids"][p0:p0 + c]
        k, v = _context(s["k"], ids, t, D, dtype), _context(s["v"], ids, t, D, dtype)
        q = s["q"][t0:t0 + m].float().view(m, Hkv, G, D).permute(1, 2, 0, 3)
        sees = torch.arange(t, device="cuda") <= torch.arange(t - m, t, device="cuda")[:, None]
        step = max(1, (1 << 28) // (G * m * t))
        for h in range(0, Hkv, step):
            x = (q[h:h + step].reshape(-1, G * m, D) @ k[h:h + step].transpose(1, 2)).mul_(scale)
            x = x.view(-1, G, m, t).masked_fill_(~sees, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = x.sub_(top).exp_()
            sums = e.sum(-1, keepdim=True)
            w = e.div_(sums)
            o = w.view(-1, G * m, t) @ v[h:h + step]
            heads = slice(h * G, (h + w.shape[0]) * G)
            out[t0:t0 + m, heads] = o.view(-1, m, D).transpose(0, 1).to(out.dtype)
            lse[t0:t0 + m, heads] = (top + sums.log()).view(-1, m).T
        t0, p0 = t0 + m, p0 + c
    return out, lse


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_rotation(s, x):
    """Every pair of channels as a complex number, turned by its angle."""
    case = s["case"]
    tok, n = s["tok_off"].tolist(), case["rot"] // 2
    where = [s["pos"].tolist()[a:b] if "pos" in s else range(t - (b - a), t)
             for a, b, t in zip(tok, tok[1:], s["total"])]
    rows = s["rope"][torch.tensor([p for w in where for p in w], dtype=torch.int64, device="cuda")].double()
    first = torch.arange(n, device="cuda") * (2 if case["inter"] else 1)
    second = first + (1 if case["inter"] else n)
    y = x.double()
    z = torch.complex(y[..., first], y[..., second]) * torch.complex(rows[:, :n], rows[:, n:])[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_row(x, dtype):
    """What a token's channels stand for once quantised, group by group; the
    keys' channels have been rounded to 16 bits by their rotation."""
    y = torch.empty_like(x)
    for a in range(0, x.shape[-1], 32):
        part = x[..., a:a + 32]
        lo = part.min(-1, keepdim=True).values
        scale = _round((part.max(-1, keepdim=True).values - lo) / 15, dtype).double()
        base = _round(lo - 16 * scale, dtype).double()
        code = torch.nan_to_num(torch.div(part - base, scale) + 0.5, nan=16.0).floor().clamp(16, 31)
        y[..., a:a + 32] = code * scale + base
    return y


def _exact_read(s, cache):
    case = s["case"]
    dtype, B, D = _DTYPE[case["dtype"]], case["B"], case["D"]
    codes = _padded(D) // 2
    page, tok = s["page_off"].tolist(), s["tok_off"].tolist()
    out = torch.empty(tok[-1], case["Hkv"], D, dtype=torch.float64, device="cuda")
    channel = torch.arange(D, device="cuda")
    word, place = channel // 8 * 4, channel % 8
    byte = word + 2 * (place % 2) + place // 4
    for r in range(case["n"]):
        at = torch.arange(s["total"][r] - s["new"][r], s["total"][r], device="cuda")
        rows = cache[s["page_ids"].long()[page[r] + torch.div(at, B, rounding_mode="floor")], :, at % B]
        code = rows[..., byte].long() >> (4 * (place // 2 % 2)) & 15
        par = rows[..., codes:codes + _padded(D) // 8].contiguous().view(dtype).double()
        group = channel // 32
        out[tok[r]:tok[r + 1]] = (16 + code) * par[..., 2 * group] + par[..., 2 * group + 1]
    return out


def exact(case, seed):
    """Angles, rotations, codes and attention by their definitions; attention one
    query head and a block of query tokens at a time."""
    if case["kind"] == "attend" and 4 * _pairs(case) * case["Hq"] * case["D"] > 6e12:
        return None
    s = prepare(case, seed)
    if case["kind"] == "table":
        turn = torch.outer(torch.arange(case["n_pos"], device="cuda").double(), s["freq"])
        z = torch.polar(torch.full_like(turn, s["factor"]), turn)
        return torch.hstack([z.real, z.imag])
    dtype = _DTYPE[case["dtype"]]
    if case["kind"] == "append":
        # the caches are laid out as they are, zeros where no token was written
        caches = [x.double() for x in (s["k"], s["v"])]
        page, tok = s["page_off"].tolist(), s["tok_off"].tolist()
        for cache, x in zip(caches, (_exact_rotation(s, s["k_new"]), s["v_new"].double())):
            for r in range(case["n"]):
                at = torch.arange(s["total"][r] - s["new"][r], s["total"][r], device="cuda")
                ids = s["page_ids"].long()[page[r] + torch.div(at, case["B"], rounding_mode="floor")]
                cache[ids, :, at % case["B"]] = x[tok[r]:tok[r + 1]]
        return _exact_rotation(s, s["q"]), *caches
    if case["kind"] == "append4":
        keys = _round(_exact_rotation(s, s["k_new"]), dtype).double()
        return _exact_rotation(s, s["q"]), _exact_row(keys, dtype), _exact_row(s["v_new"].double(), dtype)
    if case["kind"] == "read":
        return _exact_read(s, s["k"]), _exact_read(s, s["v"])
    whole = {**s, "new": s["total"], "tok_off": torch.tensor([0] + s["total"]).cumsum(0)}
    k_all, v_all = (_round(_exact_read(whole, s[x]), dtype).double() for x in "kv")
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    tok, first = s["tok_off"].tolist(), whole["tok_off"].tolist()
    for r in range(case["n"]):
        t, m = s["total"][r], s["new"][r]
        key, rows = torch.arange(t, device="cuda"), max(1, (1 << 27) // t)
        for head in range(Hq):
            k, v = (x[first[r]:first[r + 1], head * Hkv // Hq] for x in (k_all, v_all))
            for a in range(0, m, rows):
                b = min(a + rows, m)
                z = s["q"][tok[r] + a:tok[r] + b, head].double() @ k.T / D ** 0.5
                z = torch.where(key > torch.arange(t - m + a, t - m + b, device="cuda").view(-1, 1), -math.inf, z)
                total = torch.logsumexp(z, 1)
                out[tok[r] + a:tok[r] + b, head] = torch.exp(z - total[:, None]) @ v
                lse[tok[r] + a:tok[r] + b, head] = total
    return out, lse
