"""The calls that the cache operators are measured on: attention of new tokens
over paged keys and values (chunks, single tokens, both mixed), the same with
the accumulated attention weights, eviction by those weights, and the write of
new keys and values into their pages.

A request's context is a list of pages, as the package numbers them: page_ids
and page_off are what ptc_assign_ids and ptc_hash_blocks give for a trace's
blocks (u32 ids, u64 offsets), a page holds B tokens, and requests that share a
prefix share its pages.  Lengths are drawn from the case alone, so that every
seed has the same work; the seed decides where the pages lie and what they hold.

With `own` false, `run` computes the plain form from elementary torch
operations in 32 bits; with `own` true it calls the package.
"""
import math
import random

import torch

own = False

_NONE = -1  # 0xFFFFFFFF as an int32
_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One conversation's next token over a short context: latency.
        _attend("one token", n=1, past=(1012, 1012), new=(1, 1)),
        # A decode batch of 64 conversations that share a system prompt of
        # 1,024 tokens; contexts about the chat workload's median of 3,386.
        _attend("decode batch", n=64, past=(1100, 12_000), new=(1, 1), shared=1024),
        # Agents decoding over 32K to 131,072 tokens (the agentic cap).
        _attend("decode long", n=12, past=(32_768, 131_071), new=(1, 1), Hkv=4),
        # A first chunk with nothing cached: many small heads, fp16, pages with
        # the token outermost.
        _attend("first chunk", n=1, past=(0, 0), new=(333, 333), Hq=16, Hkv=16, D=64, dtype="fp16", layout="token"),
        # One engine step of continuous batching: chunks of 1 to 2,048 new
        # tokens (some requests decode) over ragged contexts.
        _attend("mixed step", n=24, past=(1, 12_000), new=(1, 2048)),
        # A chunk of 4,096 tokens deep in an agentic context.
        _attend("long chunk", n=1, past=(28_701, 28_701), new=(4096, 4096)),
        # The same two uses with the weights accumulated for eviction.
        _attend("decode weights", n=32, past=(2000, 16_000), new=(1, 1), weights=True),
        _attend("chunk weights", n=4, past=(500, 8000), new=(300, 2048), weights=True, layout="token"),
        # Four conversations cut to 512 tokens a head.
        _evict("evict small", n=4, past=(700, 1500), keep=512, sink=4, recent=64),
        # Long agentic contexts cut to 8,192 tokens a head.
        _evict("evict long", n=12, past=(9000, 131_072), keep=8192, sink=16, recent=1024),
        # A decode step's keys and values of 64 requests, one layer.
        _append("append tokens", n=64, past=(10, 8000), new=(1, 1)),
        # The chunks of a prefill step, one layer.
        _append("append chunks", n=16, past=(0, 4000), new=(100, 8192), layout="token"),
    ]


def _attend(name, n, past, new, Hq=32, Hkv=8, D=128, B=16, dtype="bf16", layout="head", shared=0, weights=False, lens=1):
    return {"name": name, "kind": "attend", "n": n, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0],
            "new_hi": new[1], "Hq": Hq, "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": shared,
            "weights": weights, "lens": lens}


def _evict(name, n, past, keep, sink, recent, Hkv=8, D=128, B=16, dtype="bf16", layout="head", lens=1):
    return {"name": name, "kind": "evict", "n": n, "past_lo": past[0], "past_hi": past[1], "new_lo": 0, "new_hi": 0,
            "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": 0, "keep": keep, "sink": sink,
            "recent": recent, "lens": lens}


def _append(name, n, past, new, Hkv=8, D=128, B=16, dtype="bf16", layout="head", lens=1):
    return {"name": name, "kind": "append", "n": n, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0],
            "new_hi": new[1], "Hkv": Hkv, "D": D, "B": B, "dtype": dtype, "layout": layout, "shared": 0, "lens": lens}


def _log_int(rng, lo, hi):
    return int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** rng.random())) - 1


def draw(rng):
    """One more case: a kind, then sizes spread over the logarithm of their
    range, cut until they cost no more than the largest listed case."""
    kind = rng.choice(["decode", "chunk", "mixed", "decode weights", "chunk weights", "evict", "append"])
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
        if kind == "evict":
            keep = _log_int(rng, 16, min(16_384, 2 * hi))
            sink = rng.randint(0, keep // 8)
            case = _evict("", n, (max(past[0], 1), hi), keep, sink, rng.randint(0, keep // 4), **same)
        elif kind == "append":
            top = _log_int(rng, 1, 8192)
            case = _append("", n, past, (rng.choice([1, top]), top), **same)
        else:
            G = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16]) if Hkv <= 8 else rng.choice([1, 2, 4])
            same.update(Hq=G * Hkv, weights=kind.endswith("weights"), shared=rng.choice([0, 0, past[0] // B * B]))
            if kind.startswith("decode"):
                new = (1, rng.choice([1, 1, 1, 3, 5]))
            else:
                top = _log_int(rng, 8, 4096)
                new = (top if kind.startswith("chunk") and rng.random() < 0.5 else _log_int(rng, 1, top), top)
                if kind == "mixed":
                    new = (1, top)
            case = _attend("", n, past, new, **same)
        if _cost(case) <= big and _state_bytes(case) <= 20e9:
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


def _kept(case):
    _, total = _lengths(case)
    return [min(t, case["keep"]) for t in total]


def _state_bytes(case):
    pages = _pages(case)[2]
    if case["kind"] == "evict":
        pages += sum(-(-k // case["B"]) for k in _kept(case))
    return 4 * pages * case["B"] * case["Hkv"] * case["D"]


def _pairs(case):
    """Query and key pairs that the causal mask leaves, for one query head."""
    new, total = _lengths(case)
    return sum(m * t - m * (m - 1) // 2 for m, t in zip(new, total))


def work(case):
    new, total = _lengths(case)
    Hkv, D, T, n = case["Hkv"], case["D"], sum(new), case["n"]
    count, shared, pages = _pages(case)
    tables = 4 * sum(count) + 8 * (n + 1) + 12 * n
    row = 4 * Hkv * D  # a token's key and value, 16 bits each
    if case["kind"] == "append":
        return {"bytes": 2 * T * row + tables, "flops": 0}
    if case["kind"] == "evict":
        kept = sum(_kept(case))
        # the weights once; each kept row read and written; weights and indices of what is kept written
        return {"bytes": 4 * Hkv * sum(total) + 2 * kept * row + 8 * Hkv * kept + tables, "flops": 0}
    Hq = case["Hq"]
    cached = sum(total) - shared * case["B"] * (n - 1)
    size = cached * row + 4 * T * Hq * D + 4 * T * Hq + tables
    if case["weights"]:
        size += 8 * Hkv * sum(total)
    return {"bytes": size, "flops": 4 * _pairs(case) * Hq * D}


def _cost(case):
    """About the microseconds of a pass at a few TB/s and half a PFLOP/s."""
    w = work(case)
    return w["bytes"] / 4e6 + w["flops"] / 5e8


# ------------------------------------------------------------------ inputs
def _randn(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if math.prod(shape) < 1 << 28 else dtype)
    return (x * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, total = _lengths(case)
    count, shared, pages = _pages(case)
    n, Hkv, D, B, dtype = case["n"], case["Hkv"], case["D"], case["B"], _DTYPE[case["dtype"]]
    kept = _kept(case) if case["kind"] == "evict" else [0] * n
    more = sum(-(-k // B) for k in kept)
    # where the pages lie: the pages of a cache in use, in no order
    where = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    ids, at = [], shared
    for c in count:
        s = min(shared, c)
        ids += [where[:s], where[at:at + c - s]]
        at += c - s
    shape = (pages + more, Hkv, B, D) if case["layout"] == "head" else (pages + more, B, Hkv, D)
    # keys whose channels differ in size, as rotary keys' do
    chan = torch.exp(0.4 * torch.randn(D, generator=g, device="cuda")).to(dtype)
    k_cache = _randn(g, shape, dtype).mul_(chan)
    v_cache = _randn(g, shape, dtype)
    if case["layout"] == "token":
        k_cache, v_cache = k_cache.transpose(1, 2), v_cache.transpose(1, 2)

    def offsets(sizes):
        return torch.tensor([0] + sizes, dtype=torch.int64).cumsum(0).cuda()

    state = {"case": case, "new": new, "total": total, "count": count, "k": k_cache, "v": v_cache,
             "page_ids": torch.cat(ids), "page_off": offsets(count), "tok_off": offsets(new),
             "kv_len": torch.tensor(total, dtype=torch.int32, device="cuda"),
             "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if case["kind"] == "append":
        state["k_new"] = _randn(g, (sum(new), Hkv, D), dtype)
        state["v_new"] = _randn(g, (sum(new), Hkv, D), dtype)
    elif case["kind"] == "attend":
        state["q"] = _randn(g, (sum(new), case["Hq"], D), dtype, 1.5)
    slots = sum(count) * B
    if case["kind"] == "evict" or case.get("weights"):
        # weights over many orders of magnitude, a part of them zero; none yet for new tokens
        mass = torch.exp(2.5 * torch.randn(Hkv, slots, generator=g, device="cuda") - 4)
        mass[torch.rand(Hkv, slots, generator=g, device="cuda") < 0.05] = 0
        at = 0
        for m, t, c in zip(new, total, count):
            mass[:, at + t - m:at + c * B] = 0
            at += c * B
        state["mass"] = mass
    if case["kind"] == "evict":
        dst = [-(-k // B) for k in kept]
        state["dst_ids"] = (pages + torch.randperm(more, generator=g, device="cuda")).to(torch.int32)
        state["dst_off"], state["dst"], state["kept"], state["first_dst"] = offsets(dst), dst, kept, pages
        k_cache[pages:] = 0
        v_cache[pages:] = 0
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2609_28870_gb300 as ptc
    case, table = s["case"], (s["k"], s["v"], s["page_ids"], s["page_off"])
    if case["kind"] == "append":
        ptc.ptc_kv_append(s["k_new"], s["v_new"], *table, s["tok_off"], s["kv_len"], status=s["status"])
        return s["k"], s["v"]
    if case["kind"] == "evict":
        keep, new_len, mass = ptc.ptc_kv_evict(*table, s["kv_len"], s["mass"], s["dst_ids"], s["dst_off"], case["keep"],
                                               case["sink"], case["recent"], max_kv_len=max(s["total"]),
                                               status=s["status"])
        return keep, new_len, mass, s["k"][s["first_dst"]:], s["v"][s["first_dst"]:]
    return ptc.ptc_paged_attention(s["q"], *table, s["tok_off"], s["kv_len"], max_q_len=max(s["new"]),
                                   mass=s.get("mass"), status=s["status"])


def _rows(cache, ids, n):
    """A request's rows from its pages: [heads, n, D] in 32 bits."""
    x = cache[ids].float()
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _run_plain(s):
    case = s["case"]
    return {"append": _plain_append, "evict": _plain_evict, "attend": _plain_attend}[case["kind"]](s)


def _plain_append(s):
    B, T = s["case"]["B"], s["k_new"].shape[0]
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(s["tok_off"], t, right=True) - 1
    pos = s["kv_len"][r] - s["tok_off"][r + 1] + t
    page = s["page_ids"][s["page_off"][r] + pos // B].long()
    s["k"][page, :, pos % B] = s["k_new"]
    s["v"][page, :, pos % B] = s["v_new"]
    return s["k"], s["v"]


def _plain_attend(s):
    case = s["case"]
    Hq, Hkv, D, B = case["Hq"], case["Hkv"], case["D"], case["B"]
    G, scale = Hq // Hkv, 1 / math.sqrt(D)
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    mass = torch.zeros_like(s["mass"]) if case["weights"] else None
    t0 = p0 = 0
    for m, t, c in zip(s["new"], s["total"], s["count"]):
        ids = s["page_ids"][p0:p0 + c]
        k, v = _rows(s["k"], ids, t), _rows(s["v"], ids, t)
        q = s["q"][t0:t0 + m].float().view(m, Hkv, G, D).permute(1, 2, 0, 3)
        sees = torch.arange(t, device="cuda") <= torch.arange(t - m, t, device="cuda")[:, None]
        step = max(1, (1 << 28) // (G * m * t))
        for h in range(0, Hkv, step):
            x = (q[h:h + step].reshape(-1, G * m, D) @ k[h:h + step].transpose(1, 2)).mul_(scale)
            x = x.view(-1, G, m, t).masked_fill_(~sees, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = x.sub_(top).exp_()
            total = e.sum(-1, keepdim=True)
            w = e.div_(total)
            o = w.view(-1, G * m, t) @ v[h:h + step]
            heads = slice(h * G, (h + w.shape[0]) * G)
            out[t0:t0 + m, heads] = o.view(-1, m, D).transpose(0, 1).to(out.dtype)
            lse[t0:t0 + m, heads] = (top + total.log()).view(-1, m).T
            if mass is not None:
                at = p0 * B
                mass[h:h + step, at:at + t] = s["mass"][h:h + step, at:at + t] + w.sum((1, 2))
        t0, p0 = t0 + m, p0 + c
    return (out, lse) if mass is None else (out, lse, mass)


def _plain_evict(s):
    case = s["case"]
    Hkv, B, keep_n = case["Hkv"], case["B"], case["keep"]
    keep = torch.full((case["n"], Hkv, keep_n), _NONE, dtype=torch.int32, device="cuda")
    new_mass = torch.zeros((Hkv, sum(s["dst"]) * B), dtype=torch.float32, device="cuda")
    heads = torch.arange(Hkv, device="cuda")[:, None]
    p0 = d0 = 0
    for r, (t, c, b, d) in enumerate(zip(s["total"], s["count"], s["kept"], s["dst"])):
        w = s["mass"][:, p0 * B:p0 * B + t]
        rank = w.clone()
        if b < t:
            rank[:, :case["sink"]] = math.inf
            rank[:, t - case["recent"]:] = math.inf
        chosen = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :b].sort(dim=1).values
        keep[r, :, :b] = chosen.to(torch.int32)
        new_mass[:, d0 * B:d0 * B + b] = w.gather(1, chosen)
        ids, to = s["page_ids"][p0:p0 + c].long(), s["dst_ids"][d0:d0 + d].long()
        pos = torch.arange(b, device="cuda")
        for cache in (s["k"], s["v"]):
            cache[to[pos // B], heads, pos % B] = cache[ids[chosen // B], heads, chosen % B]
        p0, d0 = p0 + c, d0 + d
    return keep, torch.tensor(s["kept"], dtype=torch.int32).cuda(), new_mass, s["k"][s["first_dst"]:], s["v"][s["first_dst"]:]


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """Attention by its definition, one query head and a block of query tokens
    at a time.  Eviction and appending copy values: nothing is computed."""
    if case["kind"] != "attend" or 4 * _pairs(case) * case["Hq"] * case["D"] > 6e12:
        return None
    s = prepare(case, seed)
    Hq, Hkv, D, B = case["Hq"], case["Hkv"], case["D"], case["B"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if case["weights"] else None
    tok, page = s["tok_off"].tolist(), s["page_off"].tolist()
    for r in range(case["n"]):
        t, m = s["total"][r], s["new"][r]
        key = torch.arange(t, device="cuda")
        where = s["page_ids"].long()[page[r] + torch.div(key, B, rounding_mode="floor")]
        for h in range(Hkv):
            k, v = s["k"][where, h, key % B].double(), s["v"][where, h, key % B].double()
            rows = max(1, (1 << 27) // t)
            for head in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                for a in range(0, m, rows):
                    b = min(a + rows, m)
                    z = s["q"][tok[r] + a:tok[r] + b, head].double() @ k.T / D ** 0.5
                    last = torch.arange(t - m + a, t - m + b, device="cuda").view(-1, 1)
                    z = torch.where(key > last, -math.inf, z)
                    total = torch.logsumexp(z, 1)
                    z = torch.exp(z - total[:, None])
                    out[tok[r] + a:tok[r] + b, head] = z @ v
                    lse[tok[r] + a:tok[r] + b, head] = total
                    if mass is not None:
                        mass[h, page[r] * B:page[r] * B + t] += z.sum(0)
    return (out, lse) if mass is None else (out, lse, mass)
