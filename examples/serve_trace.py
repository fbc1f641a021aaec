"""One attention layer serving the start of a trace out of a prefix cache.

The package's block ids are the cache's page lists: ptc_hash_blocks and
ptc_assign_ids give every request its list of blocks, equal prefixes get equal
ids, and a cache with one page a distinct block holds each prefix once.  The
requests come in trace order:

1. prefill   the blocks that an earlier request left in the cache are found
             (a block's previous use) and only the rest of the prompt is written
             (ptc_kv_append) and attended (ptc_paged_attention);
2. decode    all requests together, one token a step each, in private pages
             behind the shared ones, with the attention weights accumulated;
3. eviction  every request is cut to a budget a head by those weights
             (ptc_kv_evict) and decodes on over what is left.

The layer's projections are random tables by token; there are no weights to
load.  --check repeats every step densely in 64 bits: outputs, accumulated
weights and the tokens that the eviction keeps.

    python examples/serve_trace.py [--requests N] [--steps S] [--budget TOKENS] [--check]
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_28870_gb300 as ptc  # noqa: E402
import tracegen  # noqa: E402

HQ, HKV, D, B, VOCAB = 32, 8, 128, 16, 4096


class Layer:
    """Queries, keys and values of a token, by table."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda h: torch.randn(VOCAB, h, D, generator=g, device="cuda").to(torch.bfloat16)
        self.q, self.k, self.v = draw(HQ), draw(HKV), draw(HKV)


def dense(q, k, v):
    """Causal attention of the last len(q) tokens, by its definition: the outputs,
    how far a call's may lie from them by the norm of a token's head, the weights
    that each key gets by key head, and how far those may be off."""
    q, k, v = (x.double().transpose(0, 1) for x in (q, k, v))
    k, v = k.repeat_interleave(q.shape[0] // k.shape[0], 0), v.repeat_interleave(q.shape[0] // v.shape[0], 0)
    m, n, scale = q.shape[1], k.shape[1], q.shape[2] ** -0.5
    s = q @ k.transpose(1, 2) * scale
    # a score is a sum of D exact products in 32 bits; exp2 is good to 2^-21
    err = (q.abs() @ k.abs().transpose(1, 2)).amax(2, keepdim=True) * scale * q.shape[2] * 2 ** -23 + 2 ** -20
    hide = torch.arange(n, device=q.device) > torch.arange(n - m, n, device=q.device)[:, None]
    s.masked_fill_(hide, float("-inf"))
    lse = torch.logsumexp(s, -1, keepdim=True)
    w = torch.exp(s - lse)
    out = w @ v
    # A weight is rounded to 8 bits before it meets its value, and the result is.
    # The weights' errors, at most 2^-8 of each, have no direction in common: as
    # many independent ones add up to the root of their squares' sum, doubled here.
    rows = (w.square() @ v.square().sum(2, keepdim=True)).sqrt()
    off = 2 ** -8 * out.norm(dim=2, keepdim=True) + 2 * (2 ** -8 + 2 * err) * rows
    heads = lambda x: x.sum(1).view(HKV, -1, n).sum(1)
    return out.transpose(0, 1), off.transpose(0, 1), heads(w), heads(w * (2 * err + 2 ** -20 * (2 + lse.abs())))


def compare(what, out, want, off):
    """A call's outputs [tokens, heads, D] against dense's, head by head."""
    far = (out.double() - want).norm(dim=2, keepdim=True) / off
    assert bool((far <= 1).all()), f"{what}: {float(far.max()):.2f} times as far off as rounding explains"


def compare_weights(what, got, want, off):
    far = (got.double() - want).abs() - off - 2 ** -20 * want.abs()
    assert bool((far <= 0).all()), f"{what}: weights off by {float((got.double() - want).abs().max())}"


def heaviest(w, budget, sink, recent):
    """The positions that an eviction keeps, by its definition."""
    n = len(w)
    if n <= budget:
        return list(range(n))
    rest = sorted(range(sink, n - recent), key=lambda j: (-w[j], j))[:budget - sink - recent]
    return sorted([*range(sink), *rest, *range(n - recent, n)])


def offsets(sizes):
    return torch.tensor([0] + list(sizes), dtype=torch.int64).cumsum(0).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=48)
    ap.add_argument("--steps", type=int, default=8, help="tokens decoded before and after the eviction")
    ap.add_argument("--budget", type=int, default=512, help="tokens a head that the eviction keeps")
    ap.add_argument("--check", action="store_true")
    o = ap.parse_args()
    tr = tracegen.make(0, max_requests=o.requests)
    R = tr.n_req
    tokens = ptc.to_device_u32(tr.tokens)
    keys, blk_off, _ = ptc.ptc_hash_blocks(tokens, ptc.to_device_u64(tr.req_tok_off), None, B, 0)
    ids, n_blocks = ptc.ptc_assign_ids(keys)
    prev, _ = ptc.ptc_reuse_indices(ids, n_blocks)
    word = (tokens % VOCAB).long()

    # pages: one a distinct block, then private ones for what follows the full blocks
    tail = (2 * o.steps + B - 1) // B + 1
    pages = n_blocks + R * tail
    layer = Layer()
    k = torch.zeros(pages, HKV, B, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tok_off, off, seen = tr.req_tok_off.astype(np.int64), ptc.u64(blk_off).astype(np.int64), ptc.u32(prev)
    lists = [torch.cat([ids[off[r]:off[r + 1]], i32(list(range(n_blocks + r * tail, n_blocks + (r + 1) * tail)))])
             for r in range(R)]

    # 1. prefill, one request at a time
    torch.cuda.synchronize()
    began, reused = time.perf_counter(), 0
    for r in range(R):
        n = int(tok_off[r + 1] - tok_off[r])
        first = np.flatnonzero(seen[off[r]:off[r + 1]] == ptc.PTC_NONE)
        hit = min(B * int(first[0] if first.size else off[r + 1] - off[r]), n - 1)  # a token at least is computed
        reused += hit
        new = word[tok_off[r] + hit:tok_off[r + 1]]
        table = (k, v, lists[r], offsets([lists[r].numel()]))
        call = (offsets([n - hit]), i32([n]))
        ptc.ptc_kv_append(layer.k[new], layer.v[new], *table, *call, status=status)
        out, _ = ptc.ptc_paged_attention(layer.q[new], *table, *call, max_q_len=n - hit, status=status)
        if o.check:
            prompt = word[tok_off[r]:tok_off[r + 1]]
            compare("prefill", out, *dense(layer.q[new], layer.k[prompt], layer.v[prompt])[:2])
    ptc.check_status(status, "prefill")
    total = int(tok_off[-1])
    print(f"prefill: {R} requests, {total} tokens, {reused} of them ({reused / total:.0%}) out of the cache, "
          f"{(time.perf_counter() - began) * 1e3:.1f} ms")

    # 2. decode all requests together; each token is drawn, the weights add up
    g = torch.Generator(device="cuda").manual_seed(1)
    context = [word[tok_off[r]:tok_off[r + 1]] for r in range(R)]

    def decode(k, v, page_ids, page_off, lens, mass, rows, sums):
        """rows: each request's keys and values; sums: its weights and how far they may be off."""
        one, base = offsets([1] * R), (page_off * B).tolist()
        for _ in range(o.steps):
            lens += 1
            new = torch.randint(VOCAB, (R,), generator=g, device="cuda")
            table = (k, v, page_ids, page_off)
            ptc.ptc_kv_append(layer.k[new], layer.v[new], *table, one, lens, status=status)
            out, _, mass = ptc.ptc_paged_attention(layer.q[new], *table, one, lens, max_q_len=1, mass=mass, mass_out=mass,
                                                   status=status)
            if o.check:
                for r in range(R):
                    rows[r] = [torch.cat([x, t[new[r]][None]]) for x, t in zip(rows[r], (layer.k, layer.v))]
                    want, off, w, w_off = dense(layer.q[new[r]][None], *rows[r])
                    compare("decode", out[r:r + 1], want, off)
                    sums[r] = [torch.nn.functional.pad(x, (0, 1)) + y for x, y in zip(sums[r], (w, w_off))]
        ptc.check_status(status, "decode")
        if o.check:
            for r in range(R):
                n = int(lens[r])
                compare_weights("decode", mass[:, base[r]:base[r] + n], *sums[r])
                assert not mass[:, base[r] + n:base[r + 1]].any(), "weights of slots that hold no token"
        return mass

    page_ids, page_off = torch.cat(lists), offsets([x.numel() for x in lists])
    lens = i32([c.numel() for c in context])
    rows = [[layer.k[c], layer.v[c]] for c in context]
    mass = torch.zeros(HKV, page_ids.numel() * B, device="cuda")
    sums = [[torch.zeros(HKV, len(c), dtype=torch.float64, device="cuda")] * 2 for c in context]
    mass = decode(k, v, page_ids, page_off, lens, mass, rows, sums)
    print(f"decode: {o.steps} steps of {R} requests; the weights of a head add up to {float(mass.sum()) / HKV / R:.2f} a request")

    # 3. cut every request to the budget and decode on
    room = -(-(o.budget + o.steps) // B)
    k, v = (torch.cat([x, torch.zeros(R * room, HKV, B, D, dtype=x.dtype, device="cuda")]) for x in (k, v))
    dst, dst_off = i32(list(range(pages, pages + R * room))), offsets([room] * R)
    sink, recent = 4, min(64, o.budget // 2)
    keep, new_len, new_mass = ptc.ptc_kv_evict(k, v, page_ids, page_off, lens, mass, dst, dst_off, o.budget, sink, recent,
                                               max_kv_len=int(lens.max()))
    if o.check:
        heads = torch.arange(HKV, device="cuda")[:, None]
        for r in range(R):
            at, to, n, b = int(page_off[r]) * B, int(dst_off[r]) * B, int(lens[r]), int(new_len[r])
            w, kept = mass[:, at:at + n], keep[r, :, :b].long()
            assert kept.tolist() == [heaviest(x, o.budget, sink, recent) for x in w.tolist()], "eviction: other tokens kept"
            assert torch.equal(new_mass[:, to:to + b], w.gather(1, kept)), "eviction: other weights"
            rows[r] = [x[kept, heads].transpose(0, 1) for x in rows[r]]
            sums[r] = [x.gather(1, kept) for x in sums[r]]
    print(f"eviction: {int(lens.sum())} tokens a head cut to {int(new_len.sum())}, with "
          f"{float(new_mass.sum()) / float(mass.sum()):.0%} of the weight")
    decode(k, v, dst, dst_off, new_len, new_mass, rows, sums)
    print("every step checked against 64 bits" if o.check else "done")


if __name__ == "__main__":
    main()
