"""Operators around the paged cache of text tokens, for long conversations about videos that are answered by drafting, as cases that can be timed
and compared.

  rotate   queries and keys of new tokens turned by their positions, on one axis (text) or several (frame, row and column of a patch)
  tree     attention of drafted tokens over a sequence's pages: all of its history, and of the draft what a mask of each token names
  weigh    what attention weight the keys of a sequence had from its new tokens, summed over them and the query heads of a K/V head
  keep     tokens chosen by such weights (first and last ones always), their rows and weights moved together; or what was accepted of a draft

The pages are those of perf/operators.py: the pool of a layer is [page][K/V head][block of 16 tokens][block bytes].  A block holds K, V, then their scales (and for int4
their smallest values), D = head dim, a token's K at place 8 b + 4 a + i of its block for token 8 a + 4 b + i:
  16 bits  K [D / 8][place][8]          V [2][D][8 tokens]
  int8     K [D / 16][place][16]        V [2][D][8 tokens]          scales K [D / 32][place], V [D / 32][16 tokens], fp32
  int4     K [D / 32][place][16 bytes]  V [2][D / 32][16][8 bytes]  the same, then smallest values alike, 16 bits; the byte of value
           e < 16 of a group of 32 holds value e + 16 in its high half
Weights are fp32, [page][K/V head][token of the page].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
GROUP = 32
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
PLACE = [8 * (t // 4 % 2) + 4 * (t // 8) + t % 4 for t in range(16)]


# ------------------------------------------------------------------------------------------ the cases
def case(name, op, seqs, new, kv, heads, kv_heads, dim, page, store, dtype, *, ragged=False, prior=False, axes=1, pairs=0, adjacent=False, window=0,
         sinks=0, budget=0, recent=0, accept=False):
    """seqs sequences of up to kv tokens, of which up to `new` are new.  ragged: lengths fall off over the batch.
    rotate: axes of the positions, pairs of values that turn, adjacent or half a row apart.  keep: the tokens that stay (budget), `sinks` first and `recent` last
    ones among them; or (accept) a path of a draft."""
    c = dict(op=op, seqs=seqs, new=new, kv=kv, heads=heads, kv_heads=kv_heads, dim=dim, page=page, store=store, dtype=dtype, ragged=ragged, prior=prior,
             axes=axes, pairs=pairs or dim // 2, adjacent=adjacent, window=window, sinks=sinks, budget=budget, recent=recent, accept=accept)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next tokens of 32 conversations, in one layer: all launch latency.
        case("rotate-step", "rotate", 32, 1, 9000, 32, 8, 128, 16, "16", "bf16", ragged=True),
        # The patches of eight frames, 576 each, with time, row and column.
        case("rotate-frames", "rotate", 8, 576, 576, 32, 32, 128, 16, "16", "fp16", axes=3),
        # Long documents, half of each row turned, neighbours together.
        case("rotate-long", "rotate", 2, 10001, 70000, 40, 40, 128, 16, "16", "bf16", pairs=32, adjacent=True),
        # One conversation's draft of seven tokens.
        case("tree-1", "tree", 1, 7, 777, 32, 8, 128, 16, "16", "fp16"),
        # Short answers about a video, drafted, joined with what the frames gave; 4-bit cache.
        case("tree-after-frames", "tree", 8, 25, 301, 32, 32, 128, 32, "int4", "fp16", ragged=True, prior=True),
        # A serving batch of drafts over histories of hundreds to thousands of tokens, 8-bit cache.
        case("tree-batch-int8", "tree", 24, 16, 6000, 32, 8, 128, 64, "int8", "bf16", ragged=True),
        # Wide drafts for few long conversations.
        case("tree-wide", "tree", 4, 64, 9000, 32, 8, 128, 64, "16", "bf16", ragged=True),
        # What a step's single tokens attended to, 8-bit cache.
        case("weigh-step", "weigh", 16, 1, 8192, 32, 8, 128, 64, "int8", "bf16", ragged=True),
        # What the last 32 tokens of two long documents look at, before those are cut down; 4-bit cache.
        case("weigh-last", "weigh", 2, 32, 20001, 32, 8, 128, 64, "int4", "fp16", ragged=True),
        # A whole prompt: every pair of tokens.
        case("weigh-prompt", "weigh", 1, 8192, 8192, 32, 8, 128, 128, "16", "bf16"),
        # What was accepted of a batch's drafts: the path's rows move together in the pages that they were written to.
        case("accept", "keep", 32, 16, 2000, 32, 8, 128, 16, "16", "bf16", ragged=True, accept=True),
        # Three long texts cut down to 4096 tokens a head, into pages of their own.
        case("evict", "keep", 3, 24001, 24001, 32, 8, 128, 64, "16", "fp16", ragged=True, budget=4096, sinks=4, recent=512),
    ]


def draw(rng):
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["rotate", "tree", "weigh", "keep"])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (32, 4), (40, 40), (24, 8), (8, 1)])
    dim = rng.choice([64, 128, 128])
    shape = dict(heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([16, 32, 64, 128]), store=rng.choice(["16", "int8", "int4"]),
                 dtype=rng.choice(["fp16", "bf16"]), ragged=rng.random() < 0.7)
    if op == "rotate":
        seqs = size(1, 48)
        new = size(1, max(1, 20000 // seqs))
        return case(None, op, seqs, new, new + size(1, 100000), **shape, axes=rng.choice([1, 1, 2, 3, 4]), pairs=rng.choice([dim // 2, dim // 2, dim // 4, 12]),
                    adjacent=rng.random() < 0.4)
    most_rows = (1 << 20) // kv_heads                                         # rows of K
    if op == "tree":
        seqs = size(1, 48)
        new = size(1, 64)
        return case(None, op, seqs, new, new + size(1, max(2, min(20000, most_rows // seqs - new))), **shape, prior=rng.random() < 0.4)
    if op == "weigh":
        more = dict(window=size(16, 4096), sinks=rng.choice([0, 1, 4, 20, 64])) if rng.random() < 0.3 else {}
        if rng.random() < 0.5:
            seqs = size(1, 48)
            return case(None, op, seqs, 1, size(16, max(17, most_rows // seqs)), **shape, **more)
        seqs = size(1, 12)
        new = size(2, 4096)
        kv = new + size(1, max(2, min(20000, most_rows // seqs - new)))
        new = max(2, min(new, (1 << 24) // (seqs * kv)))                      # the largest listed case has 2^25 pairs a head
        return case(None, op, seqs, new, kv, **shape, **more)
    if rng.random() < 0.3:
        return case(None, op, size(1, 48), size(2, 64), 64 + size(1, 3000), **shape, accept=True)
    seqs = size(1, 16)
    kv = size(8, max(9, min(24000, (1 << 20) // (2 * seqs * kv_heads))))
    budget = size(2, kv)
    sinks, recent = rng.randint(0, min(8, budget // 4)), rng.randint(0, budget // 2)
    return case(None, op, seqs, kv, kv, **shape, budget=budget, sinks=sinks, recent=recent)


def lengths(c):
    """(new tokens, tokens with the new ones) of every sequence."""
    new, kv = [], []
    for s in range(c["seqs"]):
        fall = 1.0 - 0.93 * s / c["seqs"] if c["ragged"] else 1.0
        total = max(1, int(c["kv"] * fall))
        n = min(total, c["new"])
        if c["op"] in ("rotate", "keep") and c["ragged"]:
            n = min(total, max(1, int(c["new"] * fall)))
        new.append(n)
        kv.append(total)
    if c["op"] == "keep" and not c["accept"]:
        new = kv                                                              # of all tokens
    return new, kv


def row_bytes(c):
    d = c["dim"]
    return {"16": 2 * d, "int8": d + d // 8, "int4": d // 2 + d // 8 + d // 16}[c["store"]]


def work(c):
    new, kv = lengths(c)
    t, h, hq, d, r = sum(new), c["kv_heads"], c["heads"], c["dim"], row_bytes(c)
    if c["op"] == "rotate":
        return {"bytes": t * ((hq + h) * 4 * d + 4 * c["axes"]), "flops": 6 * c["pairs"] * (hq + h) * t}
    if c["op"] == "keep":
        if c["accept"]:                                   # draft in, the path's rows moved and read back
            path = sum(max(1, n // 3) for n in new)
            return {"bytes": 2 * h * (t * (2 * d + r) + path * (3 * r + 2 * d)), "flops": 0}
        stay = sum(min(n, c["budget"]) for n in new)      # weights in, rows and weights moved, rows read back
        return {"bytes": h * (4 * t + stay * (4 + 12 + 2 * (3 * r + 2 * d))), "flops": 0}
    keys = pairs = 0
    for n, total in zip(new, kv):
        first = total - n
        if not c["window"]:
            keys += total
            pairs += n * first + n * (n + 1) // 2
            continue
        lo = max(0, first - c["window"] + 1)
        keys += total - lo + min(c["sinks"], lo)
        for p in range(first, total):
            lo = max(0, p - c["window"] + 1)
            pairs += p + 1 - lo + min(c["sinks"], lo)
    if c["op"] == "weigh":
        return {"bytes": h * (r * keys + 4 * sum(kv)) + t * hq * (2 * d + 4), "flops": 2 * d * hq * pairs}
    return {"bytes": 2 * r * h * keys + t * (hq * (4 * d + 4 + (4 * d + 4 if c["prior"] else 0)) + 8), "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------ inputs
def parts_of(c):
    """Offsets in bytes of a block's K, V, scales of K and of V, smallest values of K and of V, and its size."""
    d = c["dim"]
    code = {"16": 32 * d, "int8": 16 * d, "int4": 8 * d}[c["store"]]
    scale = 0 if c["store"] == "16" else 2 * d                                # 16 tokens x d / 32 x 4 bytes
    zero = d if c["store"] == "int4" else 0
    at = [0]
    for n in (code, code, scale, scale, zero, zero):
        at.append(at[-1] + n)
    return at


def fields(c, pool):
    """Views of the pool's parts, each [page][K/V head][block][...] as described at the top."""
    d, at, dt = c["dim"], parts_of(c), DTYPES[c["dtype"]]

    def part(dtype, k, shape):
        n = dtype.itemsize
        return pool.view(dtype)[..., at[k] // n:at[k + 1] // n].unflatten(-1, shape)

    if c["store"] == "16":
        return dict(k=part(dt, 0, (d // 8, 16, 8)), v=part(dt, 1, (2, d, 8)))
    if c["store"] == "int8":
        f = dict(k=part(torch.int8, 0, (d // 16, 16, 16)), v=part(torch.int8, 1, (2, d, 8)))
    else:
        f = dict(k=part(torch.uint8, 0, (d // 32, 16, 16)), v=part(torch.uint8, 1, (2, d // 32, 16, 8)))
    f.update(ks=part(torch.float32, 2, (d // 32, 16)), vs=part(torch.float32, 3, (d // 32, 16)))
    if c["store"] == "int4":
        f.update(kz=part(dt, 4, (d // 32, 16)), vz=part(dt, 5, (d // 32, 16)))
    return f


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new, kv = lengths(c)
    dt, d, h, hq, page, n, op = DTYPES[c["dtype"]], c["dim"], c["kv_heads"], c["heads"], c["page"], c["seqs"], c["op"]
    start = [0]
    for x in new:
        start.append(start[-1] + x)
    t, evict = start[-1], op == "keep" and not c["accept"]
    held = [0 if op == "rotate" else -(-x // page) for x in kv]               # pages of each sequence
    fresh = [-(-min(x, c["budget"]) // page) if evict else 0 for x in kv]     # and of what stays of it
    n_pages = sum(held) + sum(fresh) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table, to = (torch.full((n, max(1, max(pages))), -1, dtype=torch.int32, device=DEV) for pages in (held, fresh))
    at = 0
    for tab, pages in ((table, held), (to, fresh)):
        for s in range(n):
            tab[s, :pages[s]] = order[at:at + pages[s]]
            at += pages[s]
    state = dict(c=c, table=table, new=max(new), kv=max(kv), tokens=t,
                 start=torch.tensor(start, dtype=torch.int32, device=DEV), length=torch.tensor(kv, dtype=torch.int32, device=DEV),
                 pool=torch.zeros((n_pages, h, page // 16, parts_of(c)[-1]), dtype=torch.uint8, device=DEV))
    # what a layer's projection gives for the new tokens: queries, keys and values side by side; channels differ in scale
    channel = torch.exp(0.5 * torch.randn((2, h, d), generator=g, device=DEV))
    if not evict:
        qkv = torch.randn((t, hq + 2 * h, d), generator=g, device=DEV)
        qkv[:, hq:] *= channel.reshape(2 * h, d)
        state["qkv"] = qkv.to(dt)
        del qkv
    if op != "rotate":                                                        # the pages as earlier calls and this token's write left them
        for s in range(n):
            for lo in range(0, kv[s], 1 << 16):
                at = torch.arange(lo, min(kv[s], lo + (1 << 16)), device=DEV)
                k, v = ((torch.randn((len(at), h, d), generator=g, device=DEV) * channel[i]).to(dt) for i in (0, 1))
                write_rows(c, state["pool"], k, v, table[s].long()[at // page], at % page)
    if op == "rotate":
        # places in the text; or frame, row and column of a 24 x 24 grid of patches, from where the text before it ends
        row = torch.arange(t, device=DEV)
        seq = torch.searchsorted(state["start"], row, right=True) - 1
        first = state["length"][seq] - (state["start"][seq + 1] - state["start"][seq])
        i = row - state["start"][seq]
        after = torch.randint(0, 30, (n,), generator=g, device=DEV)[seq]
        axes = [i] if c["axes"] == 1 else [i // 576 + seq, i // 24 % 24, i % 24, i % 576][:c["axes"]]
        state["position"] = torch.stack([first + after + a for a in axes]).to(torch.int32).contiguous()
        state["frequency"] = 10000.0 ** (-torch.arange(c["pairs"], dtype=torch.float64, device=DEV) / c["pairs"])
        state["sections"] = [c["pairs"] * (a + 1) // c["axes"] - c["pairs"] * a // c["axes"] for a in range(c["axes"])]
    if op == "tree" or c["accept"]:
        # each drafted token follows the history or one before it, more often a late one; what it sees is itself and what it follows
        late = torch.rand((n, max(new)), generator=g, device=DEV).sqrt()
        parent = (late * (torch.arange(max(new), device=DEV) + 1)).long() - 1
        seen = torch.zeros((n, max(new) + 1), dtype=torch.int64, device=DEV)   # the last one: the history
        each = torch.arange(n, device=DEV)
        for i in range(max(new)):
            seen[:, i] = seen[each, parent[:, i]] | torch.tensor(1, device=DEV) << i
        row = torch.arange(t, device=DEV)
        seq = torch.searchsorted(state["start"], row, right=True) - 1
        state["seen"] = seen[seq, row - state["start"][seq]].contiguous()
    if c["prior"]:
        state["prior"] = torch.randn((t, hq, d), generator=g, device=DEV) * 0.1
        state["prior_lse"] = 5.0 + torch.randn((t, hq), generator=g, device=DEV)
    if op == "weigh":                                                         # log-sums as the attention of the same tokens gave them
        state["lse"] = torch.logsumexp(logits(state, causal(state), keys(state)[0]), -1).permute(0, 3, 1, 2).flatten(2)[rows_of(state)].contiguous()
        state["weights"] = torch.zeros((n_pages, h, page), device=DEV)
    if c["accept"]:                                                           # a third of each draft, in its order
        keep = torch.full((n, 1, max(1, max(new) // 3)), -1, dtype=torch.int32, device=DEV)
        for s in range(n):
            m = max(1, new[s] // 3)
            keep[s, 0, :m] = torch.randperm(new[s], generator=g, device=DEV)[:m].sort().values
        state["keep"] = keep
        stay = [max(1, x // 3) for x in new]
    if evict:
        # sums of attention weights: most of them small, many the same
        x = torch.exp(2.0 * torch.randn((n_pages, h, page), generator=g, device=DEV))
        state["weights"] = torch.where(x < 0.5, torch.floor(x * 16) / 16, x)
        state["to"] = to
        stay = [min(x, c["budget"]) for x in new]
    if op == "keep":                                                          # the rows that stayed, for reading them back
        back = [0]
        for x in stay:
            back.append(back[-1] + x)
        state["back"] = torch.tensor(back, dtype=torch.int32, device=DEV)
        state["left"] = torch.tensor([b - a + x for a, b, x in zip(new, kv, stay)], dtype=torch.int32, device=DEV)
        state["stay"] = back[-1]
    if own:                                                                   # the handle, and the batch that all layers of a step share
        from paper_2602_14236_amd import binding
        cfg = binding.make_pages_config(n_layers=1, n_kv_heads=h, n_heads=hq, head_dim=d, page_tokens=page, n_pages=n_pages,
                                        dtype=dt, store=c["store"])
        state["pages"] = binding.SaliPages(cfg, DEV, pool=state["pool"])
        if op == "rotate":
            state["rotary"] = binding.Rotary(state["frequency"], state["sections"], adjacent=c["adjacent"])
        else:
            state["batch"] = binding.PageBatch(state["start"], state["length"], table, t, max_q=state["new"], max_kv=state["kv"])
        if op == "keep":
            state["after"] = binding.PageBatch(state["back"], state["left"], to if evict else table, state["stay"], max_q=max(stay), max_kv=state["kv"])
    return state


# ------------------------------------------------------------------------------------------ plain forms
def quantised(c, x):
    """Codes [T, H, D / 32, 32], scales and smallest values [T, H, D / 32] of rows x, every step one operation in 32 bits."""
    g = x.float().unflatten(-1, (c["dim"] // GROUP, GROUP))
    if c["store"] == "int8":
        m, low, most = g.abs().amax(-1), None, 127.0
    else:
        low = g.amin(-1)
        m, most = g.amax(-1) - low, 15.0
        g = g - low[..., None]
    steps = torch.full_like(m, most)
    scale, inv = m / steps, torch.where(m > 0, steps / m, 0.0)
    return (g * inv[..., None]).round().clamp(-most if low is None else 0.0, most), scale, low


def write_rows(c, pool, k, v, page, place):
    """Rows k and v [T, H, D] into tokens `place` of pages `page`."""
    f, dt, d = fields(c, pool), DTYPES[c["dtype"]], c["dim"]
    block, tok = place // 16, place % 16
    slot = torch.tensor(PLACE, device=DEV)[tok]
    if c["store"] == "16":
        f["k"][page, :, block, :, slot, :] = k.unflatten(-1, (d // 8, 8))
        f["v"][page, :, block, tok // 8, :, tok % 8] = v
        return
    for x, codes, scales, lows, at in ((k, f["k"], f["ks"], f.get("kz"), slot), (v, f["v"], f["vs"], f.get("vz"), tok)):
        q, scale, low = quantised(c, x)
        scales[page, :, block, :, at] = scale
        if low is None:
            q = q.to(torch.int8).flatten(-2)
            if x is k:
                codes[page, :, block, :, slot, :] = q.unflatten(-1, (d // 16, 16))
            else:
                codes[page, :, block, tok // 8, :, tok % 8] = q
            continue
        lows[page, :, block, :, at] = low.to(dt)
        q = q.to(torch.uint8)
        q = q[..., :16] | q[..., 16:] << 4
        if x is k:
            codes[page, :, block, :, slot, :] = q
        else:
            codes[page, :, block, tok // 8, :, :, tok % 8] = q


def read_rows(c, pool, page, place):
    """The rows that tokens `place` of pages `page` stand for: K and V, [T, H, D]."""
    f, dt = fields(c, pool), DTYPES[c["dtype"]]
    block, tok = place // 16, place % 16
    slot = torch.tensor(PLACE, device=DEV)[tok]
    if c["store"] == "16":
        return f["k"][page, :, block, :, slot, :].flatten(-2), f["v"][page, :, block, tok // 8, :, tok % 8]
    rows = []
    for codes, scales, lows, at in ((f["k"], f["ks"], f.get("kz"), slot), (f["v"], f["vs"], f.get("vz"), tok)):
        scale = scales[page, :, block, :, at][..., None]
        if lows is None:
            q = codes[page, :, block, :, slot, :].flatten(-2) if at is slot else codes[page, :, block, tok // 8, :, tok % 8]
            rows.append((q.unflatten(-1, (-1, GROUP)).float() * scale).to(dt).flatten(-2))
            continue
        q = codes[page, :, block, :, slot, :] if at is slot else codes[page, :, block, tok // 8, :, :, tok % 8]
        q = torch.cat((q & 15, q >> 4), -1)
        # code * scale + low rounded once to 32 bits: the product and the sum are exact in 64
        rows.append((q.double() * scale + lows[page, :, block, :, at][..., None]).float().to(dt).flatten(-2))
    return rows


def rows_of(s):
    """Sequence and place among its new tokens of every row."""
    row = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(s["start"], row, right=True) - 1
    return seq, row - s["start"][seq]


def run_rotate(s):
    c, hq, h = s["c"], s["c"]["heads"], s["c"]["kv_heads"]
    q, k = s["qkv"][:, :hq], s["qkv"][:, hq:hq + h]
    if own:
        q_out, k_out = (torch.empty(x.shape, dtype=x.dtype, device=DEV) for x in (q, k))
        s["pages"].rotate(s["rotary"], s["position"], q, k, q_out, k_out)
        return {"q": q_out, "k": k_out}
    m = c["pairs"]
    axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEV), torch.tensor(s["sections"], device=DEV))
    angle = s["position"].double()[axis].T * s["frequency"]                   # [tokens, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = []
    for x in (q, k):
        y = x.float()
        a, b = (y[..., :2 * m:2], y[..., 1:2 * m:2]) if c["adjacent"] else (y[..., :m], y[..., m:2 * m])
        turned = (a * cos - b * sin, b * cos + a * sin)
        turned = torch.stack(turned, -1).flatten(-2) if c["adjacent"] else torch.cat(turned, -1)
        out.append(torch.cat((turned, y[..., 2 * m:]), -1).to(x.dtype))
    return {"q": out[0], "k": out[1]}


def keys(s):
    """K and V rows of every sequence, [n, kv_heads, kv, d]."""
    c, n, kv = s["c"], s["c"]["seqs"], s["kv"]
    j = torch.arange(kv, device=DEV)
    page = s["table"][:, j // c["page"]].clamp(min=0).long()
    k, v = read_rows(c, s["pool"], page.flatten(), (j % c["page"]).repeat(n))
    return [x.unflatten(0, (n, kv)).permute(0, 2, 1, 3).float() for x in (k, v)]


def causal(s):
    """[n, new, kv]: which keys a new token sees."""
    c, j = s["c"], torch.arange(s["kv"], device=DEV)
    at = torch.arange(s["new"], device=DEV)
    count = s["start"].diff()[:, None]
    pos = (s["length"][:, None] - count + at)[..., None]
    seen = (j <= pos) & (at < count)[..., None]
    if c["window"]:
        seen &= (j > pos - c["window"]) | (j < c["sinks"])
    return seen


def drafted(s):
    """The same for a draft: what came before it, and what the token's mask names."""
    j, first = torch.arange(s["kv"], device=DEV), (s["length"] - s["start"].diff())[:, None]
    mask = torch.zeros((s["c"]["seqs"], s["new"]), dtype=torch.int64, device=DEV)
    mask[rows_of(s)] = s["seen"]
    i = j - first                                                             # [n, kv]
    named = (mask[..., None] >> i.clamp(0, 63)[:, None] & 1) == 1
    return ((i < 0)[:, None] | named & ((i >= 0) & (j < s["length"][:, None]))[:, None]) & (torch.arange(s["new"], device=DEV) < s["start"].diff()[:, None])[..., None]


def logits(s, seen, k):
    """[n, kv_heads, queries of one, new, kv], -inf where a key is out of sight."""
    c, hq, h, d = s["c"], s["c"]["heads"], s["c"]["kv_heads"], s["c"]["dim"]
    qp = torch.zeros((c["seqs"], s["new"], hq, d), device=DEV)
    qp[rows_of(s)] = s["qkv"][:, :hq].float()
    qp = qp.view(c["seqs"], s["new"], h, hq // h, d).permute(0, 2, 3, 1, 4).reshape(c["seqs"], h, -1, d)
    logit = torch.matmul(qp, k.transpose(2, 3)).mul_(d ** -0.5).unflatten(2, (hq // h, s["new"]))
    return logit.masked_fill_(~seen[:, None, None], -math.inf)


def run_tree(s):
    c, hq, d = s["c"], s["c"]["heads"], s["c"]["dim"]
    q = s["qkv"][:, :hq]
    if own:
        out = torch.empty((s["tokens"], hq, d), dtype=q.dtype, device=DEV)
        lse = torch.empty((s["tokens"], hq), dtype=torch.float32, device=DEV)
        s["pages"].attend_tree(0, s["batch"], s["seen"], q, d ** -0.5, out, lse, prior=s.get("prior"), prior_lse=s.get("prior_lse"))
        return {"out": out, "lse": lse}
    k, v = keys(s)
    logit = logits(s, drafted(s), k)
    top = logit.amax(-1, keepdim=True).clamp(min=-1e30)
    p = logit.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, p.shape[2:4]) / total
    lse = (top + total.log())[..., 0]
    seq, at = rows_of(s)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, at]
    lse = lse.permute(0, 3, 1, 2).flatten(2)[seq, at]
    if c["prior"]:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = out * (lse - both).exp()[..., None] + s["prior"] * (s["prior_lse"] - both).exp()[..., None]
        lse = both
    return {"out": out.to(q.dtype), "lse": lse}


def run_weigh(s):
    c, hq, d = s["c"], s["c"]["heads"], s["c"]["dim"]
    if own:
        s["pages"].weigh(0, s["batch"], s["qkv"][:, :hq], d ** -0.5, s["lse"], s["weights"], add=False, window=c["window"], sinks=c["sinks"])
        return {"weights": s["weights"]}
    logit = logits(s, causal(s), keys(s)[0])
    lse = torch.zeros((c["seqs"], s["new"], hq), device=DEV)
    lse[rows_of(s)] = s["lse"]
    lse = lse.unflatten(2, logit.shape[1:3]).permute(0, 2, 3, 1)[..., None]
    w = logit.sub_(lse).exp_().sum((2, 3))                                    # [n, kv_heads, kv]
    j = torch.arange(s["kv"], device=DEV)
    held = j < s["length"][:, None]
    page = s["table"].long()[:, j // c["page"]]
    s["weights"][page[held], :, (j % c["page"]).expand_as(held)[held]] = w.transpose(1, 2)[held]
    return {"weights": s["weights"]}


def run_keep(s):
    c, h, d = s["c"], s["c"]["kv_heads"], s["c"]["dim"]
    dt, evict = DTYPES[c["dtype"]], not c["accept"]
    if own:
        if evict:
            keep = torch.empty((c["seqs"], h, c["budget"]), dtype=torch.int32, device=DEV)
            s["pages"].select(s["batch"], s["weights"], c["budget"], keep, sinks=c["sinks"], recent=c["recent"])
            s["pages"].keep(0, s["batch"], keep, to=s["to"], weights=s["weights"])
        else:
            keep = s["keep"]
            s["pages"].append(0, s["batch"], s["qkv"][:, c["heads"]:c["heads"] + h], s["qkv"][:, c["heads"] + h:])
            s["pages"].keep(0, s["batch"], keep)
        back = torch.empty((2, s["stay"], h, d), dtype=dt, device=DEV)
        s["pages"].read(0, s["after"], back[0], back[1])
        return {"keep": keep, "k": back[0], "v": back[1], "weights": s["weights"]} if evict else {"k": back[0], "v": back[1]}
    count = s["start"].diff()
    first = s["length"] - count
    if evict:
        keep = chosen(s)
    else:
        seq, i = rows_of(s)
        pos = first[seq] + i
        write_rows(c, s["pool"], s["qkv"][:, c["heads"]:c["heads"] + h], s["qkv"][:, c["heads"] + h:], s["table"][seq, pos // c["page"]].long(), pos % c["page"])
        keep = s["keep"].expand(-1, h, -1)
    # parts of a block by token: [..., place, ...] of K's and [..., token, ...] of V's arrays, moved as they are
    i = torch.arange(keep.shape[2], device=DEV)
    held = keep >= 0                                                          # [n, h, budget]
    seq, head, nth = held.nonzero(as_tuple=True)
    pos, dst = first[seq] + keep[seq, head, nth], first[seq] + i[nth]
    page, place = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    to_page, to_place = (s["to"] if evict else s["table"])[seq, dst // c["page"]].long(), dst % c["page"]
    move_rows(c, s["pool"], head, page, place, to_page, to_place)
    at = held[:, 0].nonzero(as_tuple=True)                                    # as many for every head
    dst = first[at[0]] + i[at[1]]
    k, v = read_rows(c, s["pool"], (s["to"] if evict else s["table"])[at[0], dst // c["page"]].long(), dst % c["page"])
    if not evict:
        return {"k": k, "v": v}
    s["weights"][to_page, head, to_place] = s["weights"][page, head, place]
    return {"keep": keep, "k": k, "v": v, "weights": s["weights"]}


def chosen(s):
    """[n, kv_heads, budget]: places that stay, rising, -1 behind the last.  First and last ones, then those of most weight, the first ones of equal weight."""
    c, j, kv, budget = s["c"], torch.arange(s["kv"], device=DEV), s["kv"], s["c"]["budget"]
    page = s["table"][:, j // c["page"]].clamp(min=0).long()
    w = s["weights"][page, :, j % c["page"]].transpose(1, 2)                  # [n, h, kv]
    end = s["length"][:, None]
    w = w.masked_fill(((j < c["sinks"]) | (j >= end - c["recent"]))[:, None], math.inf).masked_fill((j >= end)[:, None], -math.inf)
    best = w.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    best = best.masked_fill(best >= end[..., None], kv).sort(-1).values
    best = torch.nn.functional.pad(best, (0, budget - best.shape[-1]), value=kv)
    return best.masked_fill(best == kv, -1).to(torch.int32)


def move_rows(c, pool, head, page, place, to_page, to_place):
    """Rows of tokens `place` of pages `page`, as they are stored, to tokens `to_place` of pages `to_page`."""
    f, slot = fields(c, pool), torch.tensor(PLACE, device=DEV)
    a, b = (page, head, place // 16), (to_page, head, to_place // 16)
    t, u = place % 16, to_place % 16
    moved = {}
    for name, x in f.items():                                                 # all read before the first is written
        moved[name] = x[(*a, t // 8, ..., t % 8)] if name == "v" else x[(*a, slice(None), slot[t] if name[0] == "k" else t)]
    for name, x in f.items():
        if name == "v":
            x[(*b, u // 8, ..., u % 8)] = moved[name]
        else:
            x[(*b, slice(None), slot[u] if name[0] == "k" else u)] = moved[name]


def run(s):
    return {"rotate": run_rotate, "tree": run_tree, "weigh": run_weigh, "keep": run_keep}[s["c"]["op"]](s)


# ------------------------------------------------------------------------------------------ in 64 bits
def stored(c, flat, base, tok, k_side):
    """[len(base), D]: the rows at token `tok` of the blocks whose first bytes are `base`, by the address of every value."""
    d, at, dt = c["dim"], parts_of(c), DTYPES[c["dtype"]]
    e = torch.arange(d, device=DEV)
    base, tok = base[:, None], tok[:, None]
    place = 8 * (tok // 4 % 2) + 4 * (tok // 8) + tok % 4

    def get(dtype, byte):
        return flat.view(dtype)[byte // dtype.itemsize]

    if c["store"] == "16":
        byte = (e // 8 * 16 + place) * 16 + e % 8 * 2 if k_side else ((tok // 8 * d + e) * 8 + tok % 8) * 2
        return get(dt, base + at[0 if k_side else 1] + byte).double()
    side = 0 if k_side else 1
    scale = get(torch.float32, base + at[2 + side] + (e // 32 * 16 + (place if k_side else tok)) * 4).double()
    if c["store"] == "int8":
        byte = (e // 16 * 16 + place) * 16 + e % 16 if k_side else (tok // 8 * d + e) * 8 + tok % 8
        return (get(torch.int8, base + at[side] + byte).double() * scale).float().to(dt).double()
    low = get(dt, base + at[4 + side] + (e // 32 * 16 + (place if k_side else tok)) * 2).double()
    byte = (e // 32 * 16 + place) * 16 + e % 16 if k_side else ((tok // 8 * (d // 32) + e // 32) * 16 + e % 16) * 8 + tok % 8
    code = get(torch.uint8, base + at[side] + byte).int() >> e % 32 // 16 * 4 & 15
    return (code.double() * scale + low).float().to(dt).double()


def exact(c, seed):
    global own
    was, own = own, False                                # the inputs alone
    try:
        s = prepare(c, seed)
    finally:
        own = was
    new, kv = lengths(c)
    hq, h, d, size = c["heads"], c["kv_heads"], c["dim"], parts_of(c)[-1]
    if c["op"] == "rotate":
        # as complex numbers: a pair times exp(i angle)
        which = [a for a in range(c["axes"]) for _ in range(s["sections"][a])]
        angle = torch.stack([s["position"][a].double() * s["frequency"][i] for i, a in enumerate(which)], -1)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        first, second = (range(0, 2 * c["pairs"], 2), range(1, 2 * c["pairs"], 2)) if c["adjacent"] else (range(c["pairs"]), range(c["pairs"], 2 * c["pairs"]))
        out = []
        for x in (s["qkv"][:, :hq], s["qkv"][:, hq:hq + h]):
            x = x.double()
            z = torch.complex(x[..., list(first)], x[..., list(second)]) * turn
            x[..., list(first)], x[..., list(second)] = z.real, z.imag
            out.append(x)
        return {"q": out[0], "k": out[1]}
    flat = s["pool"].flatten()

    def block_of(i, j, head):
        """First byte of the block of positions j of sequence i, and the tokens there."""
        return ((s["table"][i].long()[j // c["page"]] * h + head) * (c["page"] // 16) + j % c["page"] // 16) * size, j % 16

    if c["op"] == "keep":
        rows = [torch.zeros((s["stay"], h, d), dtype=torch.float64, device=DEV) for _ in range(2)]
        keep = np.full((c["seqs"], h, c["budget"]), -1, dtype=np.int32)
        back = s["back"].tolist()
        weights = s["weights"].clone() if not c["accept"] else None
        for i in range(c["seqs"]):
            for head in range(h):
                n = back[i + 1] - back[i]
                if c["accept"]:
                    # the draft's rows are the new ones, stored as their type's steps in 32 bits have it
                    at = s["start"][i] + s["keep"][i, 0, :n].long()
                    for side in (0, 1):
                        x = s["qkv"][at, hq + side * h + head].double()
                        if c["store"] != "16":
                            x = x.reshape(n, d // 32, 32)
                            lo = x.min(-1, keepdim=True).values if c["store"] == "int4" else torch.zeros_like(x[..., :1])
                            span = (x - lo).abs().max(-1, keepdim=True).values.float().double()
                            most = 15 if c["store"] == "int4" else 127
                            code = torch.round(((x - lo).float().double() * (most / span).float().double()).float().double())
                            x = (lo + torch.where(span > 0, code * (span / most).float().double(), 0.0)).reshape(n, d)
                        rows[side][back[i]:back[i + 1], head] = x
                    continue
                j = torch.arange(kv[i], device=DEV)
                w = s["weights"][s["table"][i].long()[j // c["page"]], head, j % c["page"]].cpu().numpy().astype(np.float64)
                always = np.zeros(kv[i], dtype=bool)
                always[:c["sinks"]] = True
                always[max(0, kv[i] - c["recent"]):] = True
                rank = np.lexsort((np.arange(kv[i]), -w, ~always))            # always first, then by weight, then by place
                stay = np.sort(rank[:n])
                keep[i, head, :n] = stay
                stay, dst = torch.from_numpy(stay).to(DEV), torch.arange(n, device=DEV)
                base, tok = block_of(i, stay, head)
                for side in (0, 1):
                    rows[side][back[i]:back[i + 1], head] = stored(c, flat, base, tok, side == 0)
                weights[s["to"][i].long()[dst // c["page"]], head, dst % c["page"]] = torch.from_numpy(w).to(DEV)[stay].float()
        if c["accept"]:
            return {"k": rows[0], "v": rows[1]}
        return {"keep": torch.from_numpy(keep), "k": rows[0], "v": rows[1], "weights": weights.double()}
    out = torch.zeros((s["tokens"], hq, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["tokens"], hq), dtype=torch.float64, device=DEV)
    weights = s["weights"].double() if c["op"] == "weigh" else None
    first = 0
    for i in range(c["seqs"]):
        j = torch.arange(kv[i], device=DEV)
        pos = torch.arange(kv[i] - new[i], kv[i], device=DEV)[:, None]
        if c["op"] == "tree":
            hidden = torch.zeros((new[i], kv[i]), dtype=torch.bool, device=DEV)
            for t, m in enumerate(s["seen"][first:first + new[i]].tolist()):
                hidden[t, kv[i] - new[i]:] = torch.tensor([m >> b & 1 == 0 for b in range(new[i])], device=DEV)
        else:
            hidden = j > pos
            if c["window"]:
                hidden = hidden | ((j <= pos - c["window"]) & (j >= c["sinks"]))
        for head in range(h):
            base, tok = block_of(i, j, head)
            k = stored(c, flat, base, tok, True)
            v = stored(c, flat, base, tok, False) if c["op"] == "tree" else None
            w = torch.zeros(kv[i], dtype=torch.float64, device=DEV)
            for one in range(head * (hq // h), (head + 1) * (hq // h)):
                x = s["qkv"][first:first + new[i], one].double() @ k.T / math.sqrt(d)
                x = x.masked_fill_(hidden, -math.inf)
                if c["op"] == "weigh":
                    w += torch.exp(x - s["lse"][first:first + new[i], one, None].double()).sum(0)
                    continue
                lse[first:first + new[i], one] = torch.logsumexp(x, -1)
                out[first:first + new[i], one] = torch.softmax(x, -1) @ v
            if c["op"] == "weigh":
                weights[s["table"][i].long()[j // c["page"]], head, j % c["page"]] = w
        first += new[i]
    if c["op"] == "weigh":
        return {"weights": weights}
    if c["prior"]:
        l2 = s["prior_lse"].double()
        w = torch.sigmoid(lse - l2)[..., None]
        out = w * out + (1 - w) * s["prior"].double()
        lse = lse + torch.nn.functional.softplus(l2 - lse)
    return {"out": out, "lse": lse}
