"""The paged cache of text tokens and its attention, as cases that can be timed and compared.

  write    new K/V rows of a batch of sequences into the pages, quantised on the way, and those rows read back
  attend   causal attention of each sequence's new tokens over its pages: single tokens, chunks, whole prompts, mixed
  window   the same where a token sees a window behind it and a few first tokens that stay visible (sinks)

An attention case with `prior` starts from an output and log-sum over other keys (the video frames that came before the
text) and joins the two.  Head counts are those of the repository's workloads (32 or 40 K/V heads, 32 query heads over 8).

Pages.  The pool of a layer is [page][K/V head][block of 16 tokens][block bytes].  A block holds K, V, then their scales (and
for int4 their smallest values), D = head dim, a token's K at place 8 b + 4 a + i of its block for token 8 a + 4 b + i:
  16 bits  K [D / 8][place][8]          V [2][D][8 tokens]
  int8     K [D / 16][place][16]        V [2][D][8 tokens]          scales K [D / 32][place], V [D / 32][16 tokens], fp32
  int4     K [D / 32][place][16 bytes]  V [2][D / 32][16][8 bytes]  the same, then smallest values alike, 16 bits; the byte of value
           e < 16 of a group of 32 holds value e + 16 in its high half
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
GROUP = 32
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
PLACE = [8 * (t // 4 % 2) + 4 * (t // 8) + t % 4 for t in range(16)]


# ------------------------------------------------------------------------------------------ the cases
def case(name, op, seqs, new, kv, heads, kv_heads, dim, page, store, dtype, *, mixed=False, ragged=False, window=0, sinks=0, prior=False):
    """seqs sequences of up to kv tokens, of which up to `new` are new.  ragged: lengths fall off over the batch.
    mixed: three sequences in four bring a single token."""
    c = dict(op=op, seqs=seqs, new=new, kv=kv, heads=heads, kv_heads=kv_heads, dim=dim, page=page, store=store, dtype=dtype,
             mixed=mixed, ragged=ragged, window=window, sinks=sinks, prior=prior)
    return dict(c, name=name) if name else c


def listed():
    return [
        # A decode step of 32 conversations: one row each, 8 K/V heads. The smallest write, all launch latency.
        case("write-step", "write", 32, 1, 500, 32, 8, 128, 16, "int8", "bf16", ragged=True),
        # A prompt of a 7B-shaped model as it comes, full precision.
        case("write-prompt", "write", 1, 2048, 2048, 32, 32, 128, 64, "16", "fp16"),
        # Three long documents, a 13B-shaped model, four bits; lengths that fit neither blocks nor pages.
        case("write-long-int4", "write", 3, 12001, 12001, 40, 40, 128, 128, "int4", "bf16", ragged=True),
        # One conversation's next token: the smallest attention.
        case("step-1", "attend", 1, 1, 777, 32, 8, 128, 16, "16", "fp16"),
        # The next tokens of a serving batch, lengths from hundreds to thousands, 8-bit cache.
        case("step-batch-int8", "attend", 48, 1, 8192, 32, 8, 128, 64, "int8", "bf16", ragged=True),
        # One token over a very long context: the cache's bytes are all that counts.
        case("step-long", "attend", 1, 1, 131072, 32, 8, 128, 64, "16", "fp16"),
        # A question after a video: short texts, a head per K/V head, joined with what the frames gave.
        case("step-after-frames", "attend", 8, 1, 300, 32, 32, 128, 32, "16", "fp16", ragged=True, prior=True),
        # A chunk of a prompt that continues a conversation about a video.
        case("chunk-after-frames", "attend", 1, 512, 4100, 32, 32, 128, 64, "16", "fp16", prior=True),
        # A serving step that mixes chunks of prompts with single tokens, 8-bit cache.
        case("mixed-int8", "attend", 24, 333, 6000, 32, 8, 128, 32, "int8", "bf16", mixed=True, ragged=True),
        # A whole prompt at once: bound by the matrix cores.
        case("prompt", "attend", 1, 8192, 8192, 32, 8, 128, 128, "16", "bf16"),
        # Long conversations that remember a window and their beginning, 4-bit cache, after a video.
        case("window-step-int4", "window", 16, 1, 32768, 32, 8, 128, 64, "int4", "fp16", ragged=True, window=4096, sinks=4, prior=True),
        # Chunks of long documents under a window; small heads.
        case("window-chunk", "window", 2, 1024, 16384, 32, 4, 64, 64, "16", "bf16", ragged=True, window=2048, sinks=20),
    ]


def draw(rng):
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["write", "attend", "attend", "window"])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (32, 4), (40, 40), (24, 8), (8, 1)])
    shape = dict(heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]),
                 store=rng.choice(["16", "int8", "int4"]), dtype=rng.choice(["fp16", "bf16"]), ragged=rng.random() < 0.7)
    if op == "write":
        seqs = size(1, 48)
        new = size(1, max(1, 12000 // seqs))
        return case(None, op, seqs, new, new + size(1, 2000), **shape)
    more = dict(prior=rng.random() < 0.4)
    if op == "window":
        more.update(window=size(16, 4096), sinks=rng.choice([0, 1, 4, 20, 64]))
    if rng.random() < 0.5:
        seqs = size(1, 64)
        kv = size(16, max(17, (1 << 20) // (seqs * kv_heads)))               # rows of the longest listed context
        return case(None, op, seqs, 1, kv, **shape, **more)
    seqs = size(1, 16)
    new = size(2, 4096)
    kv = new + size(1, max(2, min(12000, (1 << 20) // (seqs * kv_heads) - new)))
    new = max(2, min(new, (1 << 24) // (seqs * kv)))     # the largest listed case has 2^25 pairs a head
    return case(None, op, seqs, new, kv, mixed=seqs > 3 and rng.random() < 0.5, **shape, **more)


def lengths(c):
    """(new tokens, tokens with the new ones) of every sequence."""
    new, kv = [], []
    for s in range(c["seqs"]):
        fall = 1.0 - 0.93 * s / c["seqs"] if c["ragged"] else 1.0
        total = max(1, int(c["kv"] * fall))
        n = min(total, c["new"])
        if c["op"] == "write" and c["ragged"]:
            n = min(total, max(1, int(c["new"] * fall)))
        if c["mixed"] and s % 4:
            n = 1
        new.append(n)
        kv.append(total)
    return new, kv


def row_bytes(c):
    d = c["dim"]
    return {"16": 2 * d, "int8": d + d // 8, "int4": d // 2 + d // 8 + d // 16}[c["store"]]


def work(c):
    new, kv = lengths(c)
    t, h, hq, d, r = sum(new), c["kv_heads"], c["heads"], c["dim"], row_bytes(c)
    if c["op"] == "write":
        return {"bytes": 2 * t * h * (4 * d + 2 * r), "flops": 0}
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
    return {"bytes": 2 * r * h * keys + t * hq * (4 * d + 4 + (4 * d + 4 if c["prior"] else 0)), "flops": 4 * d * hq * pairs}


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
    dt, d, h, hq, page, n = DTYPES[c["dtype"]], c["dim"], c["kv_heads"], c["heads"], c["page"], c["seqs"]
    held = [-(-x // page) for x in kv]                                        # pages of each sequence
    n_pages = sum(held) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((n, max(held)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s in range(n):
        table[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    start = [0]
    for x in new:
        start.append(start[-1] + x)
    t = start[-1]
    state = dict(c=c, table=table, new=max(new), kv=max(kv), tokens=t,
                 start=torch.tensor(start, dtype=torch.int32, device=DEV), length=torch.tensor(kv, dtype=torch.int32, device=DEV),
                 pool=torch.zeros((n_pages, h, page // 16, parts_of(c)[-1]), dtype=torch.uint8, device=DEV))
    # what a layer's projection gives for the new tokens: queries, keys and values side by side; channels differ in scale
    channel = torch.exp(0.5 * torch.randn((2, h, d), generator=g, device=DEV))
    qkv = torch.randn((t, hq + 2 * h, d), generator=g, device=DEV)
    qkv[:, hq:] *= channel.reshape(2 * h, d)
    state["qkv"] = qkv.to(dt)
    del qkv
    if c["op"] != "write":                                                    # the pages as earlier calls and this token's write left them
        for s in range(n):
            for lo in range(0, kv[s], 1 << 16):
                at = torch.arange(lo, min(kv[s], lo + (1 << 16)), device=DEV)
                k, v = ((torch.randn((len(at), h, d), generator=g, device=DEV) * channel[i]).to(dt) for i in (0, 1))
                write_rows(c, state["pool"], k, v, table[s].long()[at // page], at % page)
    if c["prior"]:
        state["prior"] = torch.randn((t, hq, d), generator=g, device=DEV) * 0.1
        state["prior_lse"] = 5.0 + torch.randn((t, hq), generator=g, device=DEV)
    if own:                                                                   # the handle, and the batch that all layers of a step share
        from paper_2602_14236_amd import binding
        cfg = binding.make_pages_config(n_layers=1, n_kv_heads=h, n_heads=hq, head_dim=d, page_tokens=page, n_pages=n_pages,
                                        dtype=dt, store=c["store"])
        state["pages"] = binding.SaliPages(cfg, DEV, pool=state["pool"])
        state["batch"] = binding.PageBatch(state["start"], state["length"], table, t, max_q=state["new"], max_kv=state["kv"])
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


def run_write(s):
    c, qkv, hq, h = s["c"], s["qkv"], s["c"]["heads"], s["c"]["kv_heads"]
    k, v = qkv[:, hq:hq + h], qkv[:, hq + h:]
    if own:
        s["pages"].append(0, s["batch"], k, v)
        back = torch.empty((2, s["tokens"], h, c["dim"]), dtype=qkv.dtype, device=DEV)
        s["pages"].read(0, s["batch"], back[0], back[1])
        return {"k": back[0], "v": back[1]}
    t = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(s["start"], t, right=True) - 1
    pos = s["length"][seq] - s["start"][seq + 1] + t
    page, place = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    write_rows(c, s["pool"], k, v, page, place)
    k, v = read_rows(c, s["pool"], page, place)
    return {"k": k, "v": v}


def run_attend(s):
    c, hq, h, d = s["c"], s["c"]["heads"], s["c"]["kv_heads"], s["c"]["dim"]
    q, scale = s["qkv"][:, :hq], d ** -0.5
    if own:
        out = torch.empty((s["tokens"], hq, d), dtype=q.dtype, device=DEV)
        lse = torch.empty((s["tokens"], hq), dtype=torch.float32, device=DEV)
        s["pages"].attend(0, s["batch"], q, scale, out, lse, window=c["window"], sinks=c["sinks"], prior=s.get("prior"),
                          prior_lse=s.get("prior_lse"))
        return {"out": out, "lse": lse}
    n, new, kv = c["seqs"], s["new"], s["kv"]
    j = torch.arange(kv, device=DEV)
    page = s["table"][:, j // c["page"]].clamp(min=0).long()                  # [n, kv]
    k, v = read_rows(c, s["pool"], page.flatten(), (j % c["page"]).repeat(n))
    k, v = (x.unflatten(0, (n, kv)).permute(0, 2, 1, 3).float() for x in (k, v))          # [n, h, kv, d]
    t = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(s["start"], t, right=True) - 1
    at = t - s["start"][seq]
    qp = torch.zeros((n, new, hq, d), device=DEV)
    qp[seq, at] = q.float()
    qp = qp.view(n, new, h, hq // h, d).permute(0, 2, 1, 3, 4).reshape(n, h, new * (hq // h), d)
    pos = (s["length"] - s["start"].diff())[:, None] + torch.arange(new, device=DEV)      # [n, new]
    seen = j <= pos[..., None]
    if c["window"]:
        seen &= (j > pos[..., None] - c["window"]) | (j < c["sinks"])
    logit = torch.matmul(qp, k.transpose(2, 3)).mul_(scale).unflatten(2, (new, hq // h))
    logit.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = logit.amax(-1, keepdim=True).clamp(min=-1e30)
    p = logit.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (new, hq // h)) / total
    lse = (top + total.log())[..., 0]
    out, lse = (x.transpose(1, 2)[seq, at].flatten(1, 2) for x in (out, lse))             # [tokens, hq(, d)]
    if c["prior"]:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = out * (lse - both).exp()[..., None] + s["prior"] * (s["prior_lse"] - both).exp()[..., None]
        lse = both
    return {"out": out.to(q.dtype), "lse": lse}


def run(s):
    return run_write(s) if s["c"]["op"] == "write" else run_attend(s)


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
    if c["op"] == "write":
        rows = []
        for x in (s["qkv"][:, hq:hq + h], s["qkv"][:, hq + h:]):
            x = x.double().reshape(s["tokens"], h, d // 32, 32)
            if c["store"] != "16":                       # which code a value gets is defined by steps rounded to 32 bits
                lo = x.min(-1, keepdim=True).values if c["store"] == "int4" else torch.zeros_like(x[..., :1])
                span = (x - lo).abs().max(-1, keepdim=True).values.float().double()
                top = 15 if c["store"] == "int4" else 127
                code = torch.round(((x - lo).float().double() * (top / span).float().double()).float().double())
                x = lo + torch.where(span > 0, code * (span / top).float().double(), 0.0)
            rows.append(x.reshape(s["tokens"], h, d))
        return {"k": rows[0], "v": rows[1]}
    out = torch.zeros((s["tokens"], hq, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["tokens"], hq), dtype=torch.float64, device=DEV)
    flat, first = s["pool"].flatten(), 0
    for i in range(c["seqs"]):
        j = torch.arange(kv[i], device=DEV)
        block = s["table"][i].long()[j // c["page"]], j % c["page"] // 16
        pos = torch.arange(kv[i] - new[i], kv[i], device=DEV)[:, None]
        hidden = j > pos
        if c["window"]:
            hidden = hidden | ((j <= pos - c["window"]) & (j >= c["sinks"]))
        for head in range(h):
            base = ((block[0] * h + head) * (c["page"] // 16) + block[1]) * size
            k, v = stored(c, flat, base, j % 16, True), stored(c, flat, base, j % 16, False)
            for one in range(head * (hq // h), (head + 1) * (hq // h)):
                x = s["qkv"][first:first + new[i], one].double() @ k.T / math.sqrt(d)
                x = x.masked_fill_(hidden, -math.inf)
                lse[first:first + new[i], one] = torch.logsumexp(x, -1)
                out[first:first + new[i], one] = torch.softmax(x, -1) @ v
        first += new[i]
    if c["prior"]:
        l2 = s["prior_lse"].double()
        w = torch.sigmoid(lse - l2)[..., None]
        out = w * out + (1 - w) * s["prior"].double()
        lse = lse + torch.nn.functional.softplus(l2 - lse)
    return {"out": out, "lse": lse}
