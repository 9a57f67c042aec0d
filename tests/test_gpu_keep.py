"""Weights of keys, the choice by them and moving rows together on the GPU against oracle/pages.py: weights within their derived bounds, places and bytes of the
pages equal."""
import itertools

import numpy as np
import pytest
import torch

from oracle import pages as op
from test_gpu_pages import DEV, FORMATS, TORCH, Cache, bits_of, rows

pytestmark = pytest.mark.gpu


def weights_of(c, fill=3.0):
    cfg = c.pages.cfg
    return torch.full((cfg.n_pages, cfg.n_kv_heads, cfg.page_tokens), fill, device=DEV)


def of_seq(c, w, s, n):
    """[n, n_kv] of sequence s"""
    j = np.arange(n)
    return w.cpu().numpy()[c.table[s, j // c.spec.page_tokens], :, j % c.spec.page_tokens].astype(np.float64)


# ---- weights ---------------------------------------------------------------------------------------
def weigh(c, new_and_len, add=False, window=0, sinks=0, scale=None, weights=None, room=0, hidden=None, lse=None):
    spec, t = c.spec, sum(n for n, _ in new_and_len)
    scale = spec.head_dim ** -0.5 if scale is None else scale
    q = rows(c.rng, t + room, spec.n_heads, spec.head_dim, spec.dtype).to(DEV)
    if lse is None:
        lse = torch.from_numpy((c.rng.standard_normal((t + room, spec.n_heads)) + 4).astype(np.float32)).to(DEV)
    w = weights_of(c) if weights is None else weights
    before = w.clone()
    c.pages.weigh(c.layer, c.batch(new_and_len, room), q, scale, lse, w, add=add, window=window, sinks=sinks)
    torch.cuda.synchronize()
    at, touched = 0, torch.zeros_like(w, dtype=torch.bool)
    for s, (n, total) in enumerate(new_and_len):
        if n == 0:
            continue
        k = c.stored(c.k[s][:total])
        qs = op.to_f32(bits_of(q[at:at + n]), spec.dtype).astype(np.float64)
        e, far = op.weigh(qs, k, total, scale, lse[at:at + n].cpu().numpy().astype(np.float64), window, sinks, None if hidden is None else hidden.get(s))
        at += n
        j = np.arange(total)
        there = np.ones(total, bool) if hidden is None or s not in hidden else ~hidden[s][:total]
        j = j[there]
        page, place = torch.from_numpy(c.table[s, j // spec.page_tokens]).long(), torch.from_numpy(j % spec.page_tokens)
        got = w.cpu()[page, :, place].numpy().astype(np.float64)
        old = before.cpu()[page, :, place].numpy().astype(np.float64)
        e, far = e[there], far[there]
        if add:
            older = (j < total - n)[:, None]
            e = np.where(older, e + old, e)
            far = far + np.where(older, np.abs(e) * 2.0 ** -24, 0.0)
        same = (got == e) | (np.isnan(got) & np.isnan(e))
        with np.errstate(invalid="ignore"):
            bad = ~(same | (np.abs(got - e) <= far))
        assert not bad.any(), f"sequence {s} ({n} of {total}): {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[bad][0]} against {e[bad][0]}, bound {far[bad][0]}"
        touched[page.to(DEV), :, place.to(DEV)] = True
    assert torch.equal(w[~touched], before[~touched])
    return q, lse, w


@pytest.mark.parametrize("store,dtype,dim", FORMATS)
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (24, 1)])
def test_weights(store, dtype, dim, heads, kv_heads):
    """Single tokens, chunks and whole texts, set and added."""
    c = Cache(op.PagesSpec(kv_heads, heads, dim, 32, dtype, store), [1, 64, 90, 17, 300, 33], 1)
    w = weights_of(c)
    for batch in ([(1, 1), (64, 64), (10, 90), (17, 17), (9, 300), (2, 33)], [(1, 1), (1, 64), (1, 90), (1, 17), (1, 300), (1, 33)],
                  [(0, 1), (33, 47), (8, 65), (0, 17), (150, 300), (0, 0)]):
        for add in (False, True):
            weigh(c, batch, add, weights=w)
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("dtype,store", itertools.product(("fp16", "bf16"), ("16", "int4")))
@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 0), (40, 5), (500, 64), (64, 200)])
def test_weights_under_windows(dtype, store, window, sinks):
    c = Cache(op.PagesSpec(2, 4, 64, 16, dtype, store), [700, 90, 30], 2)
    for batch in ([(1, 700), (1, 90), (1, 30)], [(300, 700), (90, 90), (7, 30)]):
        weigh(c, batch, window=window, sinks=sinks)


@pytest.mark.parametrize("store", ("16", "int8"))
def test_weights_of_long_texts(store):
    c = Cache(op.PagesSpec(2, 8, 128, 64, "bf16", store), [3001, 40, 1200], 3)
    for batch in ([(1, 3001), (1, 40), (1, 1200)], [(32, 3001), (32, 40), (32, 1200)], [(1000, 3000), (40, 40), (1, 1200)]):
        weigh(c, batch, add=True)


@pytest.mark.parametrize("heads,kv_heads", [(3, 1), (10, 2), (40, 1), (64, 1), (70, 1), (128, 1), (384, 2)])
def test_weights_of_wide_groups(heads, kv_heads):
    """Groups that do not divide a step's rows, fill it, or take several; rows in chunks; windows."""
    c = Cache(op.PagesSpec(kv_heads, heads, 64, 16, "fp16", "int8"), [333, 30, 90], 22)
    lse = (c.rng.standard_normal((400, heads)) + 4).astype(np.float32)
    lse[5, heads // 2], lse[60] = float("-inf"), float("-inf")
    for batch in ([(1, 333), (1, 30), (1, 90)], [(200, 300), (9, 29), (90, 90)], [(33, 300), (0, 29), (1, 90)]):
        for window in (0, 50):
            t = sum(n for n, _ in batch)
            weigh(c, batch, window=window, sinks=3, lse=torch.from_numpy(lse[:t]).to(DEV))


def test_shares_of_attention():
    """With the attention's own log-sums the weights of a row sum to one: for each K/V head as many as rows."""
    c = Cache(op.PagesSpec(2, 8, 128, 16, "fp16", "16"), [500], 4)
    for n in (1, 30, 500):
        q, _, lse = c.attend([(n, 500)])
        w = weights_of(c)
        c.pages.weigh(0, c.batch([(n, 500)]), q, 128 ** -0.5, lse, w, add=False)
        sums = of_seq(c, w, 0, 500).sum(0)
        assert np.abs(sums / (4 * n) - 1).max() < 2.0 ** -12      # exp of differences of numbers below 2^6, errors of 2^-17 at the most


def test_rows_without_weight():
    """Rows whose log-sum says that they saw nothing; a K that is not finite is its own key's affair."""
    c = Cache(op.PagesSpec(1, 2, 64, 16, "fp16", "16"), [60], 5, history=False)
    c.k[0][7, 0, 3], c.k[0][20, 0, 0] = float("nan"), float("inf")
    c.write([(60, 60)])
    lse = torch.full((9, 2), 3.0, device=DEV)
    lse[2], lse[5, 1] = float("-inf"), float("-inf")
    weigh(c, [(9, 60)], lse=lse)
    weigh(c, [(9, 60)], lse=torch.full((9, 2), float("-inf"), device=DEV))
    lse[0, 0] = float("nan")
    weigh(c, [(9, 60)], lse=lse)
    lse[0, 0] = float("inf")
    weigh(c, [(9, 60)], lse=lse)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5])
def test_weights_by_scale(scale):
    c = Cache(op.PagesSpec(1, 4, 64, 16, "bf16", "int8"), [150, 30], 6)
    weigh(c, [(6, 150), (30, 30)], scale=scale, room=3, lse=torch.full((39, 4), 20.0, device=DEV))


@pytest.mark.parametrize("n", [1, 6, 20, 150])
def test_a_scale_of_zero_whatever_the_products(n):
    """All keys that a row sees have exp(-lse) of it, as the attention whose log-sum that is has it, though products of the queries and keys pass fp32."""
    c = Cache(op.PagesSpec(1, 4, 128, 16, "bf16", "16"), [200], 27, history=False)
    c.k[0][:] = c.k[0] * 2.0 ** 70
    c.write([(200, 200)])
    q = rows(c.rng, n, 4, 128, "bf16").to(DEV) * 2.0 ** 70
    q[n // 2, 1, 5] = float("nan")
    out, lse, w = torch.empty_like(q), torch.empty((n, 4), device=DEV), weights_of(c)
    c.pages.attend(0, c.batch([(n, 200)]), q, 0.0, out, lse)
    seen = np.arange(201 - n, 201)
    assert np.abs(lse.cpu().numpy() - np.log(seen)[:, None]).max() < 2.0 ** -18       # sums of ones and a logarithm below 8 in fp32
    c.pages.weigh(0, c.batch([(n, 200)]), q, 0.0, lse, w, add=False)
    e = np.array([4 * (1.0 / seen[seen > j]).sum() for j in range(200)])
    # lse and its product with log2 e a rounding each of numbers below 8, exp2, and sums of up to 4 n numbers
    assert np.abs(of_seq(c, w, 0, 200)[:, 0] / e - 1).max() < 2.0 ** -17 + (4 * n + 64) * 2.0 ** -24


def test_weights_of_pages_that_are_none():
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(1, 2, 64, 16, "bf16", "int4"), [200], 7)
    c.table[0, 3], c.table[0, 12] = 10 ** 6, -1
    hidden = np.zeros(200, bool)
    hidden[48:64] = hidden[192:] = True
    for n in (1, 50):
        weigh(c, [(n, 200)], hidden={0: hidden})
    assert c.pages.get_status() == binding.FAULT_PAGE


def test_wrong_batches_have_no_weights():
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(1, 4, 64, 16, "fp16", "16"), [100, 40], 8)
    q, lse, w = rows(c.rng, 8, 4, 64, "fp16").to(DEV), torch.zeros((8, 4), device=DEV), weights_of(c)
    keep = torch.full((2, 1, 3), 7, dtype=torch.int32, device=DEV)
    pool = c.pages.pool.clone()
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    table = torch.from_numpy(c.table).to(DEV)
    for start, length in (((0, 5, 8), (4, 2)), ((5, 0, 8), (100, 40))):
        batch = binding.PageBatch(ints(*start), ints(*length), table, 8, max_q=8, max_kv=100)
        c.pages.weigh(0, batch, q, 0.125, lse, w)
        c.pages.select(batch, w, 3, keep)
        c.pages.keep(0, batch, keep)
        c.pages.keep(0, batch, keep, to=table.clone(), weights=w)
        assert c.pages.get_status() == binding.FAULT_BATCH and (w == 3).all() and (keep == 7).all() and torch.equal(c.pages.pool, pool)


@pytest.mark.parametrize("n", [1, 9, 40, 150])
def test_sequences_without_new_tokens(n):
    """Their weights stay what they are, set or added, and their lists are empty; of a batch of such sequences alone nothing is written, lists neither."""
    c = Cache(op.PagesSpec(2, 8, 64, 16, "fp16", "16"), [60, 200, 17], 28)
    for add in (False, True):
        _, _, w = weigh(c, [(0, 60), (n, 200), (0, 17)], add)
        assert (of_seq(c, w, 0, 60) == 3).all() and (of_seq(c, w, 2, 17) == 3).all()
    before = c.pages.pool.clone()
    keep = select(c, [(0, 60), (n, 200), (0, 17)], w, 5)
    assert (keep[[0, 2]] == -1).all() and (keep[1] >= 0).any()
    keep.fill_(7)
    old = w.clone()
    empty = c.batch([(0, 60), (0, 200), (0, 17)])
    c.pages.weigh(0, empty, torch.empty((0, 8, 64), dtype=torch.float16, device=DEV), 0.125, torch.empty((0, 8), device=DEV), w, add=False)
    c.pages.select(empty, w, 5, keep)
    c.pages.keep(0, empty, keep)
    assert (keep == 7).all() and torch.equal(w, old) and torch.equal(before, c.pages.pool) and c.pages.get_status() == 0


@pytest.mark.parametrize("n", [1, 12, 40, 150])
def test_weights_of_a_batch_that_begins_later(n):
    """Rows before the batch's first are not its own."""
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(2, 8, 64, 16, "fp16", "16"), [300, 200], 23)
    q = rows(c.rng, 2 * n + 5, 8, 64, "fp16").to(DEV)
    lse, w, late = torch.full((2 * n + 5, 8), 3.0, device=DEV), weights_of(c), weights_of(c)
    lse[:5] = float("nan")
    c.pages.weigh(0, c.batch([(n, 300), (n, 200)]), q[5:], 0.125, lse[5:].contiguous(), w, add=False)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    batch = binding.PageBatch(ints(5, 5 + n, 5 + 2 * n), ints(300, 200), torch.from_numpy(c.table).to(DEV), 2 * n + 5, max_q=n, max_kv=300)
    c.pages.weigh(0, batch, q, 0.125, lse, late, add=False)
    assert torch.equal(w, late) and c.pages.get_status() == 0


def test_pools_past_32_bits():
    """Weights, choice and move in the last pages of a pool of 5 GB."""
    c = Cache(op.PagesSpec(8, 8, 128, 256, "bf16", "16"), [700], 24, extra_pages=5000, history=False)
    n_pages = c.pages.cfg.n_pages
    c.table[0, :3] = [n_pages - 1, n_pages - 3, n_pages - 2]
    c.write([(700, 700)])
    for n in (1, 40, 700):
        weigh(c, [(n, 700)])
    w = weights_of(c)
    w.copy_(torch.rand(w.shape, device=DEV))
    keep = select(c, [(700, 700)], w, 50, sinks=1, recent=9)
    old = of_seq(c, w, 0, 700)
    to = torch.tensor([[n_pages - 5]], dtype=torch.int32, device=DEV)
    kept = keep.cpu().numpy()[0]
    k, v = (torch.empty((50, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    after = c.b.PageBatch(torch.tensor([0, 50], dtype=torch.int32, device=DEV), torch.tensor([50], dtype=torch.int32, device=DEV), to, 50, max_kv=50)
    for place in (to, None):
        c.pages.keep(0, c.batch([(700, 700)]), keep, to=place, weights=w)
        if place is None:
            after = c.b.PageBatch(*after.tensors[:2], torch.from_numpy(c.table).to(DEV), 50, max_kv=50)
        c.pages.read(0, after, k, v)
        for h in range(8):
            assert torch.equal(k[:, h].cpu(), c.k[0][kept[h], h]) and torch.equal(v[:, h].cpu(), c.v[0][kept[h], h])
            page = n_pages - 5 if place is not None else n_pages - 1
            assert np.array_equal(w[page, h, :50].cpu().numpy().astype(np.float64), old[kept[h], h])
    assert c.pages.get_status() == 0


# ---- the choice ------------------------------------------------------------------------------------
def select(c, new_and_len, w, budget, sinks=0, recent=0):
    keep = torch.full((len(new_and_len), c.spec.n_kv_heads, budget), 7, dtype=torch.int32, device=DEV)
    c.pages.select(c.batch(new_and_len), w, budget, keep, sinks=sinks, recent=recent)
    got = keep.cpu().numpy()
    for s, (n, total) in enumerate(new_and_len):
        if total == 0:
            assert (got[s] == -1).all()
            continue
        x = of_seq(c, w, s, total)[total - n:]
        for h in range(c.spec.n_kv_heads):
            e = op.select(x[:, h], budget, sinks, recent)
            assert got[s, h].tolist() == e + [-1] * (budget - len(e)), (s, h, n, total)
    return keep


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (7, 2, 5), (40, 4, 16), (64, 0, 0), (300, 4, 64), (299, 0, 299), (10, 0, 0)])
@pytest.mark.parametrize("kind", ["spread", "same", "ties", "few", "odd"])
def test_choice(budget, sinks, recent, kind):
    c = Cache(op.PagesSpec(3, 3, 64, 16, "fp16", "int4"), [300, 1, 65, 64, 11, 0], 9)
    w = weights_of(c)
    r = torch.Generator(device=DEV).manual_seed(budget)
    x = torch.randn(w.shape, generator=r, device=DEV)
    w.copy_({"spread": torch.exp(3 * x), "same": torch.full_like(x, 0.25), "ties": torch.floor(2 * x) / 2, "few": torch.where(x > 2, x, 0.0),
             "odd": torch.where(x > 1.5, float("nan"), torch.where(x < -1.5, float("inf"), torch.where(x < -1, float("-inf"), torch.where(x < 0, -0.0, 0.0))))}[kind])
    for batch in ([(300, 300), (1, 1), (65, 65), (64, 64), (11, 11), (0, 0)], [(299, 300), (0, 1), (20, 64), (64, 64), (1, 10), (0, 0)]):
        select(c, batch, w, budget, sinks, recent)
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2049, 5000])
def test_choice_of_long_texts(n):
    """Against a sort."""
    c = Cache(op.PagesSpec(2, 2, 64, 64, "fp16", "int4"), [n], 10, history=False)
    w = weights_of(c)
    w.copy_(torch.floor(4 * torch.randn(w.shape, generator=torch.Generator(device=DEV).manual_seed(n), device=DEV)))
    against_a_sort(c, n, w, n // 3, 4, 100)


def against_a_sort(c, n, w, budget, sinks, recent):
    keep = torch.empty((1, c.spec.n_kv_heads, budget), dtype=torch.int32, device=DEV)
    c.pages.select(c.batch([(n, n)]), w, budget, keep, sinks=sinks, recent=recent)
    x, i = of_seq(c, w, 0, n), np.arange(n)
    always = (i < sinks) | (i >= n - recent)
    for h in range(c.spec.n_kv_heads):
        rank = np.lexsort((i, -x[:, h], ~always))
        assert np.array_equal(keep[0, h].cpu().numpy(), np.sort(rank[:budget]))


def test_choice_of_texts_longer_than_lds():
    """Keys that do not fit the part of LDS they are kept in."""
    n = 70001
    c = Cache(op.PagesSpec(1, 1, 64, 256, "fp16", "int4"), [n], 11, history=False)
    w = weights_of(c)
    w.copy_(torch.floor(100 * torch.randn(w.shape, generator=torch.Generator(device=DEV).manual_seed(n), device=DEV)))
    for budget in (1, 4096, 60000, 70000):
        against_a_sort(c, n, w, budget, 1 if budget > 1 else 0, budget // 8)


def test_choice_among_pages_that_are_none():
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(1, 1, 64, 16, "fp16", "16"), [100], 12)
    c.table[0, 2] = -1
    w = weights_of(c, float("-inf"))
    keep = torch.empty((1, 1, 84), dtype=torch.int32, device=DEV)
    c.pages.select(c.batch([(100, 100)]), w, 84, keep)
    assert keep.flatten().tolist() == [i for i in range(100) if i < 32 or i >= 48] and c.pages.get_status() == binding.FAULT_PAGE


# ---- moving rows -----------------------------------------------------------------------------------
def moved(c, pool, new_and_len, keep, to=None, weights=None):
    """The pool (and weights) after the move, byte by byte."""
    spec, cfg = c.spec, c.pages.cfg
    blocks, heads = spec.page_tokens // 16, spec.n_kv_heads
    old = pool[:cfg.n_layers * cfg.n_pages * heads * blocks * spec.block_bytes].reshape(cfg.n_layers, cfg.n_pages, heads, blocks, spec.block_bytes)
    new = old.copy()
    w_old = None if weights is None else weights.copy()
    at = [op.bytes_of_token(spec, t) for t in range(16)]
    for s, (n, total) in enumerate(new_and_len):
        base = total - n
        for h in range(heads):
            line = keep[s, h if keep.shape[1] > 1 else 0]
            for i, k in enumerate(line[:n]):
                if k < 0 or k >= n or (to is None and k < i):
                    continue
                src, dst = base + k, base + i
                table = c.table if to is None else to
                if dst // spec.page_tokens >= table.shape[1]:
                    continue
                p, r = c.table[s, src // spec.page_tokens], table[s, dst // spec.page_tokens]
                if not 0 <= r < cfg.n_pages:
                    continue
                a, b = src % spec.page_tokens, dst % spec.page_tokens
                new[c.layer, r, h, b // 16, at[b % 16]] = old[c.layer, p, h, a // 16, at[a % 16]] if 0 <= p < cfg.n_pages else 0
                if weights is not None:
                    weights[r, h, b] = w_old[p, h, a] if 0 <= p < cfg.n_pages else 0
    return new


def keep_and_check(c, new_and_len, keep, to=None, weights=None):
    before = c.pages.pool.cpu().numpy().copy()
    w = None if weights is None else weights.cpu().numpy().copy()
    c.pages.keep(c.layer, c.batch(new_and_len), torch.from_numpy(keep).to(DEV), to=None if to is None else torch.from_numpy(to).to(DEV), weights=weights)
    torch.cuda.synchronize()
    e = moved(c, before, new_and_len, keep, to, w)
    got = c.pages.pool.cpu().numpy()[:e.size].reshape(e.shape)
    bad = np.argwhere(got != e)
    assert bad.size == 0, f"{len(bad)} bytes differ, first {bad[0]}: {got[tuple(bad[0])]} against {e[tuple(bad[0])]}"
    if weights is not None:
        assert np.array_equal(weights.cpu().numpy(), w)


def lists(rng, new_and_len, heads, width, share):
    """Rising places, of each head's own or of all"""
    keep = np.full((len(new_and_len), heads, width), -1, np.int32)
    for s, (n, _) in enumerate(new_and_len):
        m = min(width, max(1, int(n * share))) if n else 0
        for h in range(heads):
            keep[s, h, :m] = np.sort(rng.permutation(n)[:m])
    return keep


def elsewhere(c, new_and_len, width):
    """A page table of the pages that nothing has."""
    used = {int(x) for s, (_, t) in enumerate(new_and_len) for x in c.table[s, :-(-t // c.spec.page_tokens)]}
    free = c.rng.permutation([x for x in range(c.pages.cfg.n_pages) if x not in used]).astype(np.int32)
    to, at = np.full((len(new_and_len), width), -9, np.int32), 0
    for s, (n, t) in enumerate(new_and_len):
        for i in range((t - n) // c.spec.page_tokens, min(width, -(-t // c.spec.page_tokens))):
            to[s, i] = free[at]
            at += 1
    return to


@pytest.mark.parametrize("store,dtype,dim", FORMATS)
@pytest.mark.parametrize("heads_of_list", ["own", "all"])
def test_moving(store, dtype, dim, heads_of_list):
    """Whole texts and drafts, in place and elsewhere, with and without weights; every other byte of the pool stays."""
    lengths = [1, 64, 90, 17, 700, 33]
    batches = ([(1, 1), (64, 64), (90, 90), (17, 17), (700, 700), (33, 33)], [(1, 1), (10, 64), (5, 90), (0, 17), (333, 650), (2, 31)])
    for batch in batches:
        for share, place in itertools.product((0.3, 0.95), ("here", "elsewhere")):
            c = Cache(op.PagesSpec(2, 2, dim, 32, dtype, store), lengths, 13, layers=2, layer=1, extra_pages=40)
            w = weights_of(c)
            w.copy_(torch.rand(w.shape, device=DEV))
            keep = lists(c.rng, batch, 2 if heads_of_list == "own" else 1, 400, share)
            keep_and_check(c, batch, keep, None if place == "here" else elsewhere(c, batch, 22), None if share < 0.5 else w)
            assert c.pages.get_status() == 0


@pytest.mark.parametrize("store", ("16", "int8", "int4"))
def test_entries_that_move_nothing(store):
    """Entries out of range or below their place, tables that are too narrow, pages that are none."""
    from paper_2602_14236_amd import binding
    batch = [(100, 100), (20, 50)]
    for place in ("here", "elsewhere"):
        c = Cache(op.PagesSpec(2, 2, 64, 16, "bf16", store), [100, 50], 14, extra_pages=20)
        keep = np.full((2, 1, 70), -1, np.int32)
        keep[0, 0, :30] = np.arange(30) * 3
        keep[0, 0, 3], keep[0, 0, 9], keep[0, 0, 20] = 100, 2, 2 ** 31 - 1
        keep[1, 0, :12] = [4, -5, 3, 7, 5, 30, 6, 9, 8, 19, 20, 19]
        keep[1, 0, 20:] = 19
        to = None if place == "here" else elsewhere(c, batch, 7)
        keep_and_check(c, batch, keep, to)
        assert c.pages.get_status() == binding.FAULT_BATCH
    for place in ("here", "elsewhere"):
        c = Cache(op.PagesSpec(2, 2, 64, 16, "bf16", store), [100, 50], 15, extra_pages=20)
        to = None if place == "here" else elsewhere(c, batch, 7)
        c.table[0, 3] = -4
        if to is not None:
            to[1, 2] = 10 ** 7
            to[0, 1] = -1
        w = weights_of(c)
        w.copy_(torch.rand(w.shape, device=DEV))
        keep_and_check(c, batch, lists(c.rng, batch, 2, 60, 0.6), to, w)
        assert c.pages.get_status() == binding.FAULT_PAGE
    c = Cache(op.PagesSpec(2, 2, 64, 16, "bf16", store), [100, 50], 16, extra_pages=20)
    keep_and_check(c, batch, lists(c.rng, batch, 1, 60, 0.6), elsewhere(c, batch, 3))
    assert c.pages.get_status() == binding.FAULT_BATCH


@pytest.mark.parametrize("width", [0, 1])
def test_tables_too_narrow_for_all_of_a_list(width):
    """Nothing moves, in the batch's pages either."""
    from paper_2602_14236_amd import binding
    batch = [(30, 60), (20, 50)]
    c = Cache(op.PagesSpec(2, 2, 64, 16, "fp16", "16"), [60, 50], 26, extra_pages=20)
    w = weights_of(c)
    keep = lists(c.rng, batch, 2, 20, 0.5)
    before = c.pages.pool.clone()
    c.pages.keep(0, c.batch(batch), torch.from_numpy(keep).to(DEV), to=torch.zeros((2, width), dtype=torch.int32, device=DEV), weights=w)
    assert torch.equal(before, c.pages.pool) and (w == 3).all() and c.pages.get_status() == binding.FAULT_BATCH


def test_any_order_elsewhere():
    """Elsewhere a list may be in any order, a row twice."""
    batch = [(100, 100), (40, 50)]
    c = Cache(op.PagesSpec(2, 2, 64, 16, "fp16", "int8"), [100, 50], 17, extra_pages=20)
    keep = c.rng.integers(0, 40, (2, 2, 90)).astype(np.int32)
    keep_and_check(c, batch, keep, elsewhere(c, batch, 7))
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("store", ("16", "int4"))
def test_long_texts_in_place(store):
    """Many chunks, one after the other in the same pages."""
    n = 6001
    for share in (0.1, 0.7, 1.0):
        c = Cache(op.PagesSpec(1, 1, 64, 64, "fp16", store), [n], 18)
        keep_and_check(c, [(n, n)], lists(c.rng, [(n, n)], 1, n, share))


# ---- together --------------------------------------------------------------------------------------
@pytest.mark.parametrize("store,dtype", itertools.product(("16", "int8", "int4"), ("fp16", "bf16")))
def test_a_conversation(store, dtype):
    """A prompt, a draft of which a path is accepted, then the text cut down by what was attended to, and a next token over what stayed: its attention is that over
    the rows that stayed."""
    from paper_2602_14236_amd import binding
    spec = op.PagesSpec(2, 8, 64, 16, dtype, store)
    c = Cache(spec, [200, 120], 19, history=False)
    r = binding.Rotary(10000.0 ** (-torch.arange(32, dtype=torch.float64, device=DEV) / 32), [12, 10, 10])
    w = weights_of(c, 0.0)
    text = [160, 90]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)

    def turned(x, pos):
        """keys at their positions"""
        y = x.to(DEV)
        c.pages.rotate(r, pos, None, y)
        return y.cpu()

    for s in (0, 1):
        i = torch.arange(len(c.k[s]), dtype=torch.int32, device=DEV)
        c.k[s] = turned(c.k[s], torch.stack([i, i // 5, i % 5]))
    # the prompts
    batch = [(n, n) for n in text]
    c.write(batch)
    q, out, lse = c.attend(batch)
    c.pages.weigh(0, c.batch(batch), q, 64 ** -0.5, lse, w)
    # a draft of six tokens each; the path 1, 3, 4 is accepted
    parents = [-1, -1, 0, 1, 3, 2]
    draft = [(6, n + 6) for n in text]
    c.write(draft)
    from test_gpu_drafts import attend as attend_tree
    attend_tree(c, draft, binding.draft_masks(parents) * 2)
    path = np.array([[[1, 3, 4]]] * 2, np.int32)
    keep_and_check(c, draft, path)
    for s, n in enumerate(text):
        for rows_ in (c.k[s], c.v[s]):
            rows_[n:n + 3] = rows_[[n + 1, n + 3, n + 4]].clone()
    text = [n + 3 for n in text]
    batch = [(3, n) for n in text]
    q, out, lse = c.attend(batch)
    c.pages.weigh(0, c.batch(batch), q, 64 ** -0.5, lse, w)
    # cut down
    whole = [(n, n) for n in text]
    keep = select(c, whole, w, 70, sinks=2, recent=20)
    kept = keep.cpu().numpy()
    old_w = [of_seq(c, w, s, n) for s, n in enumerate(text)]
    keep_and_check(c, whole, kept, None, w)
    for s in (0, 1):
        c.k[s][:70] = torch.stack([c.k[s][kept[s, h], h] for h in (0, 1)], 1)
        c.v[s][:70] = torch.stack([c.v[s][kept[s, h], h] for h in (0, 1)], 1)
        new_w = of_seq(c, w, s, 70)
        for h in (0, 1):
            assert np.array_equal(new_w[:, h], old_w[s][kept[s, h], h])
    # the next tokens, at the positions that follow
    for s, n in enumerate(text):
        c.k[s][70:72] = turned(c.k[s][70:72], ints([[n, n + 1]] * 3))
    batch = [(2, 72), (2, 72)]
    c.write(batch)
    q, out, lse = c.attend(batch)
    c.pages.weigh(0, c.batch(batch), q, 64 ** -0.5, lse, w)
    assert c.pages.get_status() == 0


def test_replayed_and_on_a_stream():
    """Weights, choice and move captured in one graph, replayed with other lengths; every replay against the calls made one by one on a side stream."""
    c = Cache(op.PagesSpec(2, 8, 64, 16, "bf16", "int8"), [300, 200], 20, extra_pages=20)
    start, length = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    table = torch.from_numpy(c.table).to(DEV)
    to = torch.from_numpy(elsewhere(c, [(300, 300), (200, 200)], 4)).to(DEV)
    q = rows(c.rng, 500, 8, 64, "bf16").to(DEV)
    lse, w = torch.full((500, 8), 4.0, device=DEV), weights_of(c, 0.0)
    keep = torch.zeros((2, 2, 50), dtype=torch.int32, device=DEV)
    batch = c.b.PageBatch(start, length, table, 500, max_q=300, max_kv=300)

    def calls(stream=None):
        c.pages.weigh(0, batch, q, 0.125, lse, w, add=False, stream=stream)
        c.pages.select(batch, w, 50, keep, sinks=2, recent=8, stream=stream)
        c.pages.keep(0, batch, keep, to=to, weights=w, stream=stream)

    calls()
    torch.cuda.synchronize()
    pool0 = c.pages.pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for lens in ((300, 200), (60, 7), (299, 1)):
        start.copy_(torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32))
        length.copy_(torch.tensor(lens, dtype=torch.int32))
        results = []
        for how in ("graph", "stream", "graph"):
            c.pages.pool.copy_(pool0)
            w.zero_()
            keep.fill_(9)
            torch.cuda.synchronize()
            if how == "graph":
                graph.replay()
            else:
                side = torch.cuda.Stream()
                calls(side)
            torch.cuda.synchronize()
            results.append((c.pages.pool.clone(), w.clone(), keep.clone()))
        for got in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], got))
    assert c.pages.get_status() == 0


def test_refusals():
    """What the library refuses, by code; nothing is launched."""
    from paper_2602_14236_amd import binding as b
    c = Cache(op.PagesSpec(2, 4, 64, 16, "fp16", "16"), [40], 21, extra_pages=3)
    p, lib, h = c.pages, c.pages.lib, c.pages.handle
    q = rows(c.rng, 8, 4, 64, "fp16").to(DEV)
    lse, w, keep = torch.zeros((8, 4), device=DEV), weights_of(c), torch.full((1, 2, 5), 7, dtype=torch.int32, device=DEV)
    before = p.pool.clone()
    batch = c.batch([(8, 40)])
    good = b.sali_rows(q.data_ptr(), 256, 64)

    def changed(**kw):
        v = {n: getattr(batch.c, n) for n, _ in b.sali_page_batch._fields_}
        return b.sali_page_batch(*{**v, **kw}.values())

    weigh = lambda bt=batch.c, rows_=good, scale=0.1, window=0, sinks=0, l=lse.data_ptr(), to=w.data_ptr(), layer=0: \
        lib.sali_pages_weigh(h, layer, bt, rows_, scale, window, sinks, l, 0, to, None)
    assert weigh(None) == -1 and weigh(rows_=None) == -1 and weigh(l=None) == -1 and weigh(to=None) == -1
    assert weigh(layer=1) == -2 and weigh(window=-1) == -2 and weigh(sinks=-1) == -2 and weigh(changed(max_kv=-1)) == -2
    assert weigh(scale=float("nan")) == -4 and weigh(scale=float("inf")) == -4
    assert weigh(l=lse.data_ptr() + 2) == -3 and weigh(to=w.data_ptr() + 1) == -3 and weigh(rows_=b.sali_rows(q.data_ptr() + 2, 256, 64)) == -3
    select = lambda bt=batch.c, from_=w.data_ptr(), budget=5, sinks=0, recent=0, to=keep.data_ptr(): lib.sali_pages_select(h, bt, from_, budget, sinks, recent, to, None)
    assert select(None) == -1 and select(from_=None) == -1 and select(to=None) == -1
    assert select(budget=0) == -2 and select(sinks=-1) == -2 and select(recent=-1) == -2 and select(sinks=3, recent=3) == -2 and select(sinks=2 ** 31 - 1, recent=2 ** 31 - 1) == -2
    assert select(from_=w.data_ptr() + 2) == -3 and select(to=keep.data_ptr() + 2) == -3
    move = lambda bt=batch.c, list_=keep.data_ptr(), heads=2, width=5, to=None, to_width=0, weights=None, layer=0: \
        lib.sali_pages_keep(h, layer, bt, list_, heads, width, to, to_width, weights, None)
    assert move(None) == -1 and move(list_=None) == -1
    assert move(heads=0) == -2 and move(heads=3) == -2 and move(width=-1) == -2 and move(to=keep.data_ptr(), to_width=-1) == -2 and move(layer=-1) == -2
    assert move(list_=keep.data_ptr() + 1) == -3 and move(to=keep.data_ptr() + 2, to_width=1) == -3 and move(weights=w.data_ptr() + 2) == -3
    # nothing to do
    for bt in (changed(n_seqs=0), changed(n_tokens=0), changed(max_q=0), changed(max_kv=0)):
        assert weigh(bt) == 0 and select(bt) == 0 and move(bt) == 0
    assert move(width=0, list_=None) == 0
    torch.cuda.synchronize()
    assert p.get_status() == 0 and (w == 3).all() and (keep == 7).all() and torch.equal(before, p.pool)


def test_calls_of_more_blocks_than_a_launch_takes():
    """By the batch's sizes, whatever its arrays hold"""
    from paper_2602_14236_amd import binding as b
    c = Cache(op.PagesSpec(2, 4, 64, 16, "fp16", "16"), [40], 21, extra_pages=3)
    q = rows(c.rng, 8, 4, 64, "fp16").to(DEV)
    lse, w, batch = torch.zeros((8, 4), device=DEV), weights_of(c), c.batch([(8, 40)])
    long = b.sali_page_batch(*{**{n: getattr(batch.c, n) for n, _ in b.sali_page_batch._fields_}, "max_kv": 128 * 2 ** 22}.values())
    assert c.pages.lib.sali_pages_weigh(c.pages.handle, 0, long, b.sali_rows(q.data_ptr(), 256, 64), 0.1, 0, 0, lse.data_ptr(), 0, w.data_ptr(), None) == -2
    torch.cuda.synchronize()
    assert (w == 3).all() and c.pages.get_status() == 0


@pytest.mark.parametrize("n", [1, 30, 200])
def test_weights_at_any_address_of_a_float(n):
    c = Cache(op.PagesSpec(2, 8, 64, 32, "bf16", "16"), [430], 25)
    q = rows(c.rng, n, 8, 64, "bf16").to(DEV)
    size = weights_of(c).numel()
    lists, all_weights = [], []
    for off in range(4):
        base = torch.full((size + 4,), 3.0, device=DEV)
        w = base[off:off + size].view(weights_of(c).shape)
        batch = c.batch([(n, 430)])
        lse = torch.zeros((n, 8), device=DEV)
        c.pages.attend(0, batch, q, 0.125, torch.empty_like(q), lse)
        c.pages.weigh(0, batch, q, 0.125, lse, w, add=False)
        lists.append(select(c, [(430, 430)], w, 40, sinks=1, recent=3))
        all_weights.append(w.clone())
        assert (base[:off] == 3).all() and (base[off + size:] == 3).all()
    assert all(torch.equal(all_weights[0], x) for x in all_weights) and all(torch.equal(lists[0], x) for x in lists)
