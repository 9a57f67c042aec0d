"""Attention of drafted tokens over the pages on the GPU against oracle/pages.py (float64), within the bounds that oracle.pages.bounds derives."""
import itertools

import numpy as np
import pytest
import torch

from oracle import pages as op
from test_gpu_pages import DEV, FORMATS, TORCH, Cache, bits_of, rows

pytestmark = pytest.mark.gpu


def signed(m):
    return m - (1 << 64) if m >> 63 else m


def trees(rng, new_and_len):
    """A mask for every row: each token follows the text or one before it."""
    from paper_2602_14236_amd import binding
    masks = []
    for n, _ in new_and_len:
        masks += binding.draft_masks([int(rng.integers(-1, i)) for i in range(n)])
    return masks


def attend(c, new_and_len, masks, scale=None, prior=False, check=True, room=0, hidden=None, q=None):
    """attend_tree of a Cache, checked; its results"""
    spec, t = c.spec, sum(n for n, _ in new_and_len)
    q = rows(c.rng, t + room, spec.n_heads, spec.head_dim, spec.dtype).to(DEV) if q is None else q
    out = torch.full((t + room, spec.n_heads, spec.head_dim), 7.0, dtype=TORCH[spec.dtype], device=DEV)
    lse = torch.full((t + room, spec.n_heads), 7.0, device=DEV)
    scale = spec.head_dim ** -0.5 if scale is None else scale
    seen = torch.tensor(list(masks) + [-1] * room, dtype=torch.int64, device=DEV)
    pr = pl = None
    if prior:
        pr = torch.from_numpy(c.rng.standard_normal((t + room, spec.n_heads, spec.head_dim)).astype(np.float32)).to(DEV)
        pl = torch.from_numpy(c.rng.standard_normal((t + room, spec.n_heads)).astype(np.float32) + 3).to(DEV)
    c.pages.attend_tree(c.layer, c.batch(new_and_len, room), seen, q, scale, out, lse, prior=pr, prior_lse=pl)
    torch.cuda.synchronize()
    if check:
        verify(c, new_and_len, masks, q, out, lse, scale, pr, pl, hidden)
    return q, out, lse


def verify(c, new_and_len, masks, q, out, lse, scale, prior=None, prior_lse=None, hidden=None):
    spec, at = c.spec, 0
    out, lse = op.to_f32(bits_of(out), spec.dtype).astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for s, (n, t) in enumerate(new_and_len):
        if n == 0:
            continue
        k, v = c.stored(c.k[s][:t]), c.stored(c.v[s][:t])
        qs = op.to_f32(bits_of(q[at:at + n]), spec.dtype).astype(np.float64)
        pr = None if prior is None else prior[at:at + n].cpu().numpy().astype(np.float64)
        pl = None if prior_lse is None else prior_lse[at:at + n].cpu().numpy().astype(np.float64)
        seen = op.drafted([int(m) for m in masks[at:at + n]], t)
        e_out, e_lse, mass, reach = op.attend(qs, k, v, t, scale, 0, 0, pr, pl, None if hidden is None else hidden.get(s), seen)
        d_out, d_lse = op.bounds(spec, e_out, e_lse, mass, reach, t, np.abs(v[np.isfinite(v)]).max(initial=0.0))
        for got, exp, far, what in ((out[at:at + n], e_out, d_out, "out"), (lse[at:at + n], e_lse, d_lse, "lse")):
            same = (got == exp) | (np.isnan(got) & np.isnan(exp))
            with np.errstate(invalid="ignore"):
                bad = ~(same | (np.abs(got - exp) <= far))
            assert not bad.any(), f"{what} of sequence {s} ({n} of {t}): {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: " \
                                  f"{got[bad][0]} against {exp[bad][0]}, bound {np.broadcast_to(far, got.shape)[bad][0]}"
        at += n


@pytest.mark.parametrize("store,dtype,dim", FORMATS)
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (24, 1)])
def test_drafts(store, dtype, dim, heads, kv_heads):
    """One token to 64, with and without a history, drafts that cross blocks, tiles and pages."""
    c = Cache(op.PagesSpec(kv_heads, heads, dim, 32, dtype, store), [1, 64, 90, 17, 300, 33, 128], 1)
    for batch in ([(1, 1), (64, 64), (10, 90), (17, 17), (9, 300), (2, 33), (64, 128)], [(1, 1), (1, 60), (3, 80), (1, 17), (4, 299), (2, 31), (4, 128)],
                  [(0, 1), (33, 47), (8, 65), (0, 17), (7, 300), (0, 0), (16, 97)]):
        attend(c, batch, trees(c.rng, batch))
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("store,dtype", itertools.product(("16", "int8", "int4"), ("fp16", "bf16")))
@pytest.mark.parametrize("n", [4, 8, 13, 16, 40, 64])
def test_long_histories(store, dtype, n):
    """Stretches and shares with their merges, one text alone and among short ones."""
    c = Cache(op.PagesSpec(2, 8, 128, 64, dtype, store), [5000, 70, 2500, 64], n)
    for batch in ([(n, 5000), (1, 70), (n // 2, 2500), (n, 64)], [(n, 4990), (0, 0), (0, 0), (0, 0)]):
        attend(c, batch, trees(c.rng, batch), prior=n % 8 == 0)


@pytest.mark.parametrize("store,dtype,dim", FORMATS)
@pytest.mark.parametrize("n,group", [(9, 4), (11, 5), (16, 4), (33, 2), (25, 8), (64, 4), (64, 6)])
def test_row_sets(store, dtype, dim, n, group):
    """33 to 256 rows, in every number of sets of 32, and more; alone, among others of fewer rows, in one block and in stretches."""
    c = Cache(op.PagesSpec(2, 2 * group, dim, 16, dtype, store), [700, 150, n, 66], n * group)
    for batch in ([(n, 700), (max(1, n // 3), 150), (n, n), (2, 66)], [(0, 0), (n, 150), (0, 0), (n, 66)]):
        attend(c, batch, trees(c.rng, batch), prior=group == 4)
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("group", [2, 12])
def test_infinities_of_small_weight(group):
    """An infinity or NaN in V far below the strongest key, where its weight is rounded to zero: it reaches every row that sees it, and only values of its own."""
    n = 20
    c = Cache(op.PagesSpec(1, group, 64, 16, "fp16", "16"), [300], 9, history=False)
    c.k[0][7, 0] *= 20
    c.v[0][100, 0, 5], c.v[0][200, 0, 6], c.v[0][30, 0, 60] = float("inf"), float("-inf"), float("nan")
    c.write([(300, 300)])
    attend(c, [(n, 300)], trees(c.rng, [(n, 300)]), scale=1.0)


@pytest.mark.parametrize("dtype", ("fp16", "bf16"))
@pytest.mark.parametrize("n,total", [(6, 6), (6, 100), (64, 64), (64, 200), (20, 50)])
def test_masks(dtype, n, total):
    """Masks that no tree has: nothing of the draft, all of it, every second token, tokens behind the row's own, bits past the draft; rows that see nothing at all."""
    c = Cache(op.PagesSpec(1, 4, 64, 16, dtype, "16"), [total], n)
    every = (1 << 64) - 1
    for masks in ([0] * n, [signed(every)] * n, [signed(0xAAAAAAAAAAAAAAAA)] * n, [signed(every ^ (1 << i)) for i in range(n)],
                  [signed(every << n & every) if n < 64 else 0 for _ in range(n)], [signed(1 << (n - 1 - i)) for i in range(n)]):
        _, out, lse = attend(c, [(n, total)], masks)
        assert c.pages.get_status() == 0


@pytest.mark.parametrize("n", [6, 40])
def test_rows_that_see_nothing(n):
    c = Cache(op.PagesSpec(1, 4, 64, 16, "fp16", "16"), [n], n)
    masks = [0 if i % 3 == 0 else 1 << i for i in range(n)]
    _, out, lse = attend(c, [(n, n)], masks)
    assert (out[::3] == 0).all() and torch.isneginf(lse[::3]).all()
    attend(c, [(n, n)], masks, prior=True)
    attend(c, [(n, n)], [0] * n)


@pytest.mark.parametrize("n", [3, 8, 30])
def test_a_chain_is_a_causal_text(n):
    """The mask of tokens that follow one another: the same as attend, to the bounds of both."""
    c = Cache(op.PagesSpec(2, 8, 128, 16, "bf16", "int8"), [400, 35], n)
    batch = [(n, 400), (n, 35)]
    masks = [signed((1 << (i + 1)) - 1) for i in range(n)] * 2
    q, out, lse = attend(c, batch, masks)
    c.check(batch, q, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("n,heads", [(5, 2), (12, 4), (40, 4)])
def test_keys_out_of_sight_are_not_finite(n, heads):
    """Infinities and NaN in K and V of drafted tokens reach those that see them, and nobody else."""
    c = Cache(op.PagesSpec(1, heads, 64, 16, "fp16", "16"), [90], 3, history=False)
    c.v[0][88, 0, 5], c.v[0][87, 0, 6], c.v[0][86, 0, 7], c.k[0][89, 0, 1] = float("inf"), float("-inf"), float("nan"), float("nan")
    c.write([(90, 90)])
    masks = [signed(0)] * n
    q, out, lse = attend(c, [(n, 90)], masks)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    masks = [signed(1 << i) for i in range(n)]
    masks[0] |= 1 << (n - 2)
    masks[1] |= 1 << (n - 3)
    masks[n - 1] = 0
    attend(c, [(n, 90)], masks, q=q)


def test_rows_past_the_batch_and_strides():
    c = Cache(op.PagesSpec(2, 8, 64, 16, "fp16", "16"), [100, 40], 4)
    batch = [(5, 100), (3, 40)]
    q, out, lse = attend(c, batch, trees(c.rng, batch), room=4)
    assert (out[8:] == 7).all() and (lse[8:] == 7).all()
    wide = torch.full((8, 12, 64), 7.0, dtype=torch.float16, device=DEV)
    masks = trees(c.rng, batch)
    qkv = rows(c.rng, 8, 12, 64, "fp16").to(DEV)
    lse = torch.empty((8, 8), device=DEV)
    c.pages.attend_tree(0, c.batch(batch), torch.tensor(masks, device=DEV), qkv[:, :8], 0.125, wide[:, 2:10], lse)
    verify(c, batch, masks, qkv[:, :8], wide[:, 2:10], lse, 0.125)
    assert (wide[:, :2] == 7).all() and (wide[:, 10:] == 7).all()


@pytest.mark.parametrize("n", [3, 9, 50])
def test_a_batch_that_begins_later(n):
    """Rows before the batch's first keep what they hold."""
    c = Cache(op.PagesSpec(2, 8, 64, 16, "bf16", "int8"), [300, 100], 10)
    batch, t = [(n, 300), (n, 100)], 2 * n + 6
    masks = trees(c.rng, batch)
    q = rows(c.rng, t, 8, 64, "bf16").to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((t, 8), 7.0, device=DEV)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    late = c.b.PageBatch(ints(6, 6 + n, 6 + 2 * n), ints(300, 100), torch.from_numpy(c.table).to(DEV), t, max_q=n, max_kv=300)
    c.pages.attend_tree(0, late, torch.tensor([0] * 6 + masks, device=DEV), q, 0.125, out, lse)
    verify(c, batch, masks, q[6:], out[6:], lse[6:], 0.125)
    assert (out[:6] == 7).all() and (lse[:6] == 7).all() and c.pages.get_status() == 0


def test_pools_past_32_bits():
    c = Cache(op.PagesSpec(8, 32, 128, 256, "bf16", "16"), [700], 11, extra_pages=5000, history=False)
    c.table[0, :3] = [c.pages.cfg.n_pages - 1, 5, c.pages.cfg.n_pages - 2]
    c.write([(700, 700)])
    for n in (5, 40):
        attend(c, [(n, 700)], trees(c.rng, [(n, 700)]))
    assert c.pages.get_status() == 0


@pytest.mark.parametrize("n", [4, 40])
def test_pages_that_are_none(n):
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(1, 2, 64, 16, "bf16", "int4"), [200], 5)
    table = c.table.copy()
    table[0, 3], table[0, 12] = 10 ** 6, -1
    hidden = np.zeros(200, bool)
    hidden[48:64] = hidden[192:208] = True
    batch, masks = [(n, 200)], trees(c.rng, [(n, 200)])
    c.table = table
    attend(c, batch, masks, hidden={0: hidden})
    assert c.pages.get_status() == binding.FAULT_PAGE


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(scale):
    c = Cache(op.PagesSpec(1, 4, 64, 16, "fp16", "16"), [150, 30], 6)
    for batch in ([(6, 150), (4, 30)], [(40, 150), (4, 30)]):
        attend(c, batch, trees(c.rng, batch), scale=scale)


def test_wrong_batches_are_left_out():
    from paper_2602_14236_amd import binding
    c = Cache(op.PagesSpec(1, 4, 64, 16, "fp16", "16"), [100, 40], 7)
    q = rows(c.rng, 8, 4, 64, "fp16").to(DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((8, 4), 7.0, device=DEV)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    table = torch.from_numpy(c.table).to(DEV)
    seen = torch.full((8,), -1, dtype=torch.int64, device=DEV)
    for start, length in (((0, 5, 8), (4, 2)), ((5, 0, 8), (100, 40))):
        c.pages.attend_tree(0, binding.PageBatch(ints(*start), ints(*length), table, 8, max_q=8, max_kv=100), seen, q, 0.125, out, lse)
        assert c.pages.get_status() == binding.FAULT_BATCH and (out == 7).all() and (lse == 7).all()
    with pytest.raises(binding.SaliError) as e:
        c.pages.attend_tree(0, binding.PageBatch(ints(0, 5, 8), ints(100, 40), table, 8, max_q=65, max_kv=100), seen, q, 0.125, out, lse)
    assert e.value.code == -2
    with pytest.raises(ValueError):
        c.pages.attend_tree(0, c.batch([(5, 100), (3, 40)]), seen[:7], q, 0.125, out, lse)


def test_replayed():
    """Captured once, replayed with other lengths, masks and queries."""
    c = Cache(op.PagesSpec(2, 8, 128, 32, "bf16", "16"), [700, 300], 8)
    for most in (4, 16):
        start, length = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
        seen = torch.zeros(2 * most, dtype=torch.int64, device=DEV)
        q = torch.zeros((2 * most, 8, 128), dtype=torch.bfloat16, device=DEV)
        out, lse = torch.zeros_like(q), torch.zeros((2 * most, 8), device=DEV)
        batch = c.b.PageBatch(start, length, torch.from_numpy(c.table).to(DEV), 2 * most, max_q=most, max_kv=700)
        c.pages.attend_tree(0, batch, seen, q, 128 ** -0.5, out, lse)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.pages.attend_tree(0, batch, seen, q, 128 ** -0.5, out, lse)
        for lens in ([(most, 700), (most, 300)], [(1, 3), (most, 290)], [(most, most), (most // 2, 100)]):
            t = sum(n for n, _ in lens)
            masks = trees(c.rng, lens)
            seen[:t] = torch.tensor(masks, device=DEV)
            start.copy_(torch.tensor([0, lens[0][0], t], dtype=torch.int32))
            length.copy_(torch.tensor([n for _, n in lens], dtype=torch.int32))
            q.copy_(rows(c.rng, 2 * most, 8, 128, "bf16"))
            graph.replay()
            torch.cuda.synchronize()
            verify(c, lens, masks, q, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("store,dtype,dim", FORMATS)
@pytest.mark.parametrize("n,total,group", [(5, 5, 4), (40, 40, 4), (64, 64, 2), (30, 41, 8), (40, 500, 4)])
def test_only_the_output_is_rounded(store, dtype, dim, n, total, group):
    """Weights are two 16-bit numbers each, whichever kernel a draft takes: in op.bounds the weights' own term is then half a step of half a step (what the first number
    leaves is at most half a step of the weight, and the second one rounds that; fp16's smallest step counts as there).  Rows that see three drafted tokens, whose values
    cancel: a weight rounded once would be off by some hundred times the rest of the bound."""
    c = Cache(op.PagesSpec(2, 2 * group, dim, 16, dtype, store), [total], 31)
    spec, scale = c.spec, dim ** -0.5
    masks = [signed(sum(1 << int(i) for i in c.rng.choice(n, 3, replace=False))) for _ in range(n)]
    q, out, lse = attend(c, [(n, total)], masks)
    k, v = c.stored(c.k[0][:total]), c.stored(c.v[0][:total])
    qs = op.to_f32(bits_of(q), dtype).astype(np.float64)
    e_out, e_lse, mass, reach = op.attend(qs, k, v, total, scale, seen=op.drafted(masks, total))
    u = spec.half_step
    step = reach * (dim * 2.0 ** -24 + 4 * 2.0 ** -23) + 2.0 ** -21 + (total + 64) * 2.0 ** -24
    far = 1.01 * ((2 * step[..., None] + u * u) * mass + u * np.abs(e_out)) + 2.0 ** -24
    if dtype == "fp16":
        far = far + total * 2.0 ** -35 * np.abs(v).max()
    bad = np.abs(op.to_f32(bits_of(out), dtype) - e_out) > far
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}"
