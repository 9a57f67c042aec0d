"""Rotary positions on the GPU against oracle/pages.py (float64): axes, pairs in both orders, far positions, strides, values that are not finite."""
import itertools

import numpy as np
import pytest
import torch

from oracle import pages as op
from test_gpu_pages import DEV, TORCH, bits_of, rows

pytestmark = pytest.mark.gpu


def handle(dtype, dim, heads=6, kv_heads=2):
    from paper_2602_14236_amd import binding
    return binding.SaliPages(binding.make_pages_config(n_kv_heads=kv_heads, n_heads=heads, head_dim=dim, page_tokens=16, n_pages=1, dtype=TORCH[dtype]), DEV)


def frequencies(pairs):
    return 10000.0 ** (-np.arange(pairs, dtype=np.float64) / pairs)


def rotary(pairs, sections=None, adjacent=False):
    from paper_2602_14236_amd import binding
    return binding.Rotary(torch.from_numpy(frequencies(pairs)).to(DEV), sections, adjacent=adjacent)


def check(got, x, position, pairs, sections, adjacent, inverse, dtype):
    half = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    x = op.to_f32(bits_of(x), dtype).astype(np.float64)
    e, size = op.rotate(x, position, frequencies(pairs), sections, adjacent, inverse)
    got = op.to_f32(bits_of(got), dtype).astype(np.float64)
    # sine and cosine in fp32 (2^-22), two products and their sum (2^-23), the angle (2^31 turns at the most, 2^-52 of them twice: 2^-18 radians); then one rounding, of
    # numbers down to the type's smallest
    reach = np.abs(position.astype(np.float64)).max(initial=1.0)
    far = size * (2.0 ** -21 + 8 * reach * 2.0 ** -52) + half * np.abs(e) * 1.01 + (2.0 ** -25 if dtype == "fp16" else 2.0 ** -134)
    same = (got == e) | (np.isnan(got) & np.isnan(e))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - e) <= far))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[bad][0]} against {e[bad][0]}, bound {far[bad][0]}"


def positions(rng, axes, n, most=20000):
    return rng.integers(-3, most, (axes, n)).astype(np.int32)


@pytest.mark.parametrize("dtype,dim", itertools.product(("fp16", "bf16"), (64, 128)))
@pytest.mark.parametrize("axes,adjacent", itertools.product((1, 2, 3, 4), (False, True)))
def test_axes_and_orders(dtype, dim, axes, adjacent):
    rng = np.random.default_rng(axes)
    p = handle(dtype, dim)
    for pairs, n in ((dim // 2, 5), (dim // 4, 33), (12, 3), (max(1, axes), 70), (dim // 2 - 1, 2), (8, 1)):
        cuts = np.sort(rng.integers(0, pairs + 1, axes - 1))
        sections = np.diff(np.concatenate([[0], cuts, [pairs]])).tolist()          # empty ones among them
        pos = positions(rng, axes, n)
        q, k = rows(rng, n, 6, dim, dtype).to(DEV), rows(rng, n, 2, dim, dtype).to(DEV)
        q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        p.rotate(rotary(pairs, sections, adjacent), torch.from_numpy(pos).to(DEV), q, k, q_out, k_out)
        check(q_out, q, pos, pairs, sections, adjacent, False, dtype)
        check(k_out, k, pos, pairs, sections, adjacent, False, dtype)
        still = slice(2 * pairs, None)
        assert torch.equal(q_out[..., still], q[..., still])


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 1), (24, 8), (32, 8), (40, 40), (33, 11), (128, 1), (200, 100)])
@pytest.mark.parametrize("pairs,adjacent", [(64, False), (64, True), (24, False), (13, False), (13, True)])
def test_long_calls_are_their_parts(heads, kv_heads, pairs, adjacent):
    """Of every number of heads: blocks that have a token each, and several for a token."""
    rng = np.random.default_rng(heads)
    torch.manual_seed(heads)
    p, n, t = handle("bf16", 128, heads, kv_heads), 1030, rotary(pairs, None, adjacent)
    pos = torch.from_numpy(positions(rng, 1, n)).to(DEV)
    q, k = (torch.randn((n, h, 128), dtype=torch.float32, device=DEV).to(torch.bfloat16) for h in (heads, kv_heads))
    q_out, k_out, q_part, k_part = (torch.full_like(x, 7.0) for x in (q, k, q, k))
    p.rotate(t, pos, q, k, q_out, k_out)
    for lo in range(0, n, 103):
        at = slice(lo, lo + 103)
        p.rotate(t, pos[:, at].contiguous(), q[at], k[at], q_part[at], k_part[at])
    assert torch.equal(q_out, q_part) and torch.equal(k_out, k_part)
    few = np.r_[0:3, 700, n - 1]
    check(q_out[few], q[few], pos.cpu().numpy()[:, few], pairs, [pairs], adjacent, False, "bf16")
    check(k_out[few], k[few], pos.cpu().numpy()[:, few], pairs, [pairs], adjacent, False, "bf16")


@pytest.mark.parametrize("dtype", ("fp16", "bf16"))
@pytest.mark.parametrize("pairs,adjacent", [(64, False), (24, False), (64, True), (12, False), (12, True)])
def test_rows_past_the_caches(dtype, pairs, adjacent):
    """Calls of 128 MB of rows and more, and one just below, in every layout, in place and not: the same bits as in short calls."""
    rng, heads, kv_heads = np.random.default_rng(7), 200, 100
    torch.manual_seed(7)
    p, t = handle(dtype, 128, heads, kv_heads), rotary(pairs, None, adjacent)
    limit = (128 << 20) // (2 * 128 * (heads + kv_heads))
    for n in (limit, limit + 1, 2100):
        pos = torch.from_numpy(positions(rng, 1, n)).to(DEV)
        qkv = torch.randn((n, heads + 2 * kv_heads, 128), dtype=torch.float32, device=DEV).to(TORCH[dtype])
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        q_out, k_out, q_part, k_part = (torch.full_like(x, 7.0, memory_format=torch.contiguous_format) for x in (q, k, q, k))
        p.rotate(t, pos, q, k, q_out, k_out)
        for lo in range(0, n, 300):
            at = slice(lo, lo + 300)
            p.rotate(t, pos[:, at].contiguous(), q[at], k[at], q_part[at], k_part[at])
        assert torch.equal(q_out, q_part) and torch.equal(k_out, k_part)
        few = np.r_[0:2, n - 1]
        check(q_out[few], q[few], pos.cpu().numpy()[:, few], pairs, [pairs], adjacent, False, dtype)
        check(k_out[few], k[few], pos.cpu().numpy()[:, few], pairs, [pairs], adjacent, False, dtype)
        still = v.clone()
        p.rotate(t, pos, q, k)
        assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(v, still)
        p.rotate(t, pos, q, k, inverse=True)
        p.rotate(t, pos, q_out, k_out, q_part, k_part, inverse=True)
        assert torch.equal(q, q_part) and torch.equal(k, k_part)


@pytest.mark.parametrize("dtype", ("fp16", "bf16"))
@pytest.mark.parametrize("pairs,adjacent", [(64, False), (64, True), (20, False), (20, True)])
def test_in_place_strided_and_back(dtype, pairs, adjacent):
    """Queries and keys as slices of one product's output, in place; inverse is the oracle's too; the rest of the array keeps its bits."""
    rng = np.random.default_rng(5)
    p = handle(dtype, 128)
    r = rotary(pairs, adjacent=adjacent)
    for n in (1, 7, 1500):
        pos = positions(rng, 1, n, 100000)
        qkv = rows(rng, n, 10, 128, dtype).to(DEV)
        before = qkv.clone()
        for inverse in (False, True):
            now = qkv.clone()
            p.rotate(r, torch.from_numpy(pos).to(DEV)[0], qkv[:, :6], qkv[:, 6:8], inverse=inverse)
            check(qkv[:, :6], now[:, :6], pos, pairs, [pairs], adjacent, inverse, dtype)
            check(qkv[:, 6:8], now[:, 6:8], pos, pairs, [pairs], adjacent, inverse, dtype)
        assert torch.equal(qkv[:, 8:].view(torch.int16), before[:, 8:].view(torch.int16))


def test_one_of_the_two():
    rng = np.random.default_rng(6)
    p, r = handle("fp16", 64), rotary(32)
    q, k = rows(rng, 9, 6, 64, "fp16").to(DEV), rows(rng, 9, 2, 64, "fp16").to(DEV)
    pos = positions(rng, 1, 9)
    t = torch.from_numpy(pos).to(DEV)
    both = [torch.empty_like(q), torch.empty_like(k)]
    p.rotate(r, t, q, k, *both)
    alone = [torch.empty_like(q), torch.empty_like(k)]
    p.rotate(r, t, q, None, alone[0])
    p.rotate(r, t, None, k, None, alone[1])
    assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1])
    p.rotate(r, t, None, None)


def test_keys_of_a_frame():
    """Keys as the frame cache takes them, [head][576][D], each patch at its frame, row and column."""
    rng = np.random.default_rng(7)
    p, sections = handle("fp16", 128), [16, 24, 24]
    k = rows(rng, 2, 576, 128, "fp16").to(DEV)
    i = np.arange(576)
    pos = np.stack([np.full(576, 3), i // 24, i % 24]).astype(np.int32)
    before = k.clone()
    p.rotate(rotary(64, sections), torch.from_numpy(pos).to(DEV), None, k.transpose(0, 1))
    check(k.transpose(0, 1), before.transpose(0, 1), pos, 64, sections, False, False, "fp16")


@pytest.mark.parametrize("adjacent", (False, True))
def test_farthest_positions(adjacent):
    rng = np.random.default_rng(8)
    p, r = handle("bf16", 128), rotary(64, adjacent=adjacent)
    pos = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, 2 ** 24 + 1]], np.int32)
    q = rows(rng, 7, 6, 128, "bf16").to(DEV)
    out = torch.empty_like(q)
    p.rotate(r, torch.from_numpy(pos).to(DEV), q, None, out)
    check(out, q, pos, 64, [64], adjacent, False, "bf16")
    assert torch.equal(out[0], q[0])                                              # position 0 turns nothing


@pytest.mark.parametrize("dtype", ("fp16", "bf16"))
def test_values_that_are_not_finite(dtype):
    """They stay in their pair."""
    rng = np.random.default_rng(9)
    p = handle(dtype, 64)
    q = rows(rng, 4, 6, 64, dtype).to(DEV)
    q[1, 2, 3], q[2, 0, 40], q[3, 5, 63] = float("inf"), float("nan"), float("-inf")
    pos = positions(rng, 1, 4) + 5
    for pairs, adjacent in ((32, False), (32, True), (16, False), (9, False)):
        out = torch.empty_like(q)
        p.rotate(rotary(pairs, adjacent=adjacent), torch.from_numpy(pos).to(DEV), q, None, out)
        got, x = out.float().cpu(), q.float().cpu()
        there = torch.zeros_like(x, dtype=torch.bool)
        for t, h, e in ((1, 2, 3), (2, 0, 40), (3, 5, 63)):
            there[t, h, e] = True
            if e < 2 * pairs:
                there[t, h, (e ^ 1) if adjacent else (e + pairs) % (2 * pairs)] = True
        assert torch.equal(~got.isfinite(), there)


def test_replayed():
    """A captured call takes the positions that stand there when it is replayed."""
    rng = np.random.default_rng(10)
    p, r = handle("bf16", 128), rotary(64, [20, 22, 22])
    q, k = rows(rng, 40, 6, 128, "bf16").to(DEV), rows(rng, 40, 2, 128, "bf16").to(DEV)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    pos = torch.zeros((3, 40), dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    p.rotate(r, pos, q, k, q_out, k_out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.rotate(r, pos, q, k, q_out, k_out)
    for _ in range(3):
        now = positions(rng, 3, 40)
        pos.copy_(torch.from_numpy(now))
        graph.replay()
        torch.cuda.synchronize()
        check(q_out, q, now, 64, [20, 22, 22], False, False, "bf16")
        check(k_out, k, now, 64, [20, 22, 22], False, False, "bf16")


def test_stream_and_no_tokens():
    rng = np.random.default_rng(11)
    p, r = handle("fp16", 64), rotary(32)
    q = rows(rng, 300, 6, 64, "fp16").to(DEV)
    pos = positions(rng, 1, 300)
    t, out, side = torch.from_numpy(pos).to(DEV), torch.empty_like(q), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p.rotate(r, t, q, None, out, stream=side)
    side.synchronize()
    check(out, q, pos, 32, [32], False, False, "fp16")
    p.rotate(r, t[:, :0].contiguous(), q[:0], None)
    assert p.get_status() == 0


def test_refusals():
    """What the library refuses, by code; nothing is launched."""
    from paper_2602_14236_amd import binding as b
    p, r = handle("fp16", 64), rotary(32, [16, 16])
    x = torch.full((5, 6, 64), 7.0, dtype=torch.float16, device=DEV)
    pos = torch.zeros((2, 5), dtype=torch.int32, device=DEV)
    call = lambda c, n=5, at=pos.data_ptr(), q=b.sali_rows(x.data_ptr(), 384, 64), out=b.sali_rows(x.data_ptr(), 384, 64): \
        p.lib.sali_pages_rotate(p.handle, c, at, n, 0, q, None, out, None, None)

    def table(pairs=32, axes=2, sections=(16, 16, 0, 0), frequency=None):
        import ctypes as C
        return b.sali_rotary(r.frequency.data_ptr() if frequency is None else frequency, pairs, axes, (C.c_int32 * 4)(*sections), 0, 0)

    for bad in (dict(pairs=0, sections=(0, 0, 0, 0)), dict(pairs=33, sections=(16, 17, 0, 0)), dict(axes=0), dict(axes=5), dict(sections=(16, 15, 0, 0)),
                dict(sections=(33, -1, 0, 0)), dict(axes=1)):
        assert call(table(**bad)) == -4, bad
    assert call(None) == -1 and call(table(), at=None) == -1 and call(table(), out=None) == -1 and call(table(frequency=0)) == -1
    assert call(table(), q=b.sali_rows(None, 384, 64)) == -1
    assert call(table(), n=-1) == -2 and call(table(), n=1 << 24) == -2
    assert call(table(), at=pos.data_ptr() + 2) == -3 and call(table(frequency=r.frequency.data_ptr() + 4)) == -3
    assert call(table(), q=b.sali_rows(x.data_ptr() + 8, 384, 64)) == -3 and call(table(), out=b.sali_rows(x.data_ptr(), 384, 60)) == -3
    torch.cuda.synchronize()
    assert (x == 7).all() and p.get_status() == 0
