"""Checks of rotary positions, drafts, weights, choices and moves that need no GPU: arguments that are refused, masks, and the oracle's parts."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from test_pages_arithmetic import run_pages_program
from test_pages_checks import config, pages_elsewhere  # noqa: F401  (a fixture)

NULL, SHAPE, ALIGN, CONFIG = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    from paper_2602_14236_amd import binding
    return binding.load_library()


def test_null_handles(lib):
    from paper_2602_14236_amd import binding as b
    batch, r, t = b.sali_page_batch(), b.sali_rows(), b.sali_rotary()
    assert lib.sali_pages_rotate(None, t, None, 0, 0, r, r, r, r, None) == NULL
    assert lib.sali_pages_attend_tree(None, 0, batch, None, r, 1.0, None, None, r, None, None) == NULL
    assert lib.sali_pages_weigh(None, 0, batch, r, 1.0, 0, 0, None, 0, None, None) == NULL
    assert lib.sali_pages_select(None, batch, None, 1, 0, 0, None, None) == NULL
    assert lib.sali_pages_keep(None, 0, batch, None, 1, 1, None, 0, None, None) == NULL


def test_draft_masks():
    from paper_2602_14236_amd.binding import draft_masks
    assert draft_masks([]) == []
    assert draft_masks([-1, 0, 0, 2, -1, 4]) == [1, 3, 5, 13, 16, 48]
    chain = draft_masks(list(range(-1, 63)))
    assert chain[62] == (1 << 63) - 1 and chain[63] == -1
    assert draft_masks([-1] * 64)[63] == -(1 << 63)
    torch.tensor(chain)                                          # 64 bits, signed
    for bad in ([0], [-2], [-1, 1], [-1] * 65):
        with pytest.raises(ValueError):
            draft_masks(bad)


def test_rotary_tables():
    from paper_2602_14236_amd.binding import Rotary
    f = torch.ones(32, dtype=torch.float64)
    r = Rotary(f, [16, 0, 16], adjacent=True)
    assert (r.c.pairs, r.c.axes, list(r.c.section), r.c.adjacent) == (32, 3, [16, 0, 16, 0], 1)
    assert list(Rotary(f).c.section) == [32, 0, 0, 0]
    for bad in ((f.float(),), (f[None],), (torch.ones(64, dtype=torch.float64)[::2],), (f, [16, 15]), (f, []), (f, [33, -1]), (f, [8, 8, 8, 4, 4])):
        with pytest.raises(ValueError):
            Rotary(*bad)


def test_tensors_that_are_none(pages_elsewhere):
    from paper_2602_14236_amd.binding import PageBatch, Rotary
    pages, state = pages_elsewhere
    pages._weights_shape = (5, 2, 16)
    for name in ("rotate", "attend_tree", "weigh", "select", "keep"):
        setattr(pages.lib, f"sali_pages_{name}", lambda *a, name=name: state.calls.append((name, state.device, a[-1])) or 0)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    batch = PageBatch(i(2), i(1), i(1, 5), 3, max_kv=80)
    kv, q = torch.zeros((3, 2, 64), dtype=torch.float16), torch.zeros((3, 4, 64), dtype=torch.float16)
    lse, w, seen, keep = torch.zeros((3, 4)), torch.zeros((5, 2, 16)), torch.zeros(3, dtype=torch.int64), i(1, 2, 7)
    r = Rotary(torch.ones(32, dtype=torch.float64), [16, 16])
    for stream, handle in ((None, 999), (SimpleNamespace(cuda_stream=77, device_index=-1), 77)):
        pages.rotate(r, i(2, 3), q, kv, stream=stream)
        pages.attend_tree(0, batch, seen, q, 1.0, q, lse, stream=stream)
        pages.weigh(0, batch, q, 1.0, lse, w, stream=stream)
        pages.select(batch, w, 7, keep, stream=stream)
        pages.keep(0, batch, keep, to=i(1, 9), weights=w, stream=stream)
        assert state.calls == [(name, -1, handle) for name in ("rotate", "attend_tree", "weigh", "select", "keep")]
        state.calls.clear()
    for bad in (lambda: pages.rotate(r, i(3, 3), q, kv), lambda: pages.rotate(r, i(2, 3).long(), q, kv), lambda: pages.rotate(r, i(2, 4), q, kv),
                lambda: pages.rotate(r, i(2, 3), kv, kv), lambda: pages.rotate(r, i(2, 3), q, kv.float()), lambda: pages.rotate(r, i(2, 3), q, None, q, kv),
                lambda: pages.rotate(r, i(6)[::2], q, kv), lambda: pages.attend_tree(0, batch, seen.int(), q, 1.0, q),
                lambda: pages.attend_tree(0, batch, seen[:2], q, 1.0, q), lambda: pages.attend_tree(0, batch, seen, q[:2], 1.0, q),
                lambda: pages.weigh(0, batch, q, 1.0, lse, w[:4]), lambda: pages.weigh(0, batch, q, 1.0, lse.double(), w),
                lambda: pages.weigh(0, batch, kv, 1.0, lse, w), lambda: pages.select(batch, w, 8, keep), lambda: pages.select(batch, w, 7, keep.long()),
                lambda: pages.select(batch, w, 7, i(1, 1, 7)), lambda: pages.keep(0, batch, i(2, 2, 7)), lambda: pages.keep(0, batch, keep, to=i(2, 9)),
                lambda: pages.keep(0, batch, keep, weights=w.double()), lambda: pages.keep(0, batch, keep[:, :, ::2])):
        with pytest.raises(ValueError):
            bad()
    assert state.calls == []


def test_a_single_position_is_no_array(pages_elsewhere):
    from paper_2602_14236_amd.binding import Rotary
    pages, state = pages_elsewhere
    q = torch.zeros((1, 4, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="position"):
        pages.rotate(Rotary(torch.ones(32, dtype=torch.float64)), torch.tensor(3, dtype=torch.int32), q, None)
    assert state.calls == []


def test_a_table_of_no_width_is_still_a_table(pages_elsewhere):
    """It has no address of its own; without one rows would move in the pages that they lie in."""
    from paper_2602_14236_amd.binding import PageBatch
    pages, state = pages_elsewhere
    pages._weights_shape = (5, 2, 16)
    pages.lib.sali_pages_keep = lambda *a: state.calls.append(a) or 0
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    batch = PageBatch(i(2), i(1), i(1, 5), 3, max_kv=80)
    pages.keep(0, batch, i(1, 2, 7), to=i(1, 0))
    pages.keep(0, batch, i(1, 2, 7))
    (table, width), (none, _) = ((a[6], a[7]) for a in state.calls)
    assert table and width == 0 and not none


def test_masks_of_drafts_by_key(tmp_path):
    """What 32 keys of a tile show of a mask, for every place that the tile can have before, at and behind the draft's beginning."""
    run_pages_program(tmp_path, """
int main() {
    srand(5);
    for (int round = 0; round < 2000; ++round) {
        const int n = rand() % 64 + 1;
        uint64_t mask = 0;
        for (int i = 0; i < 64; ++i) mask |= (uint64_t)(rand() % 3 == 0) << i;
        if (round % 5 == 0) mask = ~0ull;
        for (int from = -200; from < 200; ++from) {
            const DraftSight s = draft_sight(mask, n, from);
            for (int c = 0; c < 32; ++c) {
                const int i = from + c;
                const bool seen = i < 0 || (i < n && (mask >> i & 1) != 0);
                if (s.has(c) != seen) { printf("%d %d %d\\n", n, from, c); return 1; }
            }
        }
        for (int from : {-2147483647 + 1100, -100000, 100000, 2147483647 - 1100})
            if (draft_sight(mask, n, from).word != (from < 0 ? ~0u : 0u)) return 2;
        const PageSeq q = {0, n, n + rand() % 300};
        const View v = view_of_draft<32>(q);
        if (v.first != q.len - n - 1 || v.last != q.len - 1 || v.tiles != (q.len + 31) / 32 || tile_at(v, v.tiles - 1) * 32 > v.last) return 3;
        for (int t = 0; t < v.tiles; ++t)
            if (partly_hidden(v, 0, 0, 32 * t, 32) != (32 * t + 31 >= q.len - n)) return 4;
    }
    return 0;
}
""")


def test_oracle_choice():
    from oracle import pages as op
    assert op.select(np.array([1.0, 5.0, 5.0, 0.0, 5.0, 2.0]), 3) == [1, 2, 4]
    assert op.select(np.array([1.0, 5.0, 5.0, 0.0, 5.0, 2.0]), 2) == [1, 2]
    assert op.select(np.array([1.0, 5.0, 5.0, 0.0, 5.0, 2.0]), 4, 1, 2) == [0, 1, 4, 5]
    assert op.select(np.array([-0.0, 0.0, np.nan, -1.0]), 2) == [0, 2]
    assert op.select(np.array([1.0, 2.0]), 5) == [0, 1]


def test_oracle_rotation():
    """A quarter turn, the way back, and what is in no pair"""
    from oracle import pages as op
    x = np.arange(8.0).reshape(1, 1, 8)
    pos = np.array([[1], [2]], np.int32)
    f = np.array([np.pi / 2, np.pi / 2])
    out, _ = op.rotate(x, pos, f, [1, 1])
    assert np.allclose(out[0, 0], [-2, -1, 0, -3, 4, 5, 6, 7])
    out, _ = op.rotate(x, pos, f, [1, 1], adjacent=True)
    assert np.allclose(out[0, 0], [-1, 0, -2, -3, 4, 5, 6, 7])
    back, _ = op.rotate(out, pos, f, [1, 1], adjacent=True, inverse=True)
    assert np.allclose(back, x)


@pytest.mark.parametrize("store", ("16", "int8", "int4"))
def test_oracle_bytes_of_tokens(store):
    """Every byte of a block is one token's."""
    from oracle import pages as op
    spec = op.PagesSpec(1, 1, 64, 16, "fp16", store)
    at = np.concatenate([op.bytes_of_token(spec, t) for t in range(16)])
    assert np.array_equal(np.sort(at), np.arange(spec.block_bytes))
