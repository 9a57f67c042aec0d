// Arithmetic of the paged cache that the host can run too (tests/test_pages_arithmetic.py does): layout, which blocks, tiles and units a batch has.
#pragma once

#include "arith.h"
#include "sali.h"

namespace sali {

constexpr int kBlockTokens = 16;            // tokens of a block, the unit of the layout
constexpr int kMostPositions = 0x7FFFFFFF - 1024;       // tokens of a sequence
constexpr int kTileTokens = 32;             // tokens of a step of the attention: two blocks

// bytes of a block's parts, in their order
struct BlockLayout {
    uint32_t v, ks, vs, kz, vz, bytes;      // K is at 0
};
constexpr BlockLayout block_layout(int store, int dim) {
    const uint32_t d = (uint32_t)dim;
    const uint32_t codes = store == SALI_STORE_16 ? 32 * d : (store == SALI_STORE_INT8 ? 16 * d : 8 * d);
    const uint32_t scale = store == SALI_STORE_16 ? 0 : 2 * d, zero = store == SALI_STORE_INT4 ? d : 0;
    return {codes, 2 * codes, 2 * codes + scale, 2 * codes + 2 * scale, 2 * codes + 2 * scale + zero, 2 * codes + 2 * scale + 2 * zero};
}
SALI_BOTH int place_of_token(int t) { return 8 * (t >> 2 & 1) + 4 * (t >> 3) + (t & 3); }      // t = 8 a + 4 b + i
SALI_BOTH int token_of_place(int p) { return 8 * (p >> 2 & 1) + 4 * (p >> 3) + (p & 3); }      // the same exchange

template <typename T>
SALI_BOTH T least(T a, T b) { return a < b ? a : b; }
template <typename T>
SALI_BOTH T most(T a, T b) { return a < b ? b : a; }

// first, first + step, .. below count, all of them up to 2^31 - 1: counted without a sign, since the last step may end behind that
template <typename F>
SALI_BOTH void each_from(int first, int count, int step, F f) {
    for (uint32_t i = (uint32_t)first; i < (uint32_t)count; i += (uint32_t)step) f(i);
}

// One sequence of a batch: rows first .. first + n - 1 are its tokens len - n .. len - 1.  n = 0 where its numbers contradict each other, the
// rows or its table.
struct PageSeq {
    int32_t first, n, len;
};
SALI_BOTH bool page_seq_holds(int64_t a, int64_t b, int64_t len, int64_t n_tokens, int64_t max_q, int64_t room) {
    return a >= 0 && b >= a && b <= n_tokens && b - a <= max_q && len >= b - a && len <= room;
}

// Append and read take the batch by slots of one 16-token block each: sequence s owns the slots from first / 16 + 2 s on.  n tokens touch at
// most n / 16 + 2 blocks, and up to the next sequence's first slot there are that many, so a slot's sequence is found without a sum over
// those before it.
SALI_BOTH int64_t first_slot(int32_t first, int s) { return (int64_t)(first < 0 ? 0 : first) / kBlockTokens + 2ll * s; }
// The block of its sequence that a slot stands for, -1: none (slots that it has no use for, and those of rows before the batch's first, if that is not row 0).
SALI_BOTH int block_of_slot(const PageSeq& q, int s, int64_t slot) {
    const int64_t nth = slot - first_slot(q.first, s), block = (q.len - q.n) / kBlockTokens + nth;
    return q.n > 0 && nth >= 0 && block * kBlockTokens < q.len ? (int)block : -1;
}

// The keys a set of rows sees: positions first .. last of the sequence (of the set's first and last token), window and sinks.  Tiles of kTokens
// tokens that some row sees: the first `head` from the sequence's beginning, then from tile `from` on.
struct View {
    int32_t first, last;
    int32_t head, from, tiles;
};
template <int kTokens>
SALI_BOTH View view_of(int first, int last, int window, int sinks) {
    View v = {first, last, 0, 0, 0};
    const int lo = window > 0 ? most(0, first - window + 1) : 0;
    v.from = lo / kTokens;
    v.head = window > 0 ? least((sinks + kTokens - 1) / kTokens, v.from) : 0;
    v.tiles = v.head + last / kTokens + 1 - v.from;
    return v;
}
SALI_BOTH int tile_at(const View& v, int i) { return i < v.head ? i : v.from + (i - v.head); }
// has some row of the view some key of the tile's n tokens (from j0) out of sight?
SALI_BOTH bool partly_hidden(const View& v, int window, int sinks, int j0, int n) {
    if (j0 + n - 1 > v.first) return true;
    return window > 0 && j0 <= v.last - window && j0 + n > sinks;
}
SALI_BOTH bool sees(int p, int j, int window, int sinks) {
    return j <= p && (window == 0 || j > p - window || j < sinks);
}

// the same for keys counted from j0 on
struct Sight {
    int32_t last, from, sunk;               // keys up to `last` that lie behind `from` or before `sunk`
    SALI_BOTH bool has(int c) const { return c <= last && (c > from || c < sunk); }
};
SALI_BOTH Sight sight_of(int p, int j0, int window, int sinks) { return {p - j0, window == 0 ? -2147483647 : p - window - j0, sinks - j0}; }

// The keys that drafted tokens see: the history, and of the draft what each token's mask names, so all of them see the keys up to the history's last and some of
// them may see those up to the sequence's last.
template <int kTokens>
SALI_BOTH View view_of_draft(const PageSeq& q) { return {q.len - q.n - 1, q.len - 1, 0, 0, (q.len - 1) / kTokens + 1}; }
// what a mask of the draft's tokens, of which there are n, shows of 32 keys; `from`: the first of them, counted from the draft's first token
struct DraftSight {
    uint32_t word;
    SALI_BOTH bool has(int c) const { return (word >> c & 1u) != 0u; }
};
SALI_BOTH DraftSight draft_sight(uint64_t mask, int n, int from) {
    if (n < 64) mask &= (1ull << n) - 1ull;
    if (from >= 64) return {0u};
    if (from >= 0) return {(uint32_t)(mask >> from)};
    if (from <= -32) return {~0u};
    return {(uint32_t)(mask << -from) | ((1u << -from) - 1u)};
}

// `total` tiles in `blocks` stretches (blocks <= total) that differ by one at most, the longer ones first
struct Stretches {
    uint32_t each, longer;
    SALI_BOTH Stretches(uint32_t total, uint32_t blocks) : each(total / blocks), longer(total - total / blocks * blocks) {}
    SALI_BOTH uint32_t start(uint32_t block) const { return block * each + least(block, longer); }
    SALI_BOTH uint32_t of(uint32_t tile) const {
        const uint32_t in_longer = longer * (each + 1);
        return tile < in_longer ? tile / (each + 1) : longer + (tile - in_longer) / each;
    }
};
constexpr int kStreamMinTiles = 4;          // of a stretch
// Blocks of the tile kernel: 32 rows a wave, and of each step's keys 8 a wave.  A block of twelve waves has a compute unit to itself, of those of four waves
// three share one.
constexpr int tile_rows(int waves) { return 32 * waves; }
constexpr int tile_keys(int waves) { return 8 * waves; }

// row tiles of a batch by slots, as those of blocks in append: sequence s owns the slots from first * group / rows + s on
SALI_BOTH int64_t tile_slots(int64_t n_tokens, int group, int64_t n_seqs, int rows) { return n_tokens * group / rows + n_seqs; }
// How the row tiles' work is shared out, one of two ways.
// Shares: row tiles with more tiles of keys than a fair share of the whole are cut, into at most twice as many parts as they have shares, so there are
// at most tile_parts of them a head; the pieces are then taken the longest first.
SALI_BOTH int tile_shares(int n_kv, int waves) { return ((waves == 12 ? 256 : 512) + n_kv - 1) / n_kv; }
SALI_BOTH int tile_parts(int n_kv, int waves) { return 2 * tile_shares(n_kv, waves); }
// tiles of a share of `sum` tiles a head
SALI_BOTH int fair_share(int64_t sum, int shares) { return (int)((most(sum, (int64_t)1) + shares - 1) / shares); }
SALI_BOTH int parts_of(int tiles, int share) { return tiles > share ? (tiles + share - 1) / share : 1; }
// Stretches: all tiles of keys of a head in a row, weighted by what they cost, are cut into equal stretches, one a block.
SALI_BOTH int stretch_blocks(int in_flight, int n_kv) { return most(1, in_flight / n_kv); }
// What a tile of keys costs a row tile of `rows` rows: bringing it in, and each wave's 32 rows (4, 8 and 12 waves of rows with 96 keys: 3.0, 5.0 and 5.3 us)
SALI_BOTH int tile_weight(int rows) { return 7 + (rows + 31) / 32; }
SALI_BOTH uint64_t stretch_length(uint64_t total, int blocks) { return most((total + (uint32_t)blocks - 1u) / (uint32_t)blocks, (uint64_t)(2 * (7 + 12))); }
// A row tile with `tiles` tiles of keys of weight `weight`, from position `at` of the row on.  A tile of keys is of the stretch that its start lies in.
struct TileSpan {
    uint64_t at;
    int32_t tiles, weight;
    SALI_BOTH uint64_t end() const { return at + (uint64_t)((uint32_t)tiles * (uint32_t)weight); }
    // tiles that start before position p
    SALI_BOTH int before(uint64_t p) const {
        if (p <= at) return 0;
        return (int)(((uint32_t)(least(p, end()) - at) + (uint32_t)weight - 1u) / (uint32_t)weight);
    }
    SALI_BOTH int first_block(uint64_t length) const { return (int)(at / length); }
    SALI_BOTH int last_block(uint64_t length) const { return (int)((at + (uint64_t)((uint32_t)(tiles - 1) * (uint32_t)weight)) / length); }
};
// The piece of row tile `unit` in block `block`: a block's pieces lie side by side.
SALI_BOTH int stretch_piece(int unit, int block) { return unit + block; }

constexpr int kMostDrafted = 64;            // tokens of a draft: bits of a mask

// (rows of a batch are counted in 31 bits)
template <int kWaves>
SALI_BOTH View view_of_rows(const PageSeq& q, int row_tile, int group, int window, int sinks) {
    const uint32_t first_row = (uint32_t)row_tile * (uint32_t)tile_rows(kWaves), rows = (uint32_t)(q.n * group);
    const uint32_t last_row = least(rows, first_row + (uint32_t)tile_rows(kWaves)) - 1u, g = (uint32_t)group;
    const int first = q.len - q.n;
    return view_of<tile_keys(kWaves)>(first + (int)(first_row / g), first + (int)(last_row / g), window, sinks);
}

}  // namespace sali
