"""Arithmetic of the paged cache that kernels and host share (csrc/pages_arith.h), on the CPU: a program with the header's own code."""
import os
import subprocess

import pytest


def run_pages_program(tmp_path, body):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include <vector>\n#include "pages_arith.h"\nusing namespace sali;\n' + body)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(root, "paper_2602_14236_amd", "csrc"), "-I",
                    os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stdout


def test_places_are_an_exchange_and_blocks_are_whole_pieces(tmp_path):
    run_pages_program(tmp_path, """
int main() {
    for (int t = 0; t < 16; ++t) {
        const int a = t / 8, b = t / 4 % 2, i = t % 4;
        if (place_of_token(t) != 8 * b + 4 * a + i || token_of_place(place_of_token(t)) != t) return 1;
    }
    for (int dim : {64, 128})
        for (int store : {SALI_STORE_16, SALI_STORE_INT8, SALI_STORE_INT4}) {
            const BlockLayout l = block_layout(store, dim);
            const uint32_t bytes = store == SALI_STORE_16 ? 64 * dim : (store == SALI_STORE_INT8 ? 36 * dim : 22 * dim);
            if (l.bytes != bytes || l.v % 16 || l.ks % 16 || l.vs % 16 || l.kz % 16 || l.vz % 16 || l.bytes % 16) return 2;
        }
    return 0;
}
""")


@pytest.mark.parametrize("seed", range(3))
def test_every_block_and_row_tile_has_one_slot(tmp_path, seed):
    """Random batches: the slots of a sequence hold all blocks it touches and end before the next sequence's, and within what is launched;
    the same for tiles of rows."""
    run_pages_program(tmp_path, """
int main() {
    srand(%d);
    for (int round = 0; round < 3000; ++round) {
        const int n = rand() %% 20 + 1, group = rand() %% 3 ? 1 << rand() %% 6 : rand() %% 70 + 1;
        std::vector<int> start(n + 1, 0), len(n);
        for (int s = 0; s < n; ++s) {
            const int fresh = rand() %% 4 ? rand() %% 40 : rand() %% 700;
            start[s + 1] = start[s] + fresh;
            len[s] = fresh + rand() %% 300;
        }
        const int64_t tokens = start[n] + rand() %% 5, slots = tokens / kBlockTokens + 2ll * n, rows = rand() %% 2 ? tile_rows(4) : tile_rows(12), tiles = tile_slots(tokens, group, n, rows);
        for (int s = 0; s < n; ++s) {
            const int fresh = start[s + 1] - start[s];
            const int blocks = fresh ? (len[s] - 1) / 16 - (len[s] - fresh) / 16 + 1 : 0;
            const int64_t end = first_slot(start[s], s) + blocks, next = s + 1 < n ? first_slot(start[s + 1], s + 1) : slots;
            if (end > next) { printf("blocks of sequence %%d\\n", s); return 1; }
            const int64_t t0 = (int64_t)start[s] * group / rows + s, mine = ((int64_t)fresh * group + rows - 1) / rows;
            const int64_t t1 = s + 1 < n ? (int64_t)start[s + 1] * group / rows + s + 1 : tiles;
            if (t0 + mine > t1) { printf("tiles of sequence %%d\\n", s); return 1; }
        }
    }
    return 0;
}
""" % seed)


def test_sequences_that_contradict_their_batch_are_left_out(tmp_path):
    run_pages_program(tmp_path, """
int main() {
    // start, next start, length, rows, most new tokens, room
    if (!page_seq_holds(0, 0, 0, 0, 0, 0) || !page_seq_holds(3, 8, 5, 8, 5, 5) || !page_seq_holds(3, 4, 64, 8, 5, 64)) return 1;
    if (page_seq_holds(-1, 2, 9, 8, 5, 64)) return 2;              // rows before the array
    if (page_seq_holds(3, 2, 9, 8, 5, 64)) return 3;               // starts that fall
    if (page_seq_holds(3, 9, 9, 8, 9, 64)) return 4;               // rows past the array
    if (page_seq_holds(0, 5, 4, 8, 5, 64)) return 5;               // more new tokens than tokens
    if (page_seq_holds(0, 5, -1, 8, 5, 64)) return 6;
    if (page_seq_holds(0, 5, 65, 8, 5, 64)) return 7;              // past its table
    if (page_seq_holds(0, 6, 9, 8, 5, 64)) return 8;               // more new tokens than said
    if (page_seq_holds(0, 5, 2147483647ll, 8, 5, 2147483646ll)) return 9;
    if (page_seq_holds(-2147483647ll, 2147483647ll, 5, 8, 5, 64)) return 10;
    return 0;
}
""")


@pytest.mark.parametrize("seed", range(3))
def test_views_hold_every_key_that_is_seen(tmp_path, seed):
    run_pages_program(tmp_path, """
template <int kTokens>
int check(int first, int last, int window, int sinks) {
    const View v = view_of<kTokens>(first, last, window, sinks);
    std::vector<int> times((size_t)last / kTokens + 2, 0);
    for (int i = 0; i < v.tiles; ++i) {
        const int t = tile_at(v, i);
        if (t < 0 || t > last / kTokens || times[t]++) return 1;
    }
    for (int t = 0; t <= last / kTokens; ++t)
        for (int part = 0; part < kTokens; part += 32) {
            bool all = true, any = false;
            for (int j = t * kTokens + part; j < t * kTokens + part + 32; ++j)
                for (int p = first; p <= last; ++p) {
                    (sees(p, j, window, sinks) ? any : all) = sees(p, j, window, sinks);
                    const int j0 = j - rand() %% 64;
                    if (sight_of(p, j0, window, sinks).has(j - j0) != sees(p, j, window, sinks)) return 4;
                }
            if (any && !times[t]) return 2;
            if (!all && !partly_hidden(v, window, sinks, t * kTokens + part, 32)) return 3;
        }
    return 0;
}
int main() {
    srand(%d);
    for (int round = 0; round < 1500; ++round) {
        const int first = rand() %% 400, last = first + (rand() %% 3 ? rand() %% 20 : rand() %% 200);
        const int window = rand() %% 4 ? rand() %% 150 + 1 : 0, sinks = window && rand() %% 3 ? rand() %% 140 : 0;
        const int a = check<32>(first, last, window, sinks), b = check<96>(first, last, window, sinks);
        if (a || b) { printf("%%d..%%d window %%d sinks %%d: %%d %%d\\n", first, last, window, sinks, a, b); return 1; }
    }
    return 0;
}
""" % seed)


@pytest.mark.parametrize("seed", range(3))
def test_stretches_and_shares(tmp_path, seed):
    """Equal stretches cover the tiles and every tile knows its block; parts of cut units cover them, are no longer than a share and no more
    than there is room for; stretches of weighted row tiles cover them, every block of a cut one has tiles of it, and a block's pieces lie side by side."""
    run_pages_program(tmp_path, """
int main() {
    srand(%d);
    for (int round = 0; round < 2000; ++round) {
        const uint32_t total = rand() %% 2 ? rand() %% 3000 + 1 : (uint32_t)rand() / 2 + 1, blocks = least(total, (uint32_t)(rand() %% 768 + 1));
        const Stretches cut(total, blocks);
        if (cut.start(0) != 0 || cut.start(blocks) != total) return 1;
        for (int k = 0; k < 200; ++k) {
            const uint32_t b = rand() %% blocks, lo = cut.start(b), hi = cut.start(b + 1);
            if (lo >= hi || cut.of(lo) != b || cut.of(hi - 1) != b) return 2;
        }
    }
    for (int round = 0; round < 3000; ++round) {
        const int n_kv = rand() %% 3 ? 1 << rand() %% 7 : rand() %% 300 + 1, units = rand() %% 400 + 1;
        std::vector<int> tiles(units);
        int64_t sum = 0;
        const int longest = rand() %% 3000 + 1;
        for (int& t : tiles) sum += t = rand() %% longest + 1;
        const int waves = rand() %% 2 ? 4 : 12, share = fair_share(sum, tile_shares(n_kv, waves));
        int64_t cut = 0;
        for (int t : tiles) {
            const int parts = parts_of(t, share);
            if (parts > 1) cut += parts;
            for (int k = 0; k < parts; ++k) {
                const int lo = (int)((int64_t)t * k / parts), hi = (int)((int64_t)t * (k + 1) / parts);
                if (lo >= hi || hi - lo > share) return 3;
            }
        }
        if (cut > tile_parts(n_kv, waves)) { printf("%%lld parts, room for %%d\\n", (long long)cut, tile_parts(n_kv, waves)); return 4; }
    }
    for (int round = 0; round < 1000; ++round) {
        const int n_kv = rand() %% 3 ? 1 << rand() %% 7 : rand() %% 900 + 1, units = rand() %% 400 + 1, blocks = stretch_blocks(256, n_kv);
        if (blocks < 1 || (blocks > 1 && blocks * n_kv > 256)) return 5;
        std::vector<TileSpan> spans;
        uint64_t total = 0;
        const int longest = rand() %% 4 ? rand() %% 300 + 1 : 60000000;
        for (int u = 0; u < units; ++u) {
            spans.push_back({total, rand() %% longest + 1, tile_weight(rand() %% 384 + 1)});
            total = spans.back().end();
        }
        const uint64_t length = stretch_length(total, blocks);
        int block = 0, piece = -1, parts = 0, merges = 0;   // those so far
        for (int u = 0; u < units; ++u) {
            const TileSpan& x = spans[u];
            const int first = x.first_block(length), last = x.last_block(length);
            if (first < block || first > block + 1 || last >= blocks) return 6;
            int next = 0;                                   // of the unit's tiles
            for (int b = first; b <= last; ++b) {
                const int lo = x.before(b * length), hi = x.before((b + 1) * length), own = stretch_piece(u, b);
                if (lo != next || hi <= lo) return 7;       // every block of the unit has tiles of it
                next = hi;
                if (own <= piece || (b == block && u > 0 && own != piece + 1) || own >= units + blocks) return 8;
                piece = own;
                block = b;
            }
            if (next != x.tiles) return 9;
            if (last > first) ++merges, parts += last - first + 1;
        }
        if (merges > blocks || parts > tile_parts(n_kv, 12)) return 10;
    }
    return 0;
}
""" % seed)


@pytest.mark.parametrize("seed", range(3))
def test_slots_of_batches_that_start_behind_row_0(tmp_path, seed):
    """Parts of larger batches (the first start is not 0): every block of a sequence has one slot, and a slot that stands for none says so, those
    before the first row too; no block lies before a sequence's new tokens or behind its end."""
    run_pages_program(tmp_path, """
int main() {
    srand(%d);
    for (int round = 0; round < 3000; ++round) {
        const int n = rand() %% 20 + 1;
        std::vector<PageSeq> seqs(n);
        int row = rand() %% 400;
        for (PageSeq& q : seqs) {
            q.n = rand() %% 4 ? rand() %% 40 : rand() %% 700;
            q.first = row;
            q.len = q.n + rand() %% 300;
            row += q.n;
        }
        const int64_t slots = (row + rand() %% 5) / kBlockTokens + 2ll * n;
        std::vector<std::vector<int>> times(n);
        for (int s = 0; s < n; ++s) times[s].assign(seqs[s].len / kBlockTokens + 1, 0);
        for (int64_t slot = 0; slot < slots; ++slot) {
            int s = 0;
            while (s + 1 < n && first_slot(seqs[s + 1].first, s + 1) <= slot) ++s;
            const int block = block_of_slot(seqs[s], s, slot);
            if (block == -1) continue;
            if (block < (seqs[s].len - seqs[s].n) / kBlockTokens || block * kBlockTokens >= seqs[s].len) return 1;
            ++times[s][block];
        }
        for (int s = 0; s < n; ++s)
            for (int block = 0; block * kBlockTokens < seqs[s].len; ++block)
                if (times[s][block] != (seqs[s].n > 0 && (block + 1) * kBlockTokens > seqs[s].len - seqs[s].n)) return 2;
    }
    return 0;
}
""" % seed)


def test_counts_up_to_31_bits(tmp_path):
    """Threads that share out up to 2^31 - 1 tokens or list entries take each of theirs once and end, where a signed counter would step past the largest number and begin
    again below zero."""
    run_pages_program(tmp_path, """
int main() {
    for (int count : {0, 1, 1023, 1024, 1025, 2147483647, 2147483646, 2147483647 - 1023, 2147483647 - 1024, 2147483647 - 1025, 2147483647 - 4096})
        for (int step : {1024, 4096})
            for (int first : {0, 1, 500, 1022, 1023}) {
                const int64_t all = first < count ? ((int64_t)count - first + step - 1) / step : 0;
                int64_t seen = 0, next = first;
                bool right = true;
                each_from(first, count, step, [&](uint32_t i) {
                    right &= (int64_t)i == next && next < count;
                    next += step;
                    if (++seen > all) { printf("%d from %d by %d does not end\\n", count, first, step); exit(1); }
                });
                if (!right || seen != all) { printf("%d from %d by %d: %ld of %ld\\n", count, first, step, (long)seen, (long)all); return 2; }
            }
    return 0;
}
""")
