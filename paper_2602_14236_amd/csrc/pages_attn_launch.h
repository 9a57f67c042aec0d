// Which kernels a call of paged attention takes, and its launches, for one 16-bit type.
#pragma once

#include "pages_stream.h"
#include "pages_tile.h"

namespace sali {

namespace {

// Rows are taken 384 a block where that gives so many blocks, two rounds of one a compute unit, else 128.
constexpr int kLargeBlocks = 2 * kComputeUnits;

template <int kStore, int kDim, bool kBf16>
void launch_attend(const PagesAttend& a, hipStream_t s) {
    const int n_kv = a.geom.n_kv, group = a.group;
    const int64_t most_rows = (int64_t)a.seqs.max_q * group;
    // Rows of a sequence that the stream takes at most.  In a batch that has longer sequences: those of single tokens.  (Up to 32 rows against the tiles' 128, us:
    // 32 rows over 8192 keys, 8 heads, 40 and 70; 24 over 512, 32 heads, 14 and 26; 32 over 4096, 32 heads, 47 and 38.)
    int stream_rows = most_rows <= 16 ? 16 : 32;
    if (most_rows > 32) {
        stream_rows = group <= 16 ? 16 : 32;
        // None if the batch has no such sequence as far as its sizes tell (one of them would leave the batch short of so many tokens; if there is one all the
        // same, because rows past the batch were counted, it is the tiles').  Two chunks of 1024 tokens under a window: 85 us, with the stream's empty launches 89.
        const int64_t short_of = (int64_t)a.seqs.n_seqs * a.seqs.max_q - a.seqs.n_tokens;
        if (a.seqs.n_seqs == 1 || group > 32 || short_of < a.seqs.max_q - stream_rows / group) stream_rows = 0;
    }
    if (stream_rows > 0) {
        const int64_t reach = a.window > 0 ? (int64_t)a.window + a.seqs.max_q + a.sinks + 3 * kTileTokens : (int64_t)a.seqs.max_kv + kTileTokens;
        const int64_t tiles = min((int64_t)a.seqs.max_kv + kTileTokens, reach) / kTileTokens * a.seqs.n_seqs * n_kv;
        const PageSeqs& q = a.seqs;
        auto go = [&](auto sets) {
            constexpr int kSets = decltype(sets)::value;
            auto launch = [&](auto mode, dim3 grid) {
                hipLaunchKernelGGL((k_pages_stream<kStore, kDim, kBf16, kSets, decltype(mode)::value>), grid, dim3(64 * stream_waves(decltype(mode)::value)), 0, s, q.start, q.length,
                                   q.table, q.n_seqs, q.width, q.n_tokens, q.max_q, q.max_kv, a.geom.blocks_log2, a.window, a.sinks, group, n_kv, a,
                                   stream_rows, kStreamMinTiles);
            };
            const int64_t pairs = (int64_t)q.n_seqs * n_kv, tiles_a_pair = tiles / pairs;
            if (tiles_a_pair <= 4 * stream_waves(StreamMode::pairs) && pairs <= kComputeUnits) {
                launch(std::integral_constant<StreamMode, StreamMode::pairs>{}, dim3(n_kv, q.n_seqs));
                return;
            }
            const int blocks = (int)max((int64_t)1, min((int64_t)kComputeUnits * stream_occupancy(kStore, kSets, StreamMode::stretches), (tiles + kStreamMinTiles - 1) / kStreamMinTiles));
            const int rows = (int)min((int64_t)stream_rows, most_rows);
            launch(std::integral_constant<StreamMode, StreamMode::stretches>{}, dim3(blocks));
            hipLaunchKernelGGL((k_pages_stream_merge<kDim, kBf16>), dim3(blocks, (rows + 3) / 4), dim3(256), 0, s, a, 16 * kSets);
        };
        if (stream_rows == 16) go(std::integral_constant<int, 1>{});
        else go(std::integral_constant<int, 2>{});
    }
    if (most_rows > 32) {
        auto go = [&](auto waves, int stretches) {
            constexpr int kWaves = decltype(waves)::value;
            const int64_t blocks = stretches > 0 ? stretches : tile_slots(a.seqs.n_tokens, group, a.seqs.n_seqs, tile_rows(kWaves)) + tile_parts(n_kv, kWaves);
            const int merges = stretches > 0 ? stretches : tile_parts(n_kv, kWaves) / 2;
            if (kWaves == 12 && stretches > 0) hipLaunchKernelGGL((k_pages_plan_stretches<12>), dim3(1), dim3(kPlanThreads), 0, s, a, stream_rows + 1, stretches);
            else hipLaunchKernelGGL((k_pages_plan_shares<kWaves>), dim3(1), dim3(kPlanThreads), 0, s, a, stream_rows + 1);
            hipLaunchKernelGGL((k_pages_tile<kStore, kDim, kBf16, kWaves>), dim3((unsigned)(blocks * n_kv)), dim3(64 * kWaves), 0, s, a);
            hipLaunchKernelGGL((k_pages_tile_merge<kDim, kBf16, kWaves>), dim3(merges * n_kv, kWaves * (kDim / 32) / 4), dim3(256), 0, s, a);
        };
        // Three ways, by how many blocks of 384 rows there are and how many tiles of 96 keys each sees (us, this one against the next best):
        //   few blocks of many tiles   stretches, since whole ones would leave most of the chip idle and cut ones end at different times.  Not for
        //                              short ones: the partial results at the ends of 256 stretches take 20 to 40.  Where the two meet was measured over 500
        //                              batches: chunks of 128 to 2048 tokens, 8 and 32 K/V heads, histories of 1000 to 9000, and windows of as many, which
        //                              leave the shorter tiles an even share.  Stretches and 128 rows in shares, 32 heads over 8, 16 bits: 512 new of 2000
        //                              tokens 56.4 and 51.8, of 2500 55.6 and 56.7, of 3600 67 and 69; 2048 of 2500 102 and 95, of 3000 111 and 116, of
        //                              3600 132 and 141; 2048 of 9000 under a window of 2500 141 and 134, of 4096 201 and 201, of 6000 274 and 282.  And how many
        //                              row tiles a block, of 144 more: 0.78 (2400 of 7000 tokens) 264 and 312, 0.88 (2700) 355 and 324, 0.97 (3000)
        //                              358 and 340; over 8 bits and 64 values too 0.78 18 % apart, 0.88 and 0.97 1 to 2
        //   two rounds of blocks       384 rows in shares.  16 bits: 8192 new ones 582, with 128 rows 628; 4096 (1.3 rounds) 206 and 199.
        //                              Quantised from one round on, since a key is dequantised a third as often: 4096 206 and 219, 2048 95 and 89
        //   else                       128 rows in shares
        // (Twelve waves of 4-bit rows of 128 values have too few registers.)
        if constexpr (kStore != SALI_STORE_INT4 || kDim == 64) {
            const int64_t reach = a.window > 0 ? min((int64_t)a.seqs.max_kv, (int64_t)a.window + a.sinks) : (int64_t)a.seqs.max_kv - a.seqs.max_q / 2;
            const int64_t rows = (int64_t)a.seqs.n_tokens * group, units = rows / tile_rows(12), tiles = reach / tile_keys(12), blocks = stretch_blocks(kComputeUnits, n_kv);
            if (most_rows >= tile_rows(12) && 10 * units <= 8 * blocks && 2 * (tiles - 12) * rows >= (a.window > 0 ? 18 : 5) * blocks * tile_rows(12)) {
                go(std::integral_constant<int, 12>{}, (int)blocks);
                return;
            }
            if (most_rows >= tile_rows(12) && units * n_kv >= (kStore == SALI_STORE_16 ? 2 : 1) * kComputeUnits) {
                go(std::integral_constant<int, 12>{}, 0);
                return;
            }
        }
        go(std::integral_constant<int, 4>{}, 0);
    }
}

template <bool kBf16>
hipError_t launch_pages_attend(int store, int dim, const PagesAttend& a, hipStream_t s) {
    auto with_dim = [&](auto st) {
        if (dim == 64) launch_attend<decltype(st)::value, 64, kBf16>(a, s);
        else launch_attend<decltype(st)::value, 128, kBf16>(a, s);
    };
    if (store == SALI_STORE_16) with_dim(std::integral_constant<int, SALI_STORE_16>{});
    else if (store == SALI_STORE_INT8) with_dim(std::integral_constant<int, SALI_STORE_INT8>{});
    else with_dim(std::integral_constant<int, SALI_STORE_INT4>{});
    return hipGetLastError();
}

}  // namespace

}  // namespace sali
