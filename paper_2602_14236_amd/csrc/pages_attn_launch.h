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
    // Rows of a sequence that the stream takes at most.  In a batch that has longer sequences: those of single tokens.
    int stream_rows = most_rows <= 16 ? 16 : 32;
    if (most_rows > 32) stream_rows = a.seqs.n_seqs == 1 || group > 32 ? 0 : (group <= 16 ? 16 : 32);
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
        auto go = [&](auto waves) {
            constexpr int kWaves = decltype(waves)::value;
            const int64_t units = tile_slots(a.seqs.n_tokens, group, a.seqs.n_seqs, tile_rows(kWaves)) + tile_parts(n_kv, kWaves);
            hipLaunchKernelGGL((k_pages_plan<kWaves>), dim3(1), dim3(kPlanThreads), 0, s, a, stream_rows + 1);
            hipLaunchKernelGGL((k_pages_tile<kStore, kDim, kBf16, kWaves>), dim3((unsigned)(units * n_kv)), dim3(64 * kWaves), 0, s, a);
            hipLaunchKernelGGL((k_pages_tile_merge<kDim, kBf16, kWaves>), dim3(tile_parts(n_kv, kWaves) / 2 * n_kv, tile_rows(kWaves) / 8), dim3(256), 0, s, a);
        };
        // (twelve waves of 4-bit rows of 128 values have too few registers)
        if constexpr (kStore != SALI_STORE_INT4 || kDim == 64)
            if (most_rows >= tile_rows(12) && (int64_t)a.seqs.n_tokens * group / tile_rows(12) * n_kv >= (kStore == SALI_STORE_16 ? 2 : 1) * kComputeUnits) {
                go(std::integral_constant<int, 12>{});
                return;
            }
        go(std::integral_constant<int, 4>{});
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
