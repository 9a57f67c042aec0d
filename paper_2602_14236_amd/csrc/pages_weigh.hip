// Which kernels a call that sums attention weights takes, and its launches; the kernels stand in pages_weigh.h.
#include "pages_weigh.h"

namespace sali {

namespace {

template <int kStore, int kDim, bool kBf16>
void launch_weigh(const PagesWeigh& a, hipStream_t s) {
    const int64_t most_rows = (int64_t)a.seqs.max_q * a.group, lines = (int64_t)a.geom.n_kv * a.seqs.n_seqs;
    if (most_rows <= 32) {
        // Tiles of a wave: as many as leave 32 waves a compute unit (16 ragged sequences of up to 8192 keys in 8 bits: 24.2 us, with 16 waves 25.7, with 64 25.1), and no
        // more pages than a wave has lanes.
        const int64_t tiles = ((int64_t)a.seqs.max_kv + kTileTokens - 1) / kTileTokens;
        const int each = (int)min((int64_t)8, (tiles * lines + kComputeUnits * 32 - 1) / (kComputeUnits * 32));
        const int blocks = (int)((tiles + each * kWeighStreamWaves - 1) / (each * kWeighStreamWaves));
        const dim3 grid((unsigned)(blocks * lines));
        if (most_rows <= 16) hipLaunchKernelGGL((k_pages_weigh_stream<kStore, kDim, kBf16, 1>), grid, dim3(64 * kWeighStreamWaves), 0, s, a, blocks, each);
        else hipLaunchKernelGGL((k_pages_weigh_stream<kStore, kDim, kBf16, 2>), grid, dim3(64 * kWeighStreamWaves), 0, s, a, blocks, each);
        return;
    }
    const int padded = weigh_padded(a.group);
    const int64_t steps = ((int64_t)a.seqs.max_q * padded + kWeighRows - 1) / kWeighRows;
    auto by_kind = [&](auto launch) {
        if (a.group > kWeighRows) launch(std::integral_constant<WeighRows, WeighRows::wide>{});
        else if (padded != a.group) launch(std::integral_constant<WeighRows, WeighRows::filled>{});
        else launch(std::integral_constant<WeighRows, WeighRows::even>{});
    };
    if (steps <= kWeighFewSteps) {
        const int64_t tiles = ((int64_t)a.seqs.max_kv + kTileTokens - 1) / kTileTokens;
        // a round of three blocks a compute unit (32 new of 20001 tokens, 2 sequences in 4 bits: 21.6 us, two rounds 22.8, four 24.3)
        const int each = (int)min((int64_t)16, (tiles * lines + kComputeUnits * 3 * kWeighFewWaves - 1) / (kComputeUnits * 3 * kWeighFewWaves));
        const int blocks = (int)((tiles + each * kWeighFewWaves - 1) / (each * kWeighFewWaves));
        by_kind([&](auto kind) {
            hipLaunchKernelGGL((k_pages_weigh_few<kStore, kDim, kBf16, decltype(kind)::value>), dim3((unsigned)(blocks * lines)), dim3(64 * kWeighFewWaves),
                               (unsigned)(steps * (WeighLayout<kDim>::kBytes + 4 * kWeighRows)), s, a, blocks, each, (int)steps);
        });
        return;
    }
    const int64_t blocks = ((int64_t)a.seqs.max_kv + kWeighKeys - 1) / kWeighKeys, units = blocks * lines;
    // rows in chunks where keys alone are too few blocks: sixteen a compute unit, of 256 rows at least, as far as there is room for their sums
    int64_t chunks = max((int64_t)1, min((16 * kComputeUnits + units - 1) / units, steps / 4));
    chunks = max((int64_t)1, min(chunks, (int64_t)(a.partial_bytes / (units * kWeighKeys * sizeof(float)))));
    const int chunk_steps = (int)((steps + chunks - 1) / chunks);
    chunks = (steps + chunk_steps - 1) / chunk_steps;
    by_kind([&](auto kind) {
        hipLaunchKernelGGL((k_pages_weigh_tile<kStore, kDim, kBf16, decltype(kind)::value>), dim3((unsigned)(units * chunks)), dim3(64 * kWeighWaves), 0, s, a, (int)blocks,
                           (int)chunks, chunk_steps);
    });
    if (chunks > 1) hipLaunchKernelGGL(k_pages_weigh_merge, dim3((unsigned)units), dim3(kWeighKeys / 4), 0, s, a, (int)blocks, (int)chunks);
}

}  // namespace

hipError_t launch_pages_weigh(int dtype, int store, int dim, const PagesWeigh& a, hipStream_t s) {
    auto go = [&](auto st, auto d) {
        if (dtype == SALI_DTYPE_BF16) launch_weigh<decltype(st)::value, decltype(d)::value, true>(a, s);
        else launch_weigh<decltype(st)::value, decltype(d)::value, false>(a, s);
    };
    auto with_dim = [&](auto st) {
        if (dim == 64) go(st, std::integral_constant<int, 64>{});
        else go(st, std::integral_constant<int, 128>{});
    };
    if (store == SALI_STORE_16) with_dim(std::integral_constant<int, SALI_STORE_16>{});
    else if (store == SALI_STORE_INT8) with_dim(std::integral_constant<int, SALI_STORE_INT8>{});
    else with_dim(std::integral_constant<int, SALI_STORE_INT4>{});
    return hipGetLastError();
}

}  // namespace sali
