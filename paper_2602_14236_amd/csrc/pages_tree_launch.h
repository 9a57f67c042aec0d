// Which kernels a call of paged attention of drafted tokens takes, and its launches, for one 16-bit type.
//
// A draft is a causal text but for its last keys: all of its rows see the whole history, and of the draft what their masks name.  So the kernels are those of
// causal attention with another look at the keys from the history's end on (at most four tiles of 32), and without what only windows need.
//
// Up to 32 rows (new tokens times heads of a group) go through the stream, a launch's chain of trips where there is little history: 7 tokens of 4 heads over 777 keys, 14.4 us.
// More are row tiles of 128, four waves of 32 rows: 24 drafts of 16 tokens over up to 6000 keys in 8 bits, 8 heads, plan 6, tiles 77, merge 7 us, 190 MB at 2.5 TB/s; 4 of 64
// tokens over up to 9000 in 16 bits 6 + 58 + 13.  What bounds them is a tile's chain of load, first product, softmax and second product with three blocks a compute unit to hide it
// (64 and 128 rows give the matrix cores little: 16 and 26 % busy).  Weights are two 16-bit numbers each; with one the tiles take 64 and 49 us, and results
// are off by 2.3e-3 instead of 1.7e-3 in bfloat16.  Slower, the whole call with one number a weight, 75 us for the first as it is: 64 rows in the stream, 136; kernels of eight waves that take keys
// straight into registers, 122, or through a ring of four tiles in LDS, 115; tiles of two waves, 82, or twelve, 118; 384 or 768 shares instead of 512, 83.
#pragma once

#include "pages_attn_launch.h"

namespace sali {

namespace {

template <int kStore, int kDim, bool kBf16>
void launch_tree(const PagesAttend& a, hipStream_t s) {
    const int n_kv = a.geom.n_kv, group = a.group;
    const int64_t most_rows = (int64_t)a.seqs.max_q * group;
    int stream_rows = most_rows <= 16 ? 16 : 32;
    if (most_rows > 32) {
        // none if the batch has no draft of so few rows as far as its sizes tell
        const int64_t short_of = (int64_t)a.seqs.n_seqs * a.seqs.max_q - a.seqs.n_tokens;
        if (a.seqs.n_seqs == 1 || group > 32 || short_of < a.seqs.max_q - 32 / group) stream_rows = 0;
    }
    const int64_t reach = (int64_t)a.seqs.max_kv + kTileTokens;
    if (stream_rows == 16) launch_stream<kStore, kDim, kBf16, 1, true>(a, 16, reach, s);
    else if (stream_rows == 32) launch_stream<kStore, kDim, kBf16, 2, true>(a, 32, reach, s);
    if (most_rows <= 32) return;
    const int64_t blocks = tile_slots(a.seqs.n_tokens, group, a.seqs.n_seqs, tile_rows(4)) + tile_parts(n_kv, 4);
    hipLaunchKernelGGL((k_pages_plan_shares<4, true>), dim3(1), dim3(kPlanThreads), 0, s, a, stream_rows + 1);
    hipLaunchKernelGGL((k_pages_tile<kStore, kDim, kBf16, 4, true>), dim3((unsigned)(blocks * n_kv)), dim3(64 * 4), 0, s, a);
    hipLaunchKernelGGL((k_pages_tile_merge<kDim, kBf16, 4>), dim3(tile_parts(n_kv, 4) / 2 * n_kv, 4 * (kDim / 32) / 4), dim3(256), 0, s, a);
}

template <bool kBf16>
hipError_t launch_pages_attend_tree(int store, int dim, const PagesAttend& a, hipStream_t s) {
    auto with_dim = [&](auto st) {
        if (dim == 64) launch_tree<decltype(st)::value, 64, kBf16>(a, s);
        else launch_tree<decltype(st)::value, 128, kBf16>(a, s);
    };
    if (store == SALI_STORE_16) with_dim(std::integral_constant<int, SALI_STORE_16>{});
    else if (store == SALI_STORE_INT8) with_dim(std::integral_constant<int, SALI_STORE_INT8>{});
    else with_dim(std::integral_constant<int, SALI_STORE_INT4>{});
    return hipGetLastError();
}

}  // namespace

}  // namespace sali
