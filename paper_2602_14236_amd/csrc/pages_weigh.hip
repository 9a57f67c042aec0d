// What attention weight keys had: for every key of a sequence and K/V head, the sum of exp(s - lse) over the new tokens that see it and the query heads of the group (gfx950).
//
// Rows, scores, masks and the layout of tiles are those of attention (pages_attn.h); with lse at hand there is no maximum to find, no second product and
// nothing to join: a wave has 32 keys, walks all rows that see them, sixteen at a time, and adds the weights up in fp32, always in the same order.
#include "pages_stream.h"

namespace sali {

namespace {

constexpr int kWeighWaves = kWeighTokens / kTileTokens;

// The tile's keys as the waves of the stream have them: lane (col, hh) has rows col and tokens 8 (hh % 2) + 4 (hh / 2) .. + 3 of each block
template <int kStore, int kDim, bool kBf16>
__global__ __launch_bounds__(64 * kWeighWaves) void k_pages_weigh(PagesWeigh a, int blocks) {
    constexpr int kSteps = kDim / 32;
    constexpr float kLog2e = 1.44269504088896340736f;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, hh = lane >> 4;
    const int head = (int)(blockIdx.x % (uint32_t)a.geom.n_kv), nth = (int)(blockIdx.x / (uint32_t)a.geom.n_kv), s = nth / blocks, nth_of_seq = nth - s * blocks;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, lane, 64);
    const PageSeq seq = load_seq(a.seqs, a.geom, s, nth_of_seq == 0 && head == 0 && threadIdx.x == 0);
    if (__builtin_amdgcn_ballot_w64(falls.some()) != 0) {
        if (threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    if (seq.n == 0) return;
    const int tile = nth_of_seq * kWeighWaves + wave, j0 = tile * kTileTokens;
    if ((int64_t)tile * kTileTokens >= seq.len) return;
    const int page_tokens = kBlockTokens << a.geom.blocks_log2, first = seq.len - seq.n;
    const char* b[2];
    float* w[2];                            // where the weights of each block lie; NULL: of a page that is none, or behind the sequence's end
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int block = 2 * tile + j;
        int page = 0;
        w[j] = nullptr;
        if (block * kBlockTokens < seq.len) {
            page = a.seqs.table[(int64_t)s * a.seqs.width + (block >> a.geom.blocks_log2)];
            if ((unsigned)page >= (unsigned)a.geom.n_pages) {
                if (lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                page = 0;
            } else {
                w[j] = a.weights + ((int64_t)page * a.geom.n_kv + head) * page_tokens + (block & ((1 << a.geom.blocks_log2) - 1)) * kBlockTokens;
            }
        }
        b[j] = a.geom.pool + (uint64_t)page * a.geom.page_bytes + (uint64_t)head * a.geom.head_bytes +
               (uint32_t)(block & ((1 << a.geom.blocks_log2) - 1)) * (a.geom.head_bytes >> a.geom.blocks_log2);
    }
    if (w[0] == nullptr && w[1] == nullptr) return;
    StreamRaw<kStore, kDim> raw;
    stream_load_k<kStore, kDim>(b[0], b[1], lane, raw);
    u32x4 k[2][kSteps];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int t = 0; t < kSteps; ++t) k[j][t] = stream_k<kStore, kDim, kBf16>(raw, j, t);

    f32x4 sum[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    const int rows = seq.n * a.group, first_key = j0 + 8 * (hh & 1) + 4 * (hh >> 1);
    // rows whose tokens see some of the tile: from the one at position j0 on, and under a window up to the last that the tile's last key is in the window of
    const int from = max(0, j0 - first) * a.group;
    int upto = rows;
    if (a.window > 0 && j0 >= a.sinks) upto = (int)max((int64_t)0, min((int64_t)rows, ((int64_t)j0 + kTileTokens - 1 + a.window - first) * a.group));
    for (int r0 = from & ~15; r0 < upto; r0 += 16) {
        const int r = r0 + col, token = r / a.group, g = r - token * a.group;
        u32x4 q[kSteps];
        float lse = -INFINITY;
#pragma unroll
        for (int t = 0; t < kSteps; ++t) q[t] = (u32x4){0u, 0u, 0u, 0u};
        if (r < rows) {
            const char* const at = a.q.d + (int64_t)(seq.first + token) * a.q.token_bytes + (int64_t)(head * a.group + g) * a.q.head_bytes;
            lse = a.lse[(int64_t)(seq.first + token) * a.heads + head * a.group + g];
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const u32x4 v = load16(at + 2 * stream_k_value<kStore, kDim>(t, hh));
#pragma unroll
                for (int e = 0; e < 4; ++e) q[t][e] = (v[e] & a.q_keep) ^ a.q_flip;
            }
        }
        const bool some = lse != -INFINITY;  // a row that saw nothing has no weights
        const float lse2 = lse * kLog2e;
        const Sight sight = sight_of(first + token, first_key, a.window, a.sinks);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) x = Num<kBf16>::mma16(k[j][t], q[t], x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (some && sight.has(16 * j + e)) sum[j][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], a.scale2, -lse2));
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) sum[j][e] += __shfl_xor(sum[j][e], off);
    if (col == 0)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = first_key + 16 * j + e;
                if (w[j] == nullptr || at >= seq.len) continue;
                float* const to = w[j] + (at & 15);
                *to = a.add && at < first ? *to + sum[j][e] : sum[j][e];
            }
}

}  // namespace

hipError_t launch_pages_weigh(int dtype, int store, int dim, const PagesWeigh& a, hipStream_t s) {
    const int blocks = (int)weigh_blocks(a.seqs);
    const dim3 grid((unsigned)((int64_t)blocks * a.geom.n_kv * a.seqs.n_seqs));
    auto go = [&](auto st, auto d) {
        if (dtype == SALI_DTYPE_BF16) hipLaunchKernelGGL((k_pages_weigh<decltype(st)::value, decltype(d)::value, true>), grid, dim3(64 * kWeighWaves), 0, s, a, blocks);
        else hipLaunchKernelGGL((k_pages_weigh<decltype(st)::value, decltype(d)::value, false>), grid, dim3(64 * kWeighWaves), 0, s, a, blocks);
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
