// Attention of few new tokens a sequence (up to 64 rows: single tokens, drafts, short texts): a stream over the pages.
//
// Few rows make the products thin, so the kernel is bound by the bytes of K and V.  Every wave takes tiles of its own straight from memory into the
// operands of the 16x16x32 products, no LDS and no barrier between tiles; the next tile's K is asked for when this one's has been multiplied, V
// likewise, so that a tile (16 KB of 16-bit values) is always under way.
//
// The work of all sequences and K/V heads is one row of tiles, cut into equal stretches, one a block: whatever the lengths, all
// blocks have the same number of tiles, give or take one.  A block's stretch may end inside one pair of sequence and head and hold
// whole ones; its four waves split each such segment, meet in LDS, and leave a result (whole pairs) or a partial one, of which a block has
// at most two, at its ends.  The merge kernel joins a pair's partial results.
#pragma once

#include "pages_attn.h"

namespace sali {

namespace {

constexpr int kStreamWaves = 4;
constexpr int kStreamMinTiles = 4;          // of a block: one a wave
constexpr int stream_blocks(int sets) { return sets == 1 ? 768 : (sets == 2 ? 512 : 256); }        // that are resident at once

// A tile of 32 tokens as it lies in memory, a lane's share.  i = lane % 16, hh = lane / 16.
//   K as the A operand, 16 places of a block in rows: lane (place i, hh) has 8 values of its token a step
//   V as the A operand, 16 values of the head in rows: lane (value, hh) has tokens 8 (hh % 2) .. + 7 of block hh / 2
template <int kStore, int kDim>
struct StreamRaw;
template <int kDim>
struct StreamRaw<SALI_STORE_16, kDim> {
    u32x4 k[2][kDim / 32], v[kDim / 16];
};
template <int kDim>
struct StreamRaw<SALI_STORE_INT8, kDim> {
    u32x4 k[2][kDim / 64], v[kDim / 32];
    float ks[2][kDim / 64];
    Scales8 vs[kDim / 32];
};
template <int kDim>
struct StreamRaw<SALI_STORE_INT4, kDim> {
    u32x4 k[2];                             // head dim 64: half of it
    u32x2 v[kDim / 32];
    float ks[2];
    uint16_t kz[2];
    Scales8 vs[kDim / 32];
    u32x4 vz[kDim / 32];
};

template <int kStore, int kDim>
__device__ __forceinline__ void stream_load_k(const char* b0, const char* b1, int lane, StreamRaw<kStore, kDim>& r) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const char* b = j == 0 ? b0 : b1;
        if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
            for (int t = 0; t < kDim / 32; ++t) r.k[j][t] = load16(b + (uint32_t)(t * 1024 + lane * 16));
        } else if constexpr (kStore == SALI_STORE_INT8) {
#pragma unroll
            for (int u = 0; u < kDim / 64; ++u) {
                r.k[j][u] = load16(b + (uint32_t)(u * 1024 + lane * 16));
                r.ks[j][u] = *reinterpret_cast<const float*>(b + kAt.ks + (uint32_t)((2 * u + (lane >> 5)) * 64 + (lane & 15) * 4));
            }
        } else if constexpr (kDim == 128) {
            r.k[j] = load16(b + (uint32_t)(lane * 16));
            r.ks[j] = *reinterpret_cast<const float*>(b + kAt.ks + (uint32_t)(lane * 4));
            r.kz[j] = *reinterpret_cast<const uint16_t*>(b + kAt.kz + (uint32_t)(lane * 2));
        } else {
            const uint32_t at = (uint32_t)((lane >> 5) * 16 + (lane & 15));
            const u32x2 c = *reinterpret_cast<const u32x2*>(b + at * 16 + (uint32_t)(lane >> 4 & 1) * 8);
            r.k[j] = (u32x4){c.x, c.y, 0u, 0u};
            r.ks[j] = *reinterpret_cast<const float*>(b + kAt.ks + at * 4);
            r.kz[j] = *reinterpret_cast<const uint16_t*>(b + kAt.kz + at * 2);
        }
    }
}
template <int kStore, int kDim>
__device__ __forceinline__ void stream_load_v(const char* b0, const char* b1, int lane, StreamRaw<kStore, kDim>& r) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    const char* b = lane < 32 ? b0 : b1;
    const uint32_t i = lane & 15, a = lane >> 4 & 1;
    if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
        for (int f = 0; f < kDim / 16; ++f) r.v[f] = load16(b + kAt.v + (a * kDim + 16 * f + i) * 16);
    } else {
#pragma unroll
        for (int g = 0; g < kDim / 32; ++g) {
            if constexpr (kStore == SALI_STORE_INT8) r.v[g] = load16(b + kAt.v + (a * kDim + 32 * g + 2 * i) * 8);
            else r.v[g] = *reinterpret_cast<const u32x2*>(b + kAt.v + ((a * (kDim / 32) + g) * 16 + i) * 8);
            const f32x4* s = reinterpret_cast<const f32x4*>(b + kAt.vs + (g * 16 + 8 * a) * 4);
            r.vs[g] = {s[0], s[1]};
            if constexpr (kStore == SALI_STORE_INT4) r.vz[g] = load16(b + kAt.vz + (g * 16 + 8 * a) * 2);
        }
    }
}
// step t of a block's K
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ u32x4 stream_k(const StreamRaw<kStore, kDim>& r, int j, int t) {
    if constexpr (kStore == SALI_STORE_16) return r.k[j][t];
    else if constexpr (kStore == SALI_STORE_INT8) {
        const u32x4& c = r.k[j][t / 2];
        const uint32_t lo = t & 1 ? c.z : c.x, hi = t & 1 ? c.w : c.y;
        return values8<kBf16>(lo, hi, r.ks[j][t / 2]);
    } else {
        // bytes 0 .. 15 of a group (head dim 64: 8 of them): low halves first, then the high ones
        constexpr int kHalf = kDim / 64;
        const int part = t % kHalf, shift = t / kHalf * 4;
        const uint32_t lo = part ? r.k[j].z : r.k[j].x, hi = part ? r.k[j].w : r.k[j].y;
        return values4<kBf16>(lo >> shift & 0x0F0F0F0Fu, hi >> shift & 0x0F0F0F0Fu, r.ks[j], low_half<kBf16>(r.kz[j]));
    }
}
// first value of the head that step t of lane quarter hh multiplies
template <int kStore, int kDim>
__device__ __forceinline__ int stream_k_value(int t, int hh) {
    if constexpr (kStore == SALI_STORE_16) return 32 * t + 8 * hh;
    else if constexpr (kStore == SALI_STORE_INT8) return 64 * (t / 2) + 16 * hh + 8 * (t & 1);
    else if constexpr (kDim == 128) return 32 * hh + 8 * t;
    else return 32 * (hh >> 1) + 8 * (hh & 1) + 16 * t;
}
// product f of V, and the value of the head in its row i
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ u32x4 stream_v(const StreamRaw<kStore, kDim>& r, int f) {
    if constexpr (kStore == SALI_STORE_16) return r.v[f];
    else if constexpr (kStore == SALI_STORE_INT8) {
        const u32x4& c = r.v[f / 2];
        const uint32_t lo = f & 1 ? c.z : c.x, hi = f & 1 ? c.w : c.y;
        return values8<kBf16>(lo, hi, r.vs[f / 2]);
    } else {
        const int shift = (f & 1) * 4;
        const uint32_t lo = r.v[f / 2].x, hi = r.v[f / 2].y;
        return values4<kBf16>(lo >> shift & 0x0F0F0F0Fu, hi >> shift & 0x0F0F0F0Fu, r.vs[f / 2], r.vz[f / 2]);
    }
}
template <int kStore>
__device__ __forceinline__ int stream_v_value(int f, int i) {
    if constexpr (kStore == SALI_STORE_16) return 16 * f + i;
    else if constexpr (kStore == SALI_STORE_INT8) return 32 * (f / 2) + 2 * i + (f & 1);
    else return 16 * f + i;
}

__device__ __forceinline__ bool in_stream(const PageSeq& q, int group, int rows_max) { return q.n > 0 && (int64_t)q.n * group <= rows_max; }

// the record of a block whose last segment is a pair's first part; blocks without one leave parts = 0
struct StreamRecord {
    int32_t seq, head, slot, parts;         // slot of the first part; the others are the first segments of the following blocks
};

template <int kStore, int kDim, bool kBf16, int kSets>
__global__ __launch_bounds__(64 * kStreamWaves) void k_pages_stream(PagesAttend a, int rows_max, int min_tiles) {
    constexpr int kRows = 16 * kSets, kSteps = kDim / 32, kFs = kDim / 16, kPitch = kDim + 4;
    __shared__ __align__(16) float s_acc[kStreamWaves][kRows][kPitch];
    __shared__ float s_m[kStreamWaves][kRows], s_l[kStreamWaves][kRows];
    __shared__ int64_t s_sum[kStreamWaves];
    __shared__ int s_found;
    __shared__ int64_t s_before;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, hh = lane >> 4;
    const int n_kv = a.geom.n_kv, group = a.group;

    // ---- the block's stretch
    auto tiles_of_seq = [&](int s) -> int {
        const PageSeq q = load_seq(a.seqs, a.geom, s, blockIdx.x == 0);
        return in_stream(q, group, rows_max) ? view_of<kTileTokens>(q.len - q.n, q.len - 1, a.window, a.sinks).tiles : 0;
    };
    const int mine = (int)threadIdx.x < a.seqs.n_seqs ? tiles_of_seq(threadIdx.x) : 0;
    auto sum_block = [&](int64_t v) -> int64_t {            // inclusive over the block's threads; s_sum has the waves'
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t u = __shfl_up(v, off);
            if (lane >= off) v += u;
        }
        __syncthreads();
        if (lane == 63) s_sum[wave] = v;
        __syncthreads();
        for (int w = 0; w < wave; ++w) v += s_sum[w];
        return v;
    };
    int64_t own = mine;
    for (int s = (int)threadIdx.x + 256; s < a.seqs.n_seqs; s += 256) own += tiles_of_seq(s);
    int64_t upto = sum_block(own);
    const int64_t per_head = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3], total = per_head * n_kv;
    const int64_t blocks = max((int64_t)1, min((int64_t)gridDim.x, total / min_tiles));
    StreamRecord* records = reinterpret_cast<StreamRecord*>(a.records);
    StreamRecord record = {0, 0, 0, 0};
    int64_t at = 0, end = 0;
    if ((int64_t)blockIdx.x < blocks) {
        at = stretch_start(blockIdx.x, total, blocks);
        end = stretch_start((int64_t)blockIdx.x + 1, total, blocks);
    }
    if (at >= end) {
        if (threadIdx.x == 0) records[blockIdx.x] = record;
        return;
    }
    if (a.seqs.n_seqs <= 256) {
        if (at >= (upto - mine) * n_kv && at < upto * n_kv) {
            s_found = threadIdx.x;
            s_before = upto - mine;
        }
    } else {
        int64_t before = 0;
        for (int base = 0; base < a.seqs.n_seqs; base += 256) {
            const int s = base + (int)threadIdx.x, t = s < a.seqs.n_seqs ? tiles_of_seq(s) : 0;
            upto = before + sum_block(t);
            if (at >= (upto - t) * n_kv && at < upto * n_kv) {
                s_found = s;
                s_before = upto - t;
            }
            before += s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
            if (before * n_kv > at) break;
        }
    }
    __syncthreads();
    int s = __builtin_amdgcn_readfirstlane(s_found);
    PageSeq seq = load_seq(a.seqs, a.geom, s, false);
    View view = view_of<kTileTokens>(seq.len - seq.n, seq.len - 1, a.window, a.sinks);
    int head, done;                          // of the sequence: K/V head and its tiles before the block's
    {
        const int64_t off = at - s_before * n_kv;
        head = (int)(off / view.tiles);
        done = (int)(off - (int64_t)head * view.tiles);
    }

    bool first_segment = true;
    while (at < end) {
        const int todo = (int)min((int64_t)(view.tiles - done), end - at);
        const int rows = seq.n * group;
        const int32_t* table = a.seqs.table + (int64_t)s * a.seqs.width;
        const int pages = (seq.len + (kBlockTokens << a.geom.blocks_log2) - 1) / (kBlockTokens << a.geom.blocks_log2);
        const char* const heads = a.geom.pool + (uint64_t)head * a.geom.head_bytes;
        const uint32_t block_bytes = a.geom.head_bytes >> a.geom.blocks_log2;

        // the pages from `page0` on, one a lane
        int page0 = -64, page_of_lane = -1;
        struct Tile {
            const char* b[2];
            int live[2];                     // tokens of the block that a row may see: none of a page that is none
        };
        auto locate = [&](int i) -> Tile {
            Tile t;
            const int tile = tile_at(view, i);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int block = 2 * tile + j, index = block >> a.geom.blocks_log2;
                if ((unsigned)(index - page0) >= 64u) {
                    page0 = index;
                    page_of_lane = index + lane < pages ? table[index + lane] : -1;
                    asm volatile("" : "+v"(page_of_lane));      // waited for here: a wait behind the branch would be one for K and V too
                }
                int page = __builtin_amdgcn_readlane(page_of_lane, index - page0);
                t.live[j] = min(kBlockTokens, seq.len - block * kBlockTokens);
                if ((unsigned)page >= (unsigned)a.geom.n_pages) {
                    if (t.live[j] > 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                    t.live[j] = 0;
                    page = 0;
                }
                t.b[j] = heads + (uint64_t)page * a.geom.page_bytes + (uint32_t)(block & ((1 << a.geom.blocks_log2) - 1)) * block_bytes;
            }
            return t;
        };

        const int lo = done + (int)((int64_t)todo * wave / kStreamWaves), hi = done + (int)((int64_t)todo * (wave + 1) / kStreamWaves);
        StreamRaw<kStore, kDim> raw;
        Tile now = {};
        if (lo < hi) {
            now = locate(lo);
            stream_load_k<kStore, kDim>(now.b[0], now.b[1], lane, raw);
            stream_load_v<kStore, kDim>(now.b[0], now.b[1], lane, raw);
        }
        u32x4 q[kSets][kSteps];
        int pos[kSets];
#pragma unroll
        for (int c = 0; c < kSets; ++c) {
            const int r = 16 * c + col, token = r / group, g = r - token * group;
            pos[c] = r < rows ? view.first + token : -1;
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                q[c][t] = (u32x4){0u, 0u, 0u, 0u};
                if (r < rows) {
                    const u32x4 v = load16(a.q.d + (int64_t)(seq.first + token) * a.q.token_bytes + (int64_t)(head * group + g) * a.q.head_bytes +
                                           2 * stream_k_value<kStore, kDim>(t, hh));
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[c][t][e] = (v[e] & a.q_keep) ^ a.q_flip;
                }
            }
        }
        float m[kSets], l[kSets];
        f32x4 acc[kSets][kFs];
        uint32_t up[kSets], down[kSets];     // a bit for every value of acc: values that are not finite
#pragma unroll
        for (int c = 0; c < kSets; ++c) {
            m[c] = -INFINITY;
            l[c] = 0.0f;
            up[c] = down[c] = 0u;
#pragma unroll
            for (int f = 0; f < kFs; ++f) acc[c][f] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        }

        for (int i = lo; i < hi; ++i) {
            const int j0 = tile_at(view, i) * kTileTokens;
            const bool more = i + 1 < hi;
            const Tile next = more ? locate(i + 1) : now;
            f32x4 s2[kSets][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int c = 0; c < kSets; ++c) s2[c][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const u32x4 kf = stream_k<kStore, kDim, kBf16>(raw, j, t);
#pragma unroll
                    for (int c = 0; c < kSets; ++c) s2[c][j] = Num<kBf16>::mma16(kf, q[c][t], s2[c][j]);
                }
            }
            if (more) stream_load_k<kStore, kDim>(next.b[0], next.b[1], lane, raw);
            // lane (row col, hh): tokens 8 (hh % 2) + 4 (hh / 2) .. + 3 of each block
            const int t0 = j0 + 8 * (hh & 1) + 4 * (hh >> 1);
            const bool masked = now.live[0] < kBlockTokens || now.live[1] < kBlockTokens || partly_hidden(view, a.window, a.sinks, j0, kTileTokens);
            if (masked) {
#pragma unroll
                for (int c = 0; c < kSets; ++c)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (now.live[j] <= 0 || !sees(pos[c], t0 + 16 * j + r, a.window, a.sinks)) s2[c][j][r] = -INFINITY;
            }
            u32x4 p[kSets];
#pragma unroll
            for (int c = 0; c < kSets; ++c) {
                float top = fmaxf(fmaxf(fmaxf(s2[c][0][0], s2[c][0][1]), fmaxf(s2[c][0][2], s2[c][0][3])),
                                  fmaxf(fmaxf(s2[c][1][0], s2[c][1][1]), fmaxf(s2[c][1][2], s2[c][1][3])));
                top = max_over_quarters(top) * a.scale2;
                const float to = top > m[c] + kLag ? top : m[c];
                if (__builtin_amdgcn_ballot_w64(to != m[c]) != 0) {
                    const float by = to != m[c] ? __builtin_amdgcn_exp2f(m[c] - to) : 1.0f;
                    l[c] *= by;
#pragma unroll
                    for (int f = 0; f < kFs; ++f) acc[c][f] *= by;
                    m[c] = to;
                }
                const float ref = m[c] == -INFINITY ? 0.0f : m[c];
                uint32_t w[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float e[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s2[c][j][r], a.scale2, -ref));
                        l[c] += e[r];
                    }
                    w[j][0] = pack2<kBf16>(e[0], e[1]);
                    w[j][1] = pack2<kBf16>(e[2], e[3]);
                }
                // to the lanes that hold the same tokens of V: quarter hh takes tokens 8 (hh % 2) .. + 7 of block hh / 2
                const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                p[c] = (u32x4){(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
            }
            if (masked) {
                const int live = (hh < 2 ? now.live[0] : now.live[1]) - 8 * (hh & 1);
                if constexpr (kStore != SALI_STORE_16) {
#pragma unroll
                    for (int g = 0; g < kDim / 32; ++g) {
                        raw.vs[g] = live_tokens(raw.vs[g], live);
                        if constexpr (kStore == SALI_STORE_INT4) raw.vz[g] = live_tokens(raw.vz[g], live);
                    }
                } else {
                    bool odd = false;
#pragma unroll
                    for (int f = 0; f < kFs; ++f) {
                        raw.v[f] = live_tokens(raw.v[f], live);
                        odd |= any_not_finite<kBf16>(raw.v[f]);
                    }
                    if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                        u32x4 seen[kSets];
#pragma unroll
                        for (int c = 0; c < kSets; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int j = j0 + 16 * (hh >> 1) + 8 * (hh & 1) + 2 * e;
                                seen[c][e] = (2 * e < live && sees(pos[c], j, a.window, a.sinks) ? (uint32_t)Num<kBf16>::kOne : 0u) |
                                             (2 * e + 1 < live && sees(pos[c], j + 1, a.window, a.sinks) ? (uint32_t)Num<kBf16>::kOne << 16 : 0u);
                            }
                        // through the wave's part of LDS, one product at a time: this path is not to cost registers
                        u32x4* const mine = reinterpret_cast<u32x4*>(&s_acc[wave][0][0]) + lane;
                        static_assert(kFs * 1024 <= sizeof(s_acc[0]), "the operands of a tile's V");
#pragma unroll
                        for (int f = 0; f < kFs; ++f) mine[64 * f] = raw.v[f];
#pragma unroll 1
                        for (int f = 0; f < kFs; ++f) {
                            u32x4 finite, plus, minus;
                            take_apart<kBf16>(mine[64 * f], finite, plus, minus);
                            mine[64 * f] = finite;
#pragma unroll
                            for (int c = 0; c < kSets; ++c) {
                                const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                                const f32x4 ups = Num<kBf16>::mma16(plus, seen[c], zero), downs = Num<kBf16>::mma16(minus, seen[c], zero);
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    up[c] |= (ups[r] > 0.0f ? 1u << r : 0u) << (4 * f);
                                    down[c] |= (downs[r] > 0.0f ? 1u << r : 0u) << (4 * f);
                                }
                            }
                        }
#pragma unroll
                        for (int f = 0; f < kFs; ++f) raw.v[f] = mine[64 * f];
                    }
                }
            }
#pragma unroll
            for (int f = 0; f < kFs; ++f) {
                const u32x4 vf = stream_v<kStore, kDim, kBf16>(raw, f);
#pragma unroll
                for (int c = 0; c < kSets; ++c) acc[c][f] = Num<kBf16>::mma16(vf, p[c], acc[c][f]);
            }
            if (more) stream_load_v<kStore, kDim>(next.b[0], next.b[1], lane, raw);
            now = next;
        }

        // ---- the waves meet
#pragma unroll
        for (int c = 0; c < kSets; ++c) {
            const int r = 16 * c + col;
            const float sum = sum_over_quarters(l[c]);
            if (r >= rows) continue;
            if constexpr (kStore == SALI_STORE_16)
                if ((up[c] | down[c]) != 0)
#pragma unroll
                    for (int f = 0; f < kFs; ++f)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[c][f][e] += found((up[c] >> (4 * f + e) & 1) != 0, (down[c] >> (4 * f + e) & 1) != 0);
            if (hh == 0) {
                s_m[wave][r] = m[c];
                s_l[wave][r] = sum;
            }
#pragma unroll
            for (int f = 0; f < kFs; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_acc[wave][r][stream_v_value<kStore>(f, 4 * hh + e)] = acc[c][f][e];
        }
        __syncthreads();
        const bool whole = todo == view.tiles;
        const int slot = 2 * (int)blockIdx.x + (first_segment ? 0 : 1);
        for (int idx = threadIdx.x; idx < rows * (kDim / 4); idx += 64 * kStreamWaves) {
            const int r = idx / (kDim / 4), d = idx % (kDim / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) top = fmaxf(top, s_m[w][r]);
            float sum = 0.0f;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) {
                const float mw = s_m[w][r];
                if (s_l[w][r] == 0.0f) continue;
                const float by = __builtin_amdgcn_exp2f(mw - top);
                sum += s_l[w][r] * by;
                o += *reinterpret_cast<const f32x4*>(&s_acc[w][r][d]) * by;
            }
            if (!whole) {
                float* part = a.partial + ((size_t)slot * kRows + r) * kPitch;
                *reinterpret_cast<f32x4*>(part + 4 + d) = o;
                if (d == 0) {
                    part[0] = top;
                    part[1] = sum;
                }
                continue;
            }
            const int token = r / group, h = head * group + (r - token * group);
            const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
            const RowEnd e = row_end(top, sum, a, row);
            f32x4 pr = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.prior != nullptr) pr = *reinterpret_cast<const f32x4*>(a.prior + row * kDim + d);
            const u32x2 v = {pack2<kBf16>(joined(e, o[0], pr[0]), joined(e, o[1], pr[1])), pack2<kBf16>(joined(e, o[2], pr[2]), joined(e, o[3], pr[3]))};
            *reinterpret_cast<u32x2*>(a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes + (int64_t)h * a.out.head_bytes + 2 * d) = v;
            if (d == 0 && a.lse != nullptr) a.lse[row] = e.lse;
        }
        __syncthreads();

        if (!whole && done == 0) {                          // a pair's first part: the following blocks have the others
            const int64_t last = at + view.tiles - 1;
            record = {s, head, slot, (int)(stretch_of(last, total, blocks) - blockIdx.x) + 1};
        }
        at += todo;
        first_segment = false;
        done += todo;
        if (done == view.tiles && at < end) {
            done = 0;
            if (++head == n_kv) {
                head = 0;
                do {
                    if (++s >= a.seqs.n_seqs) break;
                    seq = load_seq(a.seqs, a.geom, s, false);
                } while (!in_stream(seq, group, rows_max));
                if (s >= a.seqs.n_seqs) break;
                view = view_of<kTileTokens>(seq.len - seq.n, seq.len - 1, a.window, a.sinks);
            }
        }
    }
    if (threadIdx.x == 0) records[blockIdx.x] = record;
}

// Joins the parts of a pair's row: grid (blocks of the stream, rows), four waves that share the parts.
template <int kDim, bool kBf16>
__global__ __launch_bounds__(256) void k_pages_stream_merge(PagesAttend a, int kernel_rows) {
    constexpr int kPitch = kDim + 4, kPer = kDim / 64;
    __shared__ float s_acc[4][kDim], s_m[4], s_l[4];
    const StreamRecord rec = reinterpret_cast<const StreamRecord*>(a.records)[blockIdx.x];
    if (rec.parts == 0) return;
    const PageSeq seq = load_seq(a.seqs, a.geom, rec.seq, false);
    const int r = blockIdx.y;
    if (r >= seq.n * a.group) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float m = -INFINITY, l = 0.0f, acc[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.0f;
#pragma unroll 4
    for (int i = wave; i < rec.parts; i += 4) {
        const int slot = i == 0 ? rec.slot : 2 * ((rec.slot >> 1) + i);
        const float* part = a.partial + ((size_t)slot * kernel_rows + r) * kPitch;
        const float pm = part[0], pl = part[1];
        float v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = part[4 + lane * kPer + e];
        const float to = fmaxf(m, pm);
        const float ref = to == -INFINITY ? 0.0f : to, by = __builtin_amdgcn_exp2f(m - ref), pby = __builtin_amdgcn_exp2f(pm - ref);
        if (pl == 0.0f) continue;               // nothing seen
        const bool none = l == 0.0f;
        l = (none ? 0.0f : l * by) + pl * pby;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = (none ? 0.0f : acc[e] * by) + v[e] * pby;
        m = to;
    }
    if (lane == 0) {
        s_m[wave] = m;
        s_l[wave] = l;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) s_acc[wave][lane * kPer + e] = acc[e];
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= kDim) return;
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float sum = 0.0f, o = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (s_l[w] == 0.0f) continue;
        const float by = __builtin_amdgcn_exp2f(s_m[w] - top);
        sum += s_l[w] * by;
        o += s_acc[w][d] * by;
    }
    const int token = r / a.group, h = rec.head * a.group + (r - token * a.group);
    const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
    const RowEnd e = row_end(top, sum, a, row);
    const float pr = a.prior != nullptr ? a.prior[row * kDim + d] : 0.0f;
    *reinterpret_cast<typename Num<kBf16>::T*>(a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes + (int64_t)h * a.out.head_bytes + 2 * d) =
        (typename Num<kBf16>::T)joined(e, o, pr);
    if (d == 0 && a.lse != nullptr) a.lse[row] = e.lse;
}

}  // namespace

}  // namespace sali
