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
constexpr int stream_occupancy(int sets) { return sets == 1 ? 3 : (sets == 2 ? 2 : 1); }           // waves a SIMD: what their registers leave room for
constexpr int kStreamMostBlocks = 256 * 3;
constexpr int stream_blocks(int sets) { return 256 * stream_occupancy(sets); }                      // that are resident at once

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

// sums over the lanes up to each
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // row_bcast 15, 31
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
    return v;
}

// The parts of a pair, as a block or a launch that joins them finds them: the first in `slot`, the others the first segments of the following
// blocks.  A block leaves a record of the pair whose first part is its last segment, parts = 0 if there is none.
struct StreamRecord {
    int32_t seq, head, slot, parts;
};
__device__ __forceinline__ int slot_of_part(const StreamRecord& r, int i) { return i == 0 ? r.slot : 2 * ((r.slot >> 1) + i); }

// Partial results are handed over past the caches that the compute dies do not share: agent-scope accesses, coherent by themselves, so that no
// fence is needed; a block counts itself in when its own have arrived.
__device__ __forceinline__ void put_pair(float* p, float a, float b) {
    const uint64_t v = (uint64_t)__builtin_bit_cast(uint32_t, a) | (uint64_t)__builtin_bit_cast(uint32_t, b) << 32;
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void get_pair(const float* p, float& a, float& b) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a = __builtin_bit_cast(float, (uint32_t)v);
    b = __builtin_bit_cast(float, (uint32_t)(v >> 32));
}

// Rows r0, r0 + step, ... of a pair from its parts, by a block of 256 threads: the parts' references and sums give their weights (a wave a row),
// then a thread takes two values of a row, sixteen parts in flight.  s_weight: [rows][kMostParts], s_sum [rows].
template <int kDim, bool kBf16, int kMostParts>
__device__ __forceinline__ void join_parts(const PagesAttend& a, const StreamRecord& rec, const PageSeq& seq, int kernel_rows, int r0, int n_rows,
                                           float (*s_weight)[kMostParts], float* s_top, float* s_sum) {
    constexpr int kPitch = kDim + 4;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int x = wave; x < n_rows; x += 4) {
        float top = -INFINITY, sum = 0.0f;
        float m[kMostParts / 64], l[kMostParts / 64];
#pragma unroll
        for (int j = 0; j < kMostParts / 64; ++j) {
            m[j] = -INFINITY;
            l[j] = 0.0f;
            const int i = 64 * j + lane;
            if (i < rec.parts) get_pair(a.partial + ((size_t)slot_of_part(rec, i) * kernel_rows + r0 + x) * kPitch, m[j], l[j]);
        }
#pragma unroll
        for (int j = 0; j < kMostParts / 64; ++j)
            if (l[j] != 0.0f) top = fmaxf(top, m[j]);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
#pragma unroll
        for (int j = 0; j < kMostParts / 64; ++j) {
            const float w = l[j] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m[j] - top);
            sum += l[j] == 0.0f ? 0.0f : l[j] * w;
            s_weight[x][64 * j + lane] = w;
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
        if (lane == 0) {
            s_top[x] = top;
            s_sum[x] = sum;
        }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < n_rows * (kDim / 2); idx += 256) {
        const int x = idx / (kDim / 2), d = idx % (kDim / 2) * 2, r = r0 + x;
        float o0 = 0.0f, o1 = 0.0f;
        for (int i0 = 0; i0 < rec.parts; i0 += 16) {
            float v0[16], v1[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                get_pair(a.partial + ((size_t)slot_of_part(rec, min(i0 + i, rec.parts - 1)) * kernel_rows + r) * kPitch + 4 + d, v0[i], v1[i]);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = i0 + i < rec.parts ? s_weight[x][i0 + i] : 0.0f;
                if (w == 0.0f) continue;                    // nothing seen, or nothing left of it
                o0 = __builtin_fmaf(v0[i], w, o0);
                o1 = __builtin_fmaf(v1[i], w, o1);
            }
        }
        const int token = r / a.group, h = rec.head * a.group + (r - token * a.group);
        const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
        const RowEnd e = row_end(s_top[x], s_sum[x], a, row);
        float p0 = 0.0f, p1 = 0.0f;
        if (a.prior != nullptr) {
            p0 = a.prior[row * kDim + d];
            p1 = a.prior[row * kDim + d + 1];
        }
        *reinterpret_cast<uint32_t*>(a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes + (int64_t)h * a.out.head_bytes + 2 * d) =
            pack2<kBf16>(joined(e, o0, p0), joined(e, o1, p1));
        if (d == 0 && a.lse != nullptr) a.lse[row] = e.lse;
    }
}

// kMerged: the last block of a pair to finish joins its parts; else a launch of its own does (k_pages_stream_merge)
template <int kStore, int kDim, bool kBf16, int kSets, bool kMerged>
__global__ __launch_bounds__(64 * kStreamWaves) __attribute__((amdgpu_waves_per_eu(stream_occupancy(kSets), stream_occupancy(kSets)))) void k_pages_stream(
    PagesAttend a, int rows_max, int min_tiles) {
    constexpr int kRows = 16 * kSets, kSteps = kDim / 32, kFs = kDim / 16, kPitch = kDim + 4;
    __shared__ __align__(16) float s_acc[kStreamWaves][kRows][kPitch];
    __shared__ float s_m[kStreamWaves][kRows], s_l[kStreamWaves][kRows];
    __shared__ int s_last;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, hh = lane >> 4;
    const int n_kv = a.geom.n_kv, group = a.group;

    // ---- the block's stretch: every wave finds it by itself, a sequence a lane
    bool bad = false;
    auto lane_seq = [&](int s) -> PageSeq {
        PageSeq q = {0, 0, 0};
        if (s >= a.seqs.n_seqs) return q;
        bool fits;
        q = read_seq(a.seqs, a.geom, s, fits);
        bad |= !fits;
        return q;
    };
    auto tiles_of = [&](const PageSeq& q) { return in_stream(q, group, rows_max) ? view_of<kTileTokens>(q.len - q.n, q.len - 1, a.window, a.sinks).tiles : 0; };
    const PageSeq first_mine = lane_seq(lane);
    const int first_tiles = tiles_of(first_mine);
    int own = first_tiles;
#pragma unroll 4
    for (int s = 64 + lane; s < a.seqs.n_seqs; s += 64) own += tiles_of(lane_seq(s));
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane(wave_scan(own), 63) * (uint32_t)n_kv;
    if (bad && blockIdx.x == 0 && wave == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
    const uint32_t blocks = max(1u, min(gridDim.x, total / (uint32_t)min_tiles));
    StreamRecord* records = reinterpret_cast<StreamRecord*>(a.records);
    StreamRecord record = {0, 0, 0, 0};
    if (blockIdx.x >= blocks || total == 0) {
        if (!kMerged && threadIdx.x == 0) records[blockIdx.x] = record;
        return;
    }
    const Stretches cut(total, blocks);
    uint32_t at = __builtin_amdgcn_readfirstlane(cut.start(blockIdx.x));
    const uint32_t end = __builtin_amdgcn_readfirstlane(cut.start(blockIdx.x + 1));
    int s = 0;
    PageSeq seq = {0, 0, 0};
    uint32_t before = 0;                    // tiles a head of the sequences before it
    {
        PageSeq q = first_mine;
        int t = first_tiles;
        for (int base = 0;;) {
            const int upto = wave_scan(t);
            const uint64_t past = __builtin_amdgcn_ballot_w64((before + (uint32_t)upto) * (uint32_t)n_kv > at);
            if (past != 0) {
                const int k = __builtin_ctzll(past);
                s = base + k;
                seq = {__builtin_amdgcn_readlane(q.first, k), __builtin_amdgcn_readlane(q.n, k), __builtin_amdgcn_readlane(q.len, k)};
                before += (uint32_t)(__builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(t, k));
                break;
            }
            before += (uint32_t)__builtin_amdgcn_readlane(upto, 63);
            base += 64;
            if (base >= a.seqs.n_seqs) return;              // the batch changed while it was read
            q = lane_seq(base + lane);
            t = tiles_of(q);
        }
    }
    View view = view_of<kTileTokens>(seq.len - seq.n, seq.len - 1, a.window, a.sinks);
    int head = __builtin_amdgcn_readfirstlane((int)((at - before * (uint32_t)n_kv) / (uint32_t)view.tiles));
    int done = (int)(at - before * (uint32_t)n_kv) - head * view.tiles;         // tiles of the pair before the block's

    bool first_segment = true;
    while (at < end) {
        const int todo = min(view.tiles - done, (int)(end - at));
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

        const int lo = done + (int)((uint32_t)todo / kStreamWaves) * wave + min(wave, todo % kStreamWaves);
        const int hi = lo + (int)((uint32_t)todo / kStreamWaves) + (wave < todo % kStreamWaves ? 1 : 0);
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
            // behind the last tile the same once more, for nothing: with loads that depend on a branch every wait would be one for all of them
            const Tile next = locate(min(i + 1, hi - 1));
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
            stream_load_k<kStore, kDim>(next.b[0], next.b[1], lane, raw);
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
            stream_load_v<kStore, kDim>(next.b[0], next.b[1], lane, raw);
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
                put_pair(part + 4 + d, o[0], o[1]);
                put_pair(part + 6 + d, o[2], o[3]);
                if (d == 0) put_pair(part, top, sum);
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
        if (!whole) {
            // the pair's first part is in the block whose stretch has its first tile; that is its last segment, and its only one if it starts there
            const uint32_t pair0 = at - (uint32_t)done, b0 = __builtin_amdgcn_readfirstlane(cut.of(pair0)), b1 = __builtin_amdgcn_readfirstlane(cut.of(pair0 + (uint32_t)view.tiles - 1u));
            const StreamRecord pair = {s, head, (int)(2 * b0 + (cut.start(b0) == pair0 ? 0u : 1u)), (int)(b1 - b0) + 1};
            if constexpr (kMerged) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // every wave: its parts have arrived
                __syncthreads();
                if (threadIdx.x == 0)
                    s_last = last_arrival(atomicInc(a.arrived + (size_t)b0 * kMergeParts + (pair.parts - 1), (uint32_t)pair.parts - 1u), pair.parts) ? 1 : 0;
                __syncthreads();
                if (s_last != 0) {
                    static_assert(sizeof(float[kRows][kMergeParts]) <= sizeof(s_acc), "the weights of the parts");
                    join_parts<kDim, kBf16, kMergeParts>(a, pair, seq, kRows, 0, rows, reinterpret_cast<float(*)[kMergeParts]>(&s_acc[0][0][0]), s_m[0], s_l[0]);
                }
            } else if (done == 0) {
                record = pair;
            }
        }
        __syncthreads();

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
    if (!kMerged && threadIdx.x == 0) records[blockIdx.x] = record;
}

// Joins the parts of the pairs, four rows a block: grid (blocks of the stream, rows / 4)
template <int kDim, bool kBf16>
__global__ __launch_bounds__(256) void k_pages_stream_merge(PagesAttend a, int kernel_rows) {
    __shared__ float s_weight[4][kStreamMostBlocks], s_top[4], s_sum[4];
    const StreamRecord rec = reinterpret_cast<const StreamRecord*>(a.records)[blockIdx.x];
    if (rec.parts == 0) return;
    bool fits;
    const PageSeq seq = read_seq(a.seqs, a.geom, rec.seq, fits);
    const int r0 = 4 * (int)blockIdx.y;
    if (r0 >= seq.n * a.group) return;
    join_parts<kDim, kBf16, kStreamMostBlocks>(a, rec, seq, kernel_rows, r0, min(4, seq.n * a.group - r0), s_weight, s_top, s_sum);
}

}  // namespace

}  // namespace sali
