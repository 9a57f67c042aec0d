// Attention of many new tokens a sequence (chunks of prompts, whole prompts): tiles of rows on the matrix cores.
//
// A block takes kWaves * kSets * 32 rows of one sequence and K/V head and walks the keys they see, 64 at a time.  The 64 keys are brought
// into LDS once for all waves (dequantised on the way, in the order of the operands) while the 64 before are worked on; a wave
// multiplies them with its kSets * 32 rows, whose queries stay in registers.
//
// The causal triangle, windows and ragged batches make blocks of very different length: a planning launch of one block writes the
// units (rows and a range of key tiles), the longest first, and cuts the keys of those that are longer than a fair share of the whole; the
// parts of a cut unit leave partial results that a merge launch joins.
#pragma once

#include "pages_attn.h"

namespace sali {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kUnitBuckets = 64;

struct TileUnit {
    int32_t seq, row_tile, lo, hi;          // tiles lo .. hi - 1 of the rows' view
    int32_t part, pad[3];                   // partial result, -1: the unit is whole
};
struct TileMerge {
    int32_t seq, row_tile, part, parts;
};
struct TilePlan {
    int32_t n_units, n_merges, pad[62];
};
struct TileScratch {
    TilePlan* plan;
    TileMerge* merges;
    TileUnit* units;
};
__host__ __device__ inline TileScratch tile_scratch(int32_t* records, int n_kv) {
    TileScratch t;
    t.plan = reinterpret_cast<TilePlan*>(records);
    t.merges = reinterpret_cast<TileMerge*>(t.plan + 1);
    t.units = reinterpret_cast<TileUnit*>(t.merges + tile_parts(n_kv));
    return t;
}

// one block
__global__ __launch_bounds__(kPlanThreads) void k_pages_plan(PagesAttend a, int rows_min) {
    __shared__ int64_t s_sum[kPlanThreads / 64];
    __shared__ int s_longest[kPlanThreads / 64];
    __shared__ int s_count[kUnitBuckets], s_next[kUnitBuckets];
    __shared__ int s_parts, s_merges;
    const TileScratch t = tile_scratch(a.records, a.geom.n_kv);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t slots = tile_slots(a.seqs.n_tokens, a.group, a.seqs.n_seqs);
    auto slot0 = [&](int s) -> int64_t { return (int64_t)max(0, a.seqs.start[s]) * a.group / kTileRows + s; };
    // the unit of slot i before any cut
    auto whole = [&](int64_t i) -> TileUnit {
        int lo = 0, n = a.seqs.n_seqs;
        while (n > 1) {
            const int half = n / 2;
            if (slot0(lo + half) <= i) {
                lo += half;
                n -= half;
            } else {
                n = half;
            }
        }
        TileUnit u = {lo, 0, 0, 0, -1, {0, 0, 0}};
        const PageSeq q = load_seq(a.seqs, a.geom, lo, true);
        const int64_t tile = i - slot0(lo);
        if (tile < 0 || (int64_t)q.n * a.group < rows_min || tile * kTileRows >= (int64_t)q.n * a.group) return u;
        u.row_tile = (int)tile;
        u.hi = view_of_rows(q, u.row_tile, a.group, a.window, a.sinks).tiles;
        return u;
    };
    if (threadIdx.x < kUnitBuckets) s_count[threadIdx.x] = 0;
    if (threadIdx.x == 0) s_parts = s_merges = 0;
    int64_t sum = 0;
    int longest = 1;
    TileUnit first = {0, 0, 0, 0, -1, {0, 0, 0}};
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        const TileUnit u = whole(i);
        if (i == threadIdx.x) first = u;
        sum += u.hi;
        longest = max(longest, u.hi);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off);
        longest = max(longest, __shfl_xor(longest, off));
    }
    if (lane == 0) {
        s_sum[wave] = sum;
        s_longest[wave] = longest;
    }
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        sum += s_sum[w];
        longest = max(longest, s_longest[w]);
    }
    const int share = fair_share(sum, a.geom.n_kv);
    const int most = min(share, longest);                   // the longest unit after the cuts
    auto bucket_of = [&](int tiles) { return kUnitBuckets - 1 - min(kUnitBuckets - 1, (int)((int64_t)tiles * (kUnitBuckets - 1) / most)); };
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        const TileUnit u = i == threadIdx.x ? first : whole(i);
        if (u.hi == 0) continue;
        const int parts = parts_of(u.hi, share);
        for (int k = 0; k < parts; ++k)
            atomicAdd(&s_count[bucket_of((int)((int64_t)u.hi * (k + 1) / parts - (int64_t)u.hi * k / parts))], 1);
    }
    __syncthreads();
    if (threadIdx.x < kUnitBuckets) {
        int v = s_count[threadIdx.x];
        const int own = v;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int u = __shfl_up(v, off);
            if (lane >= off) v += u;
        }
        s_next[threadIdx.x] = v - own;
        if (threadIdx.x == kUnitBuckets - 1) t.plan->n_units = v;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        TileUnit u = i == threadIdx.x ? first : whole(i);
        if (u.hi == 0) continue;
        const int parts = parts_of(u.hi, share), tiles = u.hi;
        int part = -1;
        if (parts > 1) {
            part = atomicAdd(&s_parts, parts);
            t.merges[atomicAdd(&s_merges, 1)] = {u.seq, u.row_tile, part, parts};
        }
        for (int k = 0; k < parts; ++k) {
            u.lo = (int)((int64_t)tiles * k / parts);
            u.hi = (int)((int64_t)tiles * (k + 1) / parts);
            u.part = parts > 1 ? part + k : -1;
            t.units[atomicAdd(&s_next[bucket_of(u.hi - u.lo)], 1)] = u;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) t.plan->n_merges = s_merges;
}

// ---- bringing 64 keys into LDS: four blocks of 16 tokens, each in the layout of 16-bit blocks (K [D / 8][place][8], V [2][D][8])
template <int kStore, int kDim, int kWaves>
struct TileRaw {
    static constexpr int kPieces = kStore == SALI_STORE_16 ? 2 * kDim : (kStore == SALI_STORE_INT8 ? kDim : kDim / 2);   // of 16 bytes, K or V of a block
    static constexpr int kShare = kPieces * 4 / kWaves;                 // a wave's: a block, or half of one
    static constexpr int kLoads = (kShare + 63) / 64;
    u32x4 k[kLoads], v[kLoads];
    float ks[kStore == SALI_STORE_16 ? 1 : kLoads];
    Scales8 vs[kStore == SALI_STORE_16 ? 1 : kLoads];
    uint16_t kz[kStore == SALI_STORE_INT4 ? kLoads : 1];
    u32x4 vz[kStore == SALI_STORE_INT4 ? kLoads : 1];
};
template <int kStore, int kDim, int kWaves>
__device__ __forceinline__ void tile_load(const char* block, int wave, int lane, TileRaw<kStore, kDim, kWaves>& r) {
    typedef TileRaw<kStore, kDim, kWaves> R;
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    const int p0 = wave % (kWaves / 4) * R::kShare;
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::kShare % 64 != 0 && lane + 64 * i >= R::kShare) continue;
        const uint32_t p = (uint32_t)(p0 + 64 * i + lane);
        r.k[i] = load16(block + p * 16);
        r.v[i] = load16(block + kAt.v + p * 16);
        if constexpr (kStore != SALI_STORE_16) {
            // K piece: [D / 16 or D / 32][place]; V piece: [2][group][8 pieces of two values or of two bytes], 16 pieces where codes are bytes
            const uint32_t kg = kStore == SALI_STORE_INT8 ? p >> 5 : p >> 4, place = p & 15;
            const uint32_t per = kStore == SALI_STORE_INT8 ? 16 : 8, a = p / (kDim / 32 * per), vg = p / per % (kDim / 32);
            r.ks[i] = *reinterpret_cast<const float*>(block + kAt.ks + (kg * 16 + place) * 4);
            const f32x4* s = reinterpret_cast<const f32x4*>(block + kAt.vs + (vg * 16 + a * 8) * 4);
            r.vs[i] = {s[0], s[1]};
            if constexpr (kStore == SALI_STORE_INT4) {
                r.kz[i] = *reinterpret_cast<const uint16_t*>(block + kAt.kz + (kg * 16 + place) * 2);
                r.vz[i] = load16(block + kAt.vz + (vg * 16 + a * 8) * 2);
            }
        }
    }
}
// ... with those of its tokens that are alive (the first `live`); V's others become zeros.  Are some of V's 16-bit values not finite?
template <int kStore, int kDim, bool kBf16, int kWaves>
__device__ __forceinline__ bool tile_store(TileRaw<kStore, kDim, kWaves>& r, int live, int wave, int lane, bool look, uint8_t* k, uint8_t* v) {
    typedef TileRaw<kStore, kDim, kWaves> R;
    const int p0 = wave % (kWaves / 4) * R::kShare, at = wave / (kWaves / 4) * (32 * kDim);
    bool odd = false;
    auto put = [](uint8_t* to, const u32x4& x) { *reinterpret_cast<u32x4*>(to) = x; };
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::kShare % 64 != 0 && lane + 64 * i >= R::kShare) continue;
        const int p = p0 + 64 * i + lane;
        if (live < kBlockTokens) {
            const int mine = live - 8 * (p / (R::kPieces / 2));
            if constexpr (kStore == SALI_STORE_16) r.v[i] = live_tokens(r.v[i], mine);
            else r.vs[i] = live_tokens(r.vs[i], mine);
            if constexpr (kStore == SALI_STORE_INT4) r.vz[i] = live_tokens(r.vz[i], mine);
        }
        if constexpr (kStore == SALI_STORE_16) {
            if (look) odd |= any_not_finite<kBf16>(r.v[i]);
            put(k + at + p * 16, r.k[i]);
            put(v + at + p * 16, r.v[i]);
        } else if constexpr (kStore == SALI_STORE_INT8) {
            uint8_t* const kd = k + at + ((p >> 4) * 32 + (p & 15)) * 16;
            put(kd, values8<kBf16>(r.k[i].x, r.k[i].y, r.ks[i]));
            put(kd + 256, values8<kBf16>(r.k[i].z, r.k[i].w, r.ks[i]));
            uint8_t* const vd = v + at + p * 32;
            put(vd, values8<kBf16>(r.v[i].x, r.v[i].y, r.vs[i]));
            put(vd + 16, values8<kBf16>(r.v[i].z, r.v[i].w, r.vs[i]));
        } else {
            const float low = low_half<kBf16>(r.kz[i]);
            constexpr uint32_t kLow = 0x0F0F0F0Fu;
            uint8_t* const kd = k + at + ((p >> 4) * 64 + (p & 15)) * 16;
            put(kd, values4<kBf16>(r.k[i].x & kLow, r.k[i].y & kLow, r.ks[i], low));
            put(kd + 256, values4<kBf16>(r.k[i].z & kLow, r.k[i].w & kLow, r.ks[i], low));
            put(kd + 512, values4<kBf16>(r.k[i].x >> 4 & kLow, r.k[i].y >> 4 & kLow, r.ks[i], low));
            put(kd + 768, values4<kBf16>(r.k[i].z >> 4 & kLow, r.k[i].w >> 4 & kLow, r.ks[i], low));
            uint8_t* const vd = v + at + ((p >> 3) * 32 + (p & 7) * 2) * 16;
            put(vd, values4<kBf16>(r.v[i].x & kLow, r.v[i].y & kLow, r.vs[i], r.vz[i]));
            put(vd + 16, values4<kBf16>(r.v[i].z & kLow, r.v[i].w & kLow, r.vs[i], r.vz[i]));
            put(vd + 256, values4<kBf16>(r.v[i].x >> 4 & kLow, r.v[i].y >> 4 & kLow, r.vs[i], r.vz[i]));
            put(vd + 272, values4<kBf16>(r.v[i].z >> 4 & kLow, r.v[i].w >> 4 & kLow, r.vs[i], r.vz[i]));
        }
    }
    return odd;
}

template <int kStore, int kDim, bool kBf16, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void k_pages_tile(PagesAttend a) {
    constexpr int kSets = kTileRows / 32 / kWaves;          // of 32 rows, a wave
    constexpr int kSteps = kDim / 16, kDt = kDim / 32, kPitch = kDim + 4;
    constexpr int kHalf = kTileKeys * kDim * 2;             // bytes of the tile's K or V
    __shared__ __align__(16) uint8_t s_k[2][kHalf], s_v[2][kHalf];
    __shared__ int s_live[2][4];            // of each block of 16 tokens: those that a row may see
    __shared__ int s_odd[2][kWaves];        // V holds values that are not finite, and some row does not see some key
    const TileScratch t = tile_scratch(a.records, a.geom.n_kv);
    const int n_kv = a.geom.n_kv;
    const int nth = (int)(blockIdx.x / (uint32_t)n_kv), head = (int)blockIdx.x - nth * n_kv;
    if (nth >= t.plan->n_units) return;
    const TileUnit unit = t.units[nth];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
    const int group = a.group;
    const PageSeq seq = load_seq(a.seqs, a.geom, unit.seq, false);
    const View view = view_of_rows(seq, unit.row_tile, group, a.window, a.sinks);
    const int32_t* table = a.seqs.table + (int64_t)unit.seq * a.seqs.width;
    const char* const heads = a.geom.pool + (uint64_t)head * a.geom.head_bytes;
    const uint32_t block_bytes = a.geom.head_bytes >> a.geom.blocks_log2;

    // the wave's block of a tile
    constexpr int kPer = kWaves / 4;                        // waves that share a block
    auto page_at = [&](int i) -> int {
        const int block = 4 * tile_at(view, i) + wave / kPer;
        return block * kBlockTokens < seq.len ? table[block >> a.geom.blocks_log2] : -1;
    };
    int live;
    auto block_at = [&](int i, int page) -> const char* {
        const int block = 4 * tile_at(view, i) + wave / kPer;
        live = max(0, min(kBlockTokens, seq.len - block * kBlockTokens));
        if ((unsigned)page >= (unsigned)a.geom.n_pages) {
            if (live > 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
            live = page = 0;
        }
        return heads + (uint64_t)page * a.geom.page_bytes + (uint32_t)(block & ((1 << a.geom.blocks_log2) - 1)) * block_bytes;
    };
    auto put_tile = [&](auto& raw, int i, int buf) {
        const bool look = kStore == SALI_STORE_16 && partly_hidden(view, a.window, a.sinks, tile_at(view, i) * kTileKeys, kTileKeys);
        const bool odd = tile_store<kStore, kDim, kBf16, kWaves>(raw, live, wave, lane, look, s_k[buf], s_v[buf]);
        if constexpr (kStore == SALI_STORE_16) {
            const bool any = __builtin_amdgcn_ballot_w64(odd) != 0;
            if (lane == 0) s_odd[buf][wave] = any ? 1 : 0;
        }
        if (lane == 0) s_live[buf][wave / kPer] = live;
    };
    typedef TileRaw<kStore, kDim, kWaves> Raw;
    Raw raw;
    int page = __builtin_amdgcn_readfirstlane(page_at(unit.lo));
    tile_load<kStore, kDim, kWaves>(block_at(unit.lo, page), wave, lane, raw);
    int page_next = unit.lo + 1 < unit.hi ? page_at(unit.lo + 1) : -1;

    const int64_t row0 = (int64_t)unit.row_tile * kTileRows + wave * 32 * kSets, rows = (int64_t)seq.n * group;
    const bool some = row0 < rows;                          // uniform over the wave
    View mine = view;
    {
        const int64_t last = min(rows, row0 + 32 * kSets) - 1;
        mine.first = seq.len - seq.n + (int)(row0 / group);
        mine.last = seq.len - seq.n + (int)(last / group);
    }
    u32x4 q[kSets][kSteps];
    int pos[kSets];
#pragma unroll
    for (int c = 0; c < kSets; ++c) {
        const int64_t r = row0 + 32 * c + col;
        const int token = (int)(r / group), g = (int)(r - (int64_t)token * group);
        pos[c] = r < rows ? seq.len - seq.n + token : -1;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            q[c][s] = (u32x4){0u, 0u, 0u, 0u};
            if (r < rows) {
                const u32x4 v = load16(a.q.d + (int64_t)(seq.first + token) * a.q.token_bytes + (int64_t)(head * group + g) * a.q.head_bytes +
                                       2 * (16 * s + 8 * hh));
#pragma unroll
                for (int e = 0; e < 4; ++e) q[c][s][e] = (v[e] & a.q_keep) ^ a.q_flip;
            }
        }
    }
    float m[kSets], l[kSets];
    f32x16 acc[kSets][kDt];
    uint64_t up[kSets], down[kSets];                        // a bit for every value of acc: values that are not finite
#pragma unroll
    for (int c = 0; c < kSets; ++c) {
        m[c] = -INFINITY;
        l[c] = 0.0f;
        up[c] = down[c] = 0u;
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[c][d][r] = 0.0f;
    }

    put_tile(raw, unit.lo, 0);
    for (int i = unit.lo; i < unit.hi; ++i) {
        const int buf = (i - unit.lo) & 1;
        __syncthreads();                                    // this tile is there, and every wave is through with the other buffer
        const bool more = i + 1 < unit.hi;
        if (more) {
            page = __builtin_amdgcn_readfirstlane(page_next);
            tile_load<kStore, kDim, kWaves>(block_at(i + 1, page), wave, lane, raw);
            if (i + 2 < unit.hi) page_next = page_at(i + 2);
        }
        const int tile0 = tile_at(view, i) * kTileKeys;
        if constexpr (kStore == SALI_STORE_16) {
            if (__builtin_amdgcn_ballot_w64(s_odd[buf][lane % kWaves] != 0) != 0) {          // the same for all waves
                if (some) {
#pragma unroll
                    for (int c = 0; c < kSets; ++c)
#pragma unroll 1
                        for (int b = 0; b < 4; ++b) {
                            u32x4 seen;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int j = tile0 + 16 * b + 8 * hh + 2 * e, there = s_live[buf][b] - 8 * hh;
                                seen[e] = (2 * e < there && sees(pos[c], j, a.window, a.sinks) ? (uint32_t)Num<kBf16>::kOne : 0u) |
                                          (2 * e + 1 < there && sees(pos[c], j + 1, a.window, a.sinks) ? (uint32_t)Num<kBf16>::kOne << 16 : 0u);
                            }
#pragma unroll 1                                            // not to cost registers
                            for (int d = 0; d < kDt; ++d) {
                                u32x4 finite, plus, minus;
                                take_apart<kBf16>(load16(s_v[buf] + b * (32 * kDim) + (hh * kDim + col + 32 * d) * 16), finite, plus, minus);
                                f32x16 zero;
#pragma unroll
                                for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
                                const f32x16 ups = Num<kBf16>::mma32(plus, seen, zero), downs = Num<kBf16>::mma32(minus, seen, zero);
                                uint32_t u = 0, w = 0;
#pragma unroll
                                for (int r = 0; r < 16; ++r) {
                                    u |= ups[r] > 0.0f ? 1u << r : 0u;
                                    w |= downs[r] > 0.0f ? 1u << r : 0u;
                                }
                                up[c] |= (uint64_t)u << (16 * d);
                                down[c] |= (uint64_t)w << (16 * d);
                            }
                        }
                }
                __syncthreads();                            // every wave has looked
                for (int p = (int)threadIdx.x; p < kHalf / 16; p += 64 * kWaves) {
                    u32x4 finite, plus, minus;
                    take_apart<kBf16>(load16(s_v[buf] + p * 16), finite, plus, minus);
                    *reinterpret_cast<u32x4*>(s_v[buf] + p * 16) = finite;
                }
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int sub = 0; sub < 2; ++sub) {
            const int j0 = tile0 + 32 * sub;
            if (!some || j0 > mine.last) break;
            const uint8_t* const kb = s_k[buf] + sub * (64 * kDim), * const vb = s_v[buf] + sub * (64 * kDim);
            f32x16 s2[kSets];
#pragma unroll
            for (int c = 0; c < kSets; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) s2[c][r] = 0.0f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const u32x4 kf = load16(kb + (col >> 4) * (32 * kDim) + ((2 * s + hh) * 16 + (col & 15)) * 16);
#pragma unroll
                for (int c = 0; c < kSets; ++c) s2[c] = Num<kBf16>::mma32(kf, q[c][s], s2[c]);
            }
            // lane (row col, hh): register r has token 8 hh + r % 8 of block r / 8
            const int live0 = __builtin_amdgcn_readfirstlane(s_live[buf][2 * sub]), live1 = __builtin_amdgcn_readfirstlane(s_live[buf][2 * sub + 1]);
            const bool masked = live0 < kBlockTokens || live1 < kBlockTokens || partly_hidden(mine, a.window, a.sinks, j0, 32);
            if (masked) {
#pragma unroll
                for (int c = 0; c < kSets; ++c)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if ((r < 8 ? live0 : live1) <= 0 || !sees(pos[c], j0 + 16 * (r / 8) + 8 * hh + r % 8, a.window, a.sinks)) s2[c][r] = -INFINITY;
            }
            u32x4 p[kSets][2];
#pragma unroll
            for (int c = 0; c < kSets; ++c) {
                float top = s2[c][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) top = fmaxf(top, s2[c][r]);
                top = max_over_halves(top) * a.scale2;
                const float to = top > m[c] + kLag ? top : m[c];
                if (__builtin_amdgcn_ballot_w64(to != m[c]) != 0) {
                    const float by = to != m[c] ? __builtin_amdgcn_exp2f(m[c] - to) : 1.0f;
                    l[c] *= by;
#pragma unroll
                    for (int d = 0; d < kDt; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[c][d][r] *= by;
                    m[c] = to;
                }
                const float ref = m[c] == -INFINITY ? 0.0f : m[c];
                float e[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s2[c][r], a.scale2, -ref));
                    l[c] += e[r];
                }
#pragma unroll
                for (int r = 0; r < 8; ++r) p[c][r / 4][r % 4] = pack2<kBf16>(e[2 * r], e[2 * r + 1]);
            }
            const uint8_t* const vl = vb + (hh * kDim + col) * 16;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int d = 0; d < kDt; ++d) {
                    const u32x4 vf = load16(vl + b * (32 * kDim) + d * 512);
#pragma unroll
                    for (int c = 0; c < kSets; ++c) acc[c][d] = Num<kBf16>::mma32(vf, p[c][b], acc[c][d]);
                }
        }
        if (more) put_tile(raw, i + 1, buf ^ 1);
    }

    // ---- results: lane (row col, hh) has values 32 d + 8 k + 4 hh .. + 3
#pragma unroll
    for (int c = 0; c < kSets; ++c) {
        const int64_t r = row0 + 32 * c + col;
        const float sum = sum_over_halves(l[c]);
        if (r >= rows) continue;
        if constexpr (kStore == SALI_STORE_16)
            if ((up[c] | down[c]) != 0)
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int x = 0; x < 16; ++x) acc[c][d][x] += found((up[c] >> (16 * d + x) & 1) != 0, (down[c] >> (16 * d + x) & 1) != 0);
        if (unit.part >= 0) {
            float* part = a.partial + (((size_t)unit.part * n_kv + head) * kTileRows + (size_t)(r - (int64_t)unit.row_tile * kTileRows)) * kPitch;
            if (hh == 0) {
                part[0] = m[c];
                part[1] = sum;
            }
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<f32x4*>(part + 4 + 32 * d + 8 * k + 4 * hh) =
                        (f32x4){acc[c][d][4 * k], acc[c][d][4 * k + 1], acc[c][d][4 * k + 2], acc[c][d][4 * k + 3]};
            continue;
        }
        const int token = (int)(r / group), h = head * group + (int)(r - (int64_t)token * group);
        const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
        const RowEnd e = row_end(m[c], sum, a, row);
        char* const out = a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes + (int64_t)h * a.out.head_bytes;
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f32x4 pr = {0.0f, 0.0f, 0.0f, 0.0f};
                const int at = 32 * d + 8 * k + 4 * hh;
                if (a.prior != nullptr) pr = *reinterpret_cast<const f32x4*>(a.prior + row * kDim + at);
                float o[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) o[x] = joined(e, acc[c][d][4 * k + x], pr[x]);
                *reinterpret_cast<u32x2*>(out + 2 * at) = (u32x2){pack2<kBf16>(o[0], o[1]), pack2<kBf16>(o[2], o[3])};
            }
        if (hh == 0 && a.lse != nullptr) a.lse[row] = e.lse;
    }
}

// Joins the parts of cut units: grid (merges * n_kv at most, kTileRows / 8), a row per 32 lanes
template <int kDim, bool kBf16>
__global__ __launch_bounds__(256) void k_pages_tile_merge(PagesAttend a) {
    constexpr int kPitch = kDim + 4, kPer = kDim / 32;
    const TileScratch t = tile_scratch(a.records, a.geom.n_kv);
    const int n_kv = a.geom.n_kv;
    const int nth = (int)(blockIdx.x / (uint32_t)n_kv), head = (int)blockIdx.x - nth * n_kv;
    if (nth >= t.plan->n_merges) return;
    const TileMerge rec = t.merges[nth];
    const PageSeq seq = load_seq(a.seqs, a.geom, rec.seq, false);
    const int in_tile = (int)blockIdx.y * 8 + (int)(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int64_t r = (int64_t)rec.row_tile * kTileRows + in_tile;
    if (r >= (int64_t)seq.n * a.group) return;
    float m = -INFINITY, l = 0.0f, acc[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.0f;
#pragma unroll 4
    for (int i = 0; i < rec.parts; ++i) {
        const float* part = a.partial + (((size_t)(rec.part + i) * n_kv + head) * kTileRows + in_tile) * kPitch;
        const float pm = part[0], pl = part[1];
        float v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = part[4 + lane * kPer + e];
        if (pl == 0.0f) continue;               // nothing seen
        const float to = fmaxf(m, pm), by = __builtin_amdgcn_exp2f(m - to), pby = __builtin_amdgcn_exp2f(pm - to);
        const bool none = l == 0.0f;
        l = (none ? 0.0f : l * by) + pl * pby;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = (none ? 0.0f : acc[e] * by) + v[e] * pby;
        m = to;
    }
    const int token = (int)(r / a.group), h = head * a.group + (int)(r - (int64_t)token * a.group);
    const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
    const RowEnd e = row_end(m, l, a, row);
    typename Num<kBf16>::T* out = reinterpret_cast<typename Num<kBf16>::T*>(a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes +
                                                                           (int64_t)h * a.out.head_bytes) + lane * kPer;
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
        const float pr = a.prior != nullptr ? a.prior[row * kDim + lane * kPer + x] : 0.0f;
        out[x] = (typename Num<kBf16>::T)joined(e, acc[x], pr);
    }
    if (lane == 0 && a.lse != nullptr) a.lse[row] = e.lse;
}

}  // namespace

}  // namespace sali
