// Attention of many new tokens a sequence (chunks of prompts, whole prompts): tiles of rows on the matrix cores.
//
// A block takes a row tile, 384 or 128 rows of one sequence and K/V head, 32 a wave, and walks the keys they see, 96 or 32 at a time.  The
// keys are brought into LDS once for all waves (dequantised on the way, in the order of the operands) while those before are worked on; a
// wave multiplies them with its rows, whose queries stay in registers.
//
// The causal triangle, windows and ragged batches make row tiles of very different length.  A planning launch of one block writes the pieces
// that blocks take: in shares, the longest first, with the keys of those cut that are longer than a fair share of the whole; or in
// stretches, all keys of all row tiles in a row and cut evenly, a block a compute unit (pages_attn_launch.h says which when).  The parts
// of a cut row tile leave partial results that a merge launch joins.
//
// What bounds it.  A wave's 32 rows and 32 keys of 128 values are 16 products of 32x32x16 (512 cycles of the matrix cores), the softmax's
// vector instructions and 16 KB from LDS.  Matrix products and LDS reads alone ran at 1235 TFLOP/s (a large library product: 1372), with
// the softmax 1010, with keys brought in through registers 945 to 958: 8192 causal tokens, 32 heads over 8 of 128 values in 570 to 588 us.  Three
// waves a SIMD hide one wave's softmax behind the others' products (one wave alone issues a vector instruction every 6.4 cycles,
// several together one every 3); blocks in lockstep of product and softmax phases were slower, 683 to 740 us.  32 rows a wave, since 64
// take more than the 168 registers that three waves leave each.
#pragma once

#include "pages_attn.h"

namespace sali {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kUnitBuckets = 64;
constexpr int kTileMostBlocks = 256;        // of a head in stretches
constexpr int kTileMostMerges = 1024;

struct __align__(16) TileUnit {             // a row tile
    TileSpan span;
    int32_t seq, row_tile, first, n, len, pad[3];           // the sequence's first new token, new tokens, tokens
};
struct __align__(16) TilePiece {            // tiles lo .. hi - 1 of its keys
    int32_t seq, row_tile, first, n, len, lo, hi, part;     // partial result, -1: it is all of them
};
struct TileMerge {
    int32_t seq, row_tile, part, parts;
};
struct TilePlan {
    int32_t stretches;                      // 0: a block takes one piece, block n the n-th
    int32_t blocks, n_merges, pad[61];
};
// One area for all the kernels: a plan, and behind the pieces the row tiles that they are made from
struct TileScratch {
    TilePlan plan;
    TileMerge merges[kTileMostMerges];
    int32_t begin[kTileMostBlocks], end[kTileMostBlocks];   // a block's pieces, in stretches
    TilePiece pieces[1];
};
static_assert(sizeof(TilePlan) == 256 && sizeof(TileUnit) == 48 && sizeof(TilePiece) == 32 && offsetof(TileScratch, pieces) % 16 == 0, "records");
__host__ __device__ inline int64_t tile_pieces(int64_t slots, int n_kv, int waves) { return slots + most(tile_parts(n_kv, waves), kTileMostBlocks); }
__host__ inline size_t tile_scratch_bytes(int64_t slots, int n_kv, int waves) {
    return offsetof(TileScratch, pieces) + (size_t)tile_pieces(slots, n_kv, waves) * sizeof(TilePiece) + (size_t)slots * sizeof(TileUnit);
}

// the row tile in a slot, or none (no tiles)
template <int kWaves>
__device__ __forceinline__ TileUnit tile_unit(const PagesAttend& a, int rows_min, int64_t slot) {
    constexpr int kTileRows = tile_rows(kWaves);
    auto slot0 = [&](int s) -> int64_t { return (int64_t)((uint32_t)min(max(0, a.seqs.start[s]), a.seqs.n_tokens) * (uint32_t)a.group / (uint32_t)kTileRows) + s; };
    int lo = 0, n = a.seqs.n_seqs;
    while (n > 1) {
        const int half = n / 2;
        if (slot0(lo + half) <= slot) {
            lo += half;
            n -= half;
        } else {
            n = half;
        }
    }
    const PageSeq q = load_seq(a.seqs, a.geom, lo, true);
    const int64_t tile = slot - slot0(lo), rows = (int64_t)q.n * a.group;
    TileUnit u = {{0, 0, 0}, lo, (int)tile, q.first, q.n, q.len, {0, 0, 0}};
    if (tile < 0 || rows < rows_min || tile * kTileRows >= rows) return u;
    u.span.tiles = view_of_rows<kWaves>(q, u.row_tile, a.group, a.window, a.sinks).tiles;
    u.span.weight = tile_weight((int)min((int64_t)kTileRows, rows - tile * kTileRows));
    return u;
}

// The plan in shares, one block (5 to 8 us: a few trips to memory one after the other)
template <int kWaves>
__global__ __launch_bounds__(kPlanThreads) void k_pages_plan_shares(PagesAttend a, int rows_min) {
    __shared__ int64_t s_sum[kPlanThreads / 64];
    __shared__ int s_longest[kPlanThreads / 64], s_falls[kPlanThreads / 64];
    __shared__ int s_count[kUnitBuckets], s_next[kUnitBuckets];
    __shared__ int s_parts, s_merges;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int64_t slots = tile_slots(a.seqs.n_tokens, a.group, a.seqs.n_seqs, tile_rows(kWaves));
    TileScratch& t = *reinterpret_cast<TileScratch*>(a.records);
    const StartFalls starts(a.seqs.start, a.seqs.n_seqs, threadIdx.x, kPlanThreads);
    if (threadIdx.x < kUnitBuckets) s_count[threadIdx.x] = 0;
    if (threadIdx.x == 0) s_parts = s_merges = 0;
    int64_t sum = 0;
    int longest = 1;
    TileUnit first = {{0, 0, 0}, 0, 0, 0, 0, 0, {0, 0, 0}};
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        const TileUnit u = tile_unit<kWaves>(a, rows_min, i);
        if (i == threadIdx.x) first = u;
        sum += u.span.tiles;
        longest = max(longest, u.span.tiles);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off);
        longest = max(longest, __shfl_xor(longest, off));
    }
    const bool falls = __builtin_amdgcn_ballot_w64(starts.some()) != 0;
    if (lane == 0) {
        s_sum[wave] = sum;
        s_longest[wave] = longest;
        s_falls[wave] = falls ? 1 : 0;
        if (falls) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
    }
    __syncthreads();
    sum = 0;
    int some_falls = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        sum += s_sum[w];
        longest = max(longest, s_longest[w]);
        some_falls |= s_falls[w];
    }
    if (some_falls != 0) slots = 0;
    const int share = fair_share(sum, tile_shares(a.geom.n_kv, kWaves));
    const int most_tiles = min(share, longest);             // of the longest piece
    auto bucket_of = [&](int tiles) { return kUnitBuckets - 1 - min(kUnitBuckets - 1, (int)((int64_t)tiles * (kUnitBuckets - 1) / most_tiles)); };
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        const TileUnit u = i == threadIdx.x ? first : tile_unit<kWaves>(a, rows_min, i);
        const int tiles = u.span.tiles;
        if (tiles == 0) continue;
        const int parts = parts_of(tiles, share);
        for (int k = 0; k < parts; ++k) atomicAdd(&s_count[bucket_of((int)((int64_t)tiles * (k + 1) / parts - (int64_t)tiles * k / parts))], 1);
    }
    __syncthreads();
    if (threadIdx.x < kUnitBuckets) {
        int v = s_count[threadIdx.x];
        const int own = v;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int x = __shfl_up(v, off);
            if (lane >= off) v += x;
        }
        s_next[threadIdx.x] = v - own;
        if (threadIdx.x == kUnitBuckets - 1) t.plan.blocks = v;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < slots; i += kPlanThreads) {
        const TileUnit u = i == threadIdx.x ? first : tile_unit<kWaves>(a, rows_min, i);
        const int tiles = u.span.tiles;
        if (tiles == 0) continue;
        const int parts = parts_of(tiles, share);
        int part = -1;
        if (parts > 1) {
            part = atomicAdd(&s_parts, parts);
            t.merges[atomicAdd(&s_merges, 1)] = {u.seq, u.row_tile, part, parts};
        }
        for (int k = 0; k < parts; ++k) {
            const int lo = (int)((int64_t)tiles * k / parts), hi = (int)((int64_t)tiles * (k + 1) / parts);
            t.pieces[atomicAdd(&s_next[bucket_of(hi - lo)], 1)] = {u.seq, u.row_tile, u.first, u.n, u.len, lo, hi, parts > 1 ? part + k : -1};
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        t.plan.stretches = 0;
        t.plan.n_merges = s_merges;
    }
}

// The plan in stretches, `blocks` of a head; one block (5 to 6 us)
template <int kWaves>
__global__ __launch_bounds__(kPlanThreads) void k_pages_plan_stretches(PagesAttend a, int rows_min, int blocks) {
    __shared__ uint64_t s_weight[kPlanThreads / 64];
    __shared__ int s_units[kPlanThreads / 64];
    __shared__ int s_parts, s_merges, s_falls;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t slots = tile_slots(a.seqs.n_tokens, a.group, a.seqs.n_seqs, tile_rows(kWaves));
    TileScratch& t = *reinterpret_cast<TileScratch*>(a.records);
    TileUnit* const units = reinterpret_cast<TileUnit*>(t.pieces + tile_pieces(slots, a.geom.n_kv, kWaves));
    if (threadIdx.x == 0) s_parts = s_merges = s_falls = 0;
    const StartFalls starts(a.seqs.start, a.seqs.n_seqs, threadIdx.x, kPlanThreads);
    // the units that there are, one behind the other
    uint64_t total = 0;
    int count = 0;
    for (int64_t i0 = 0; i0 < slots; i0 += kPlanThreads) {
        TileUnit u = {{0, 0, 0}, 0, 0, 0, 0, 0, {0, 0, 0}};
        if (i0 + threadIdx.x < slots) u = tile_unit<kWaves>(a, rows_min, i0 + threadIdx.x);
        const uint64_t own = u.span.end();                  // from 0
        const uint64_t there = __builtin_amdgcn_ballot_w64(own != 0);
        uint64_t upto = own;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint64_t v = __shfl_up(upto, off);
            if (lane >= off) upto += v;
        }
        if (i0 != 0) __syncthreads();
        if (lane == 63) {
            s_weight[wave] = upto;
            s_units[wave] = __popcll(there);
        }
        __syncthreads();
        u.span.at = total + upto - own;
        int r = count + __popcll(there & ((1ull << lane) - 1ull));
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            if (w < wave) {
                u.span.at += s_weight[w];
                r += s_units[w];
            }
            total += s_weight[w];
            count += s_units[w];
        }
        if (own != 0) units[r] = u;
    }
    if (starts.some()) {
        s_falls = 1;
        atomicOr(a.seqs.status, SALI_FAULT_BATCH);
    }
    __syncthreads();
    if (s_falls != 0) count = 0;
    const uint64_t length = stretch_length(total, blocks);
    // eight lanes a unit, a lane a block
    const int sub = lane & 7;
    for (int r = threadIdx.x >> 3; r < count; r += kPlanThreads / 8) {
        const TileUnit u = units[r];
        const int first = u.span.first_block(length), last = u.span.last_block(length);
        const int before = r > 0 ? units[r - 1].span.last_block(length) : -1;
        const int after = r + 1 < count ? units[r + 1].span.first_block(length) : blocks;
        int part = -1;
        if (last > first) {
            if (sub == 0) {
                part = atomicAdd(&s_parts, last - first + 1);
                t.merges[atomicAdd(&s_merges, 1)] = {u.seq, u.row_tile, part, last - first + 1};
            }
            part = __shfl(part, lane - sub);
        }
        for (int b = first + sub; b <= last; b += 8) {
            const uint64_t start = (uint64_t)b * length;
            const int piece = stretch_piece(r, b);
            t.pieces[piece] = {u.seq, u.row_tile, u.first, u.n, u.len, u.span.before(start), u.span.before(start + length), last > first ? part + b - first : -1};
            if (b > before) t.begin[b] = piece;
            if (b < after) t.end[b] = piece + 1;
        }
        if (r == count - 1 && sub == 0) t.plan.blocks = last + 1;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        t.plan.stretches = 1;
        if (count == 0) t.plan.blocks = 0;
        t.plan.n_merges = s_merges;
    }
}

// ---- bringing keys into LDS: blocks of 16 tokens, each in the layout of 16-bit blocks (K [D / 8][place][8], V [2][D][8]), two waves a block
// Wave w has half w % 2 of block w / 2: half of K's pieces, and of V's those of tokens 8 (w % 2) .. + 7.
template <int kStore, int kDim>
struct TileRaw {
    static constexpr int kShare = (kStore == SALI_STORE_16 ? 2 * kDim : (kStore == SALI_STORE_INT8 ? kDim : kDim / 2)) / 2;   // pieces of 16 bytes, of K or V
    static constexpr int kLoads = (kShare + 63) / 64;
    u32x4 k[kLoads], v[kLoads];
    float ks[kStore == SALI_STORE_16 ? 1 : kLoads];
    typename std::conditional<kStore == SALI_STORE_INT4, Scales8, float>::type vs[kStore == SALI_STORE_16 ? 1 : kLoads];
    uint16_t kz[kStore == SALI_STORE_INT4 ? kLoads : 1];
    u32x4 vz[kStore == SALI_STORE_INT4 ? kLoads : 1];
    static __device__ __forceinline__ bool none(int i, int lane) { return kShare % 64 != 0 && lane + 64 * i >= kShare; }
};
template <int kStore, int kDim>
__device__ __forceinline__ void tile_load_k(const char* block, int half, int lane, TileRaw<kStore, kDim>& r) {
    typedef TileRaw<kStore, kDim> R;
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::none(i, lane)) continue;
        const uint32_t p = (uint32_t)(half * R::kShare + 64 * i + lane);
        r.k[i] = load16(block + p * 16);
        if constexpr (kStore != SALI_STORE_16) {            // pieces [D / 16 or D / 32][place]
            const uint32_t at = (kStore == SALI_STORE_INT8 ? p >> 5 : p >> 4) * 16 + (p & 15);
            r.ks[i] = *reinterpret_cast<const float*>(block + kAt.ks + at * 4);
            if constexpr (kStore == SALI_STORE_INT4) r.kz[i] = *reinterpret_cast<const uint16_t*>(block + kAt.kz + at * 2);
        }
    }
}
template <int kStore, int kDim>
__device__ __forceinline__ void tile_load_v(const char* block, int half, int lane, TileRaw<kStore, kDim>& r) {
    typedef TileRaw<kStore, kDim> R;
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::none(i, lane)) continue;
        const uint32_t p = (uint32_t)(64 * i + lane);
        r.v[i] = load16(block + kAt.v + (half * R::kShare + p) * 16);
        if constexpr (kStore != SALI_STORE_16) {            // pieces of two values (8 bits) or two bytes (4 bits) of a group
            const uint32_t at = (kStore == SALI_STORE_INT8 ? p >> 4 : p >> 3) * 16 + (uint32_t)half * 8;
            if constexpr (kStore == SALI_STORE_INT8) {
                r.vs[i] = *reinterpret_cast<const float*>(block + kAt.vs + (at + (p & 7)) * 4);
            } else {
                const f32x4* s = reinterpret_cast<const f32x4*>(block + kAt.vs + at * 4);
                r.vs[i] = {s[0], s[1]};
                r.vz[i] = load16(block + kAt.vz + at * 2);
            }
        }
    }
}
__device__ __forceinline__ void put16(uint8_t* to, const u32x4& x) { *reinterpret_cast<u32x4*>(to) = x; }
constexpr uint32_t kLowHalves = 0x0F0F0F0Fu;
// `k`, `v`: where the block lies in LDS
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ void tile_store_k(const TileRaw<kStore, kDim>& r, int half, int lane, uint8_t* k) {
    typedef TileRaw<kStore, kDim> R;
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::none(i, lane)) continue;
        const int p = half * R::kShare + 64 * i + lane;
        if constexpr (kStore == SALI_STORE_16) {
            put16(k + p * 16, r.k[i]);
        } else if constexpr (kStore == SALI_STORE_INT8) {
            uint8_t* const to = k + ((p >> 4) * 32 + (p & 15)) * 16;
            put16(to, values8<kBf16>(r.k[i].x, r.k[i].y, r.ks[i]));
            put16(to + 256, values8<kBf16>(r.k[i].z, r.k[i].w, r.ks[i]));
        } else {
            const float low = low_half<kBf16>(r.kz[i]);
            uint8_t* const to = k + ((p >> 4) * 64 + (p & 15)) * 16;
            put16(to, values4<kBf16>(r.k[i].x & kLowHalves, r.k[i].y & kLowHalves, r.ks[i], low));
            put16(to + 256, values4<kBf16>(r.k[i].z & kLowHalves, r.k[i].w & kLowHalves, r.ks[i], low));
            put16(to + 512, values4<kBf16>(r.k[i].x >> 4 & kLowHalves, r.k[i].y >> 4 & kLowHalves, r.ks[i], low));
            put16(to + 768, values4<kBf16>(r.k[i].z >> 4 & kLowHalves, r.k[i].w >> 4 & kLowHalves, r.ks[i], low));
        }
    }
}
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ void tile_store_v(const TileRaw<kStore, kDim>& r, int half, int lane, uint8_t* v) {
    typedef TileRaw<kStore, kDim> R;
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i) {
        if (R::none(i, lane)) continue;
        const int p = half * R::kShare + 64 * i + lane;
        if constexpr (kStore == SALI_STORE_16) {
            put16(v + p * 16, r.v[i]);
        } else if constexpr (kStore == SALI_STORE_INT8) {
            uint8_t* const to = v + p * 32;
            put16(to, row_values8<kBf16>(r.v[i].x, r.v[i].y, r.vs[i]));
            put16(to + 16, row_values8<kBf16>(r.v[i].z, r.v[i].w, r.vs[i]));
        } else {
            uint8_t* const to = v + ((p >> 3) * 32 + (p & 7) * 2) * 16;
            put16(to, values4<kBf16>(r.v[i].x & kLowHalves, r.v[i].y & kLowHalves, r.vs[i], r.vz[i]));
            put16(to + 16, values4<kBf16>(r.v[i].z & kLowHalves, r.v[i].w & kLowHalves, r.vs[i], r.vz[i]));
            put16(to + 256, values4<kBf16>(r.v[i].x >> 4 & kLowHalves, r.v[i].y >> 4 & kLowHalves, r.vs[i], r.vz[i]));
            put16(to + 272, values4<kBf16>(r.v[i].z >> 4 & kLowHalves, r.v[i].w >> 4 & kLowHalves, r.vs[i], r.vz[i]));
        }
    }
}

// what all lanes have alike, in scalar registers
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
    return (uint64_t)(uint32_t)uniform((int)(uint32_t)v) | (uint64_t)(uint32_t)uniform((int)(uint32_t)(v >> 32)) << 32;
}

// All waves of the block, LDS accesses before it done by then (global ones may be under way)
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// (4 bits: two waves a SIMD, as the unpacking takes more registers)
template <int kStore, int kDim, bool kBf16, int kTileWaves>
__global__ __launch_bounds__(64 * kTileWaves) __attribute__((amdgpu_waves_per_eu(kStore == SALI_STORE_INT4 ? 2 : 3, 3))) void k_pages_tile(PagesAttend args) {
    constexpr int kSteps = kDim / 16, kDt = kDim / 32, kPitch = kDim + 4;
    constexpr int kBlock = 32 * kDim;                       // bytes of a block's K or V in LDS
    constexpr int kTileRows = tile_rows(kTileWaves), kTileKeys = tile_keys(kTileWaves), kBlocks = kTileKeys / kBlockTokens;
    __shared__ __align__(16) uint8_t s_k[2][kBlocks * kBlock], s_v[2][kBlocks * kBlock];
    __shared__ int s_live[2][kBlocks];                            // of each block of 16 tokens: those that a row may see
    // 16-bit tiles that not all rows see whole: V's values that are not finite, +inf or NaN and -inf or NaN, a bit a token; of each wave's
    // share whether there are any
    __shared__ uint8_t s_up[2][kStore == SALI_STORE_16 ? kTileWaves : 1][kDim], s_down[2][kStore == SALI_STORE_16 ? kTileWaves : 1][kDim];
    __shared__ int s_odd[2][kTileWaves];
    __shared__ uint64_t s_found[2][kStore == SALI_STORE_16 ? 64 * kTileWaves : 1];
    __shared__ int s_nan[kTileWaves];                             // of each wave: is there one in its results
    const int nth = (int)(blockIdx.x / (uint32_t)args.geom.n_kv);
    int piece = nth, pieces_end = nth + 1;
    {
        const TileScratch& t = *reinterpret_cast<const TileScratch*>(args.records);
        if (nth >= t.plan.blocks) return;
        if (t.plan.stretches != 0) {
            piece = uniform(t.begin[nth]);
            pieces_end = uniform(t.end[nth]);
        }
    }
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = wave & 1;
    bool look = false, again = false;                             // 16 bits: the piece's second time, with a look at all keys; the wave needs it
#pragma unroll 1
    while (piece < pieces_end) {
        // arguments and the thread's number: anew for every piece, not kept in registers through the loop
        const PagesAttend a = late_arguments<0>();
        uint32_t all = ~0u;
        asm volatile("" : "+s"(all));
        const int lane = __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u)), thread = 64 * wave + lane, col = lane & 31, hh = lane >> 5;
        TilePiece unit = reinterpret_cast<const TileScratch*>(a.records)->pieces[piece];
        const PageSeq seq = {uniform(unit.first), uniform(unit.n), uniform(unit.len)};
        unit.row_tile = uniform(unit.row_tile);
        const int lo = uniform(unit.lo), hi = uniform(unit.hi), part_of_piece = uniform(unit.part);
        const int head = (int)(blockIdx.x % (uint32_t)a.geom.n_kv), group = a.group;
        const char* const heads = a.geom.pool + (uint64_t)head * a.geom.head_bytes;
        const uint32_t block_bytes = a.geom.head_bytes >> a.geom.blocks_log2;
        const int32_t* const table = a.seqs.table + (int64_t)uniform(unit.seq) * a.seqs.width;
        const View view = view_of_rows<kTileWaves>(seq, unit.row_tile, group, a.window, a.sinks);
        View to_look_at = view;             // keys that not all rows see, or all keys
        if (look) to_look_at.first = -1;

        // ---- the wave's share of the tiles: where tile i's block lies, and its tokens
        typedef TileRaw<kStore, kDim> Raw;
        Raw raw;
        auto block_of = [&](int i) { return kBlocks * tile_at(view, i) + (wave >> 1); };
        // the pages from `page0` on, one a lane: their numbers, and which are none
        const int pages = (seq.len + (kBlockTokens << a.geom.blocks_log2) - 1) / (kBlockTokens << a.geom.blocks_log2);
        int page0 = -64;
        int page_of_lane = 0;
        uint64_t no_page = 0;
        struct Source {
            const char* block;
            int live;
        };
        auto source = [&](int i) -> Source {
            const int block = block_of(i), index = block >> a.geom.blocks_log2;
            if ((unsigned)(index - page0) >= 64u) {
                page0 = index;
                int page = index + lane < pages ? table[index + lane] : -1;
                const bool none = (unsigned)page >= (unsigned)a.geom.n_pages;
                no_page = __builtin_amdgcn_ballot_w64(none);
                page_of_lane = none ? 0 : page;
                asm volatile("" : "+v"(page_of_lane));          // waited for here: a wait behind the branch would be one for K and V too
            }
            const int nth_page = index - page0;
            const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(page_of_lane, nth_page) * a.geom.page_bytes;
            Source s;
            s.live = max(0, min(kBlockTokens, seq.len - block * kBlockTokens));
            if ((no_page >> nth_page & 1) != 0) {
                if (i < hi && s.live > 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                s.live = 0;
            }
            s.block = heads + at + (uint32_t)(block & ((1 << a.geom.blocks_log2) - 1)) * block_bytes;
            return s;
        };
        auto put_k = [&](int live, int buf, int lane) {
            tile_store_k<kStore, kDim, kBf16>(raw, half, lane, s_k[buf] + (wave >> 1) * kBlock);
            if (lane == 0 && half == 0) s_live[buf][wave >> 1] = live;
        };
        // V of tile i before it goes to LDS: zeros for the tokens that are nobody's, and what is not finite
        auto clean_v = [&](int i, int live, int buf) {
            const int mine = live - 8 * half;
            if (mine < 8)
#pragma unroll
                for (int x = 0; x < Raw::kLoads; ++x) {
                    if constexpr (kStore == SALI_STORE_16) raw.v[x] = live_tokens(raw.v[x], mine);
                    else if constexpr (kStore == SALI_STORE_INT8) raw.vs[x] = (lane & 7) < mine ? raw.vs[x] : 0.0f;
                    else {
                        raw.vs[x] = live_tokens(raw.vs[x], mine);
                        raw.vz[x] = live_tokens(raw.vz[x], mine);
                    }
                }
            if constexpr (kStore == SALI_STORE_16) {
                bool any = false;
                if (partly_hidden(to_look_at, a.window, a.sinks, tile_at(view, i) * kTileKeys, kTileKeys)) {
                    bool odd = false;
#pragma unroll
                    for (int x = 0; x < Raw::kLoads; ++x) odd |= !Raw::none(x, lane) && any_not_finite<kBf16>(raw.v[x]);
                    any = __builtin_amdgcn_ballot_w64(odd) != 0;
                    if (any)
#pragma unroll
                        for (int x = 0; x < Raw::kLoads; ++x) {
                            if (Raw::none(x, lane)) continue;
                            u32x4 plus, minus;
                            take_apart<kBf16>(raw.v[x], raw.v[x], plus, minus);
                            uint32_t up = 0, down = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t p = plus[e], m = minus[e];
                                up |= ((p & 0xFFFFu) != 0 ? 1u : 0u) << (2 * e) | (p >> 16 != 0 ? 2u : 0u) << (2 * e);
                                down |= ((m & 0xFFFFu) != 0 ? 1u : 0u) << (2 * e) | (m >> 16 != 0 ? 2u : 0u) << (2 * e);
                            }
                            s_up[buf][wave][64 * x + lane] = (uint8_t)up;
                            s_down[buf][wave][64 * x + lane] = (uint8_t)down;
                        }
                }
                if (lane == 0) s_odd[buf][wave] = any ? 1 : 0;
            }
        };
        auto put_v = [&](int buf, int lane) { tile_store_v<kStore, kDim, kBf16>(raw, half, lane, s_v[buf] + (wave >> 1) * kBlock); };

        Source next = source(lo);
        tile_load_k<kStore, kDim>(next.block, half, lane, raw);
        tile_load_v<kStore, kDim>(next.block, half, lane, raw);

        // ---- the wave's rows
        const int row0 = unit.row_tile * kTileRows + wave * 32, rows = seq.n * group, r = row0 + col;
        const int token = (int)((uint32_t)r / (uint32_t)group), of_group = r - token * group;
        const int pos = r < rows ? seq.len - seq.n + token : -1;
        const bool some = row0 < rows;                          // uniform over the wave
        View mine = view;
        mine.first = seq.len - seq.n + (int)((uint32_t)row0 / (uint32_t)group);
        mine.last = seq.len - seq.n + (int)((uint32_t)(least(rows, row0 + 32) - 1) / (uint32_t)group);
        u32x4 q[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            q[s] = (u32x4){0u, 0u, 0u, 0u};
            if (r < rows) {
                const u32x4 v = load16(a.q.d + (int64_t)(seq.first + token) * a.q.token_bytes + (int64_t)(head * group + of_group) * a.q.head_bytes +
                                       2 * (16 * s + 8 * hh));
#pragma unroll
                for (int e = 0; e < 4; ++e) q[s][e] = (v[e] & a.q_keep) ^ a.q_flip;
            }
        }
        // keys that all of the wave's rows see: j0 .. j0 + 31 with j0 up to seen_to, and from seen_from on or all of them sinks
        const int seen_to = mine.first - 31, seen_from = a.window > 0 ? mine.last - a.window + 1 : 0, sunk_to = a.sinks - 32;
        float m = -INFINITY, l = 0.0f;
        f32x16 acc[kDt];
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[d][x] = 0.0f;
        // a bit for every value of acc: infinities found, of either sign (in LDS, since there are hardly ever any)
        if constexpr (kStore == SALI_STORE_16) {
            uint32_t none = 0;
            asm volatile("" : "+v"(none));
            s_found[0][thread] = s_found[1][thread] = none;
        }

        // 32 keys from j0 on, those of blocks 2 sub and 2 sub + 1 of the tile in `buf`
        auto step = [&](int j0, int buf, int sub) {
            const uint8_t* const k = s_k[buf] + (2 * sub + (col >> 4)) * kBlock + (hh * 16 + (col & 15)) * 16;
            const uint8_t* const v = s_v[buf] + 2 * sub * kBlock + (hh * kDim + col) * 16;
            const int live_of_block = s_live[buf][2 * sub + (lane & 1)];
            f32x16 st;
#pragma unroll
            for (int x = 0; x < 16; ++x) st[x] = 0.0f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) st = Num<kBf16>::mma32(load16(k + s * 512), q[s], st);
            // lane (row col, hh): register x has token 8 hh + x % 8 of block x / 8
            if (j0 > seen_to || (j0 < seen_from && j0 > sunk_to) || __builtin_amdgcn_ballot_w64(live_of_block < kBlockTokens) != 0) {
                const int live0 = __builtin_amdgcn_readlane(live_of_block, 0), live1 = __builtin_amdgcn_readlane(live_of_block, 1);
                // relative to the lane's first key, in place (sixteen positions of keys would be sixteen registers through the loop)
                int first_key = j0 + 8 * hh;
                asm volatile("" : "+v"(first_key));
                const Sight sight = sight_of(pos, first_key, a.window, a.sinks);
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if ((x < 8 ? live0 : live1) <= 0 || !sight.has(16 * (x / 8) + x % 8)) st[x] = -INFINITY;
            }
            float tops[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) tops[x] = fmaxf(fmaxf(st[4 * x], st[4 * x + 1]), fmaxf(st[4 * x + 2], st[4 * x + 3]));
            const float top = reference_of<kBf16>(max_over_halves(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))), a.scale2);
            const float to = top > m + Num<kBf16>::kLag ? top : m;
            if (__builtin_amdgcn_ballot_w64(to != m) != 0) {
                const float by = to != m ? __builtin_amdgcn_exp2f(m - to) : 1.0f;
                l *= by;
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int x = 0; x < 16; ++x) acc[d][x] *= by;
                m = to;
            }
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int x = 0; x < 16; ++x) st[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[x], a.scale2, -ref));
#pragma unroll
            for (int x = 0; x < 4; ++x) tops[x] = (st[4 * x] + st[4 * x + 1]) + (st[4 * x + 2] + st[4 * x + 3]);
            l += (tops[0] + tops[1]) + (tops[2] + tops[3]);
            // the weights once rounded to 16 bits, half a step each, against the sum's fp32: a second number each, as the stream has it, is half as many
            // products again where the matrix cores are what a prompt waits for, and registers that three waves a SIMD do not leave (they spill)
            u32x4 p[2];
#pragma unroll
            for (int x = 0; x < 8; ++x) p[x / 4][x % 4] = pack2<kBf16>(st[2 * x], st[2 * x + 1]);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int d = 0; d < kDt; ++d) acc[d] = Num<kBf16>::mma32(load16(v + b * kBlock + d * 512), p[b], acc[d]);
        };
        auto look_for_odd = [&](int tile0, int buf) {
            if constexpr (kStore == SALI_STORE_16) {
                const int there = lane < kTileWaves ? s_odd[buf][lane] : 0;
                if (__builtin_amdgcn_ballot_w64(there != 0) == 0) return;
                uint64_t up = 0, down = 0;
                int tid = thread;
                asm volatile("" : "+v"(tid));                   // worked out here, not kept in registers through the loop
                const int at_hh = tid >> 5 & 1;
#pragma unroll 1
                for (int w = 0; w < kTileWaves; ++w) {
                    if (s_odd[buf][w] == 0) continue;
                    const Sight sight = sight_of(pos, tile0 + 8 * w, a.window, a.sinks);
                    uint32_t seen = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) seen |= (sight.has(e) ? 1u : 0u) << e;
#pragma unroll 1
                    for (int x = 0; x < 16 * kDt; ++x) {
                        const int d = 32 * (x >> 4) + 8 * (x >> 2 & 3) + 4 * at_hh + (x & 3);
                        up |= (uint64_t)((s_up[buf][w][d] & seen) != 0) << x;
                        down |= (uint64_t)((s_down[buf][w][d] & seen) != 0) << x;
                    }
                }
                s_found[0][tid] |= up;
                s_found[1][tid] |= down;
            }
        };

        lds_barrier();                                          // all waves are through with the unit before
        put_k(next.live, 0, lane);
        clean_v(lo, next.live, 0);
        put_v(0, lane);
        next = source(lo + 1);
        tile_load_k<kStore, kDim>(next.block, half, lane, raw);
        tile_load_v<kStore, kDim>(next.block, half, lane, raw);
        for (int i = lo; i < hi; ++i) {
            const int buf = (i - lo) & 1, tile0 = tile_at(view, i) * kTileKeys;
            lds_barrier();                                      // the tile is there, and all waves are through with the other buffer
            if (some && tile0 <= mine.last) {
                step(tile0, buf, 0);
                if constexpr (kBlocks > 2)
#pragma unroll 1
                    for (int sub = 1; sub < kBlocks / 2 && tile0 + 32 * sub <= mine.last; ++sub) step(tile0 + 32 * sub, buf, sub);
                look_for_odd(tile0, buf);
            }
            if (i + 1 == hi) break;
            int here = lane;                                    // addresses worked out again, not kept in registers through the step
            asm volatile("" : "+v"(here));
            put_k(next.live, buf ^ 1, here);
            clean_v(i + 1, next.live, buf ^ 1);
            put_v(buf ^ 1, here);
            next = source(i + 2);
            tile_load_k<kStore, kDim>(next.block, half, here, raw);
            tile_load_v<kStore, kDim>(next.block, half, here, raw);
        }

        // Results with a NaN wait for the second time.  (Without it 333 of 4000 tokens six times, 8 heads, 163 us, with it 165; no difference for 8192.)
        if constexpr (kStore == SALI_STORE_16) {
            if (!look) {
                float any[4] = {};
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int x = 0; x < 16; ++x) any[x % 4] += acc[d][x];
                any[0] = (any[0] + any[1]) + (any[2] + any[3]);
                again = __builtin_amdgcn_ballot_w64(any[0] != any[0]) != 0;
            }
        }
        const bool writes = again == look;
        // ---- results: lane (row col, hh) has values 32 d + 8 k + 4 hh .. + 3
        const PagesAttend b = late_arguments<0>();
        const float sum = sum_over_halves(l);
        // (worked out again, with a lane number that the compiler does not know: through the loop it has no registers for it)
        int there = lane;
        asm volatile("" : "+v"(there));
        const int end_col = there & 31, end_hh = there >> 5;
        const int end_r = row0 + end_col;
        if (end_r < rows && writes) {
            const int end_token = (int)((uint32_t)end_r / (uint32_t)b.group), end_of_group = end_r - end_token * b.group;
            if constexpr (kStore == SALI_STORE_16) {
                const uint64_t up = s_found[0][thread], down = s_found[1][thread];
                if ((up | down) != 0)
#pragma unroll
                    for (int d = 0; d < kDt; ++d)
#pragma unroll
                        for (int x = 0; x < 16; ++x) acc[d][x] += found((up >> (16 * d + x) & 1) != 0, (down >> (16 * d + x) & 1) != 0);
            }
            if (part_of_piece >= 0) {
                // as the lanes have them, side by side: the rows' references and sums, then 16 bytes a lane
                float* const part = b.partial + ((size_t)part_of_piece * b.geom.n_kv + head) * (kTileRows * kPitch);
                if (end_hh == 0) *reinterpret_cast<float2*>(part + 2 * (wave * 32 + end_col)) = make_float2(m, sum);
                f32x4* const values = reinterpret_cast<f32x4*>(part + 4 * kTileRows) + wave * (kDt * 4 * 64) + there;
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        values[(4 * d + k) * 64] = (f32x4){acc[d][4 * k], acc[d][4 * k + 1], acc[d][4 * k + 2], acc[d][4 * k + 3]};
            } else {
                const int h = head * b.group + end_of_group;
                const int64_t row = (int64_t)(seq.first + end_token) * b.heads + h;
                const RowEnd e = row_end(m, sum, b, row);
                char* const out = b.out.d + (int64_t)(seq.first + end_token) * b.out.token_bytes + (int64_t)h * b.out.head_bytes;
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        f32x4 pr = {0.0f, 0.0f, 0.0f, 0.0f};
                        const int at = 32 * d + 8 * k + 4 * end_hh;
                        if (b.prior != nullptr) pr = *reinterpret_cast<const f32x4*>(b.prior + row * kDim + at);
                        float o[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) o[x] = joined(e, acc[d][4 * k + x], pr[x]);
                        *reinterpret_cast<u32x2*>(out + 2 * at) = (u32x2){pack2<kBf16>(o[0], o[1]), pack2<kBf16>(o[2], o[3])};
                    }
                if (end_hh == 0 && b.lse != nullptr) b.lse[row] = e.lse;
            }
        }
        if constexpr (kStore == SALI_STORE_16) {
            if (!look) {
                if (there == 0) s_nan[wave] = again ? 1 : 0;
                lds_barrier();
                look = __builtin_amdgcn_ballot_w64((there < kTileWaves ? s_nan[there] : 0) != 0) != 0;
                if (look) continue;
            }
            look = again = false;
        }
        ++piece;
    }
}

// Joins the parts of cut row tiles: grid (merges * n_kv at most, a block's waves of 32 rows and 32 values / 4), a lane as in the tile's results.  Bound by the
// bytes of the partial results: 13 us for 512 rows by 4100 keys, 32 heads of 128 values in stretches (48 MB)
template <int kDim, bool kBf16, int kWaves>
__global__ __launch_bounds__(256) void k_pages_tile_merge(PagesAttend a) {
    constexpr int kPitch = kDim + 4, kDt = kDim / 32, kTileRows = tile_rows(kWaves);
    const TileScratch& t = *reinterpret_cast<const TileScratch*>(a.records);
    const int n_kv = a.geom.n_kv;
    const int nth = (int)(blockIdx.x / (uint32_t)n_kv), head = (int)blockIdx.x - nth * n_kv;
    if (nth >= t.plan.n_merges) return;
    const TileMerge rec = t.merges[nth];
    const PageSeq seq = load_seq(a.seqs, a.geom, rec.seq, false);
    const int at_wave = (int)blockIdx.y * 4 + (int)(threadIdx.x >> 6), wave = at_wave / kDt, d = at_wave % kDt, lane = threadIdx.x & 63, hh = lane >> 5;
    const int in_tile = wave * 32 + (lane & 31), r = rec.row_tile * kTileRows + in_tile;
    if (r >= seq.n * a.group) return;
    const int token = (int)((uint32_t)r / (uint32_t)a.group), h = head * a.group + (r - token * a.group);
    const int64_t row = (int64_t)(seq.first + token) * a.heads + h;
    f32x4 pr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        pr[k] = a.prior != nullptr ? *reinterpret_cast<const f32x4*>(a.prior + row * kDim + 32 * d + 8 * k + 4 * hh) : (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kFlight = 3;              // parts under way
    const size_t step = (size_t)n_kv * kTileRows * kPitch;
    const float* const first = a.partial + ((size_t)rec.part * n_kv + head) * (kTileRows * kPitch);
    const int values = 4 * kTileRows + 4 * ((wave * kDt + d) * (4 * 64) + lane);
    float m = -INFINITY, l = 0.0f;
    f32x4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = 0; i0 < rec.parts; i0 += kFlight) {
        float2 ml[kFlight];
        f32x4 v[kFlight][4];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const float* const part = first + step * (size_t)min(i0 + i, rec.parts - 1);
            ml[i] = *reinterpret_cast<const float2*>(part + 2 * in_tile);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = *reinterpret_cast<const f32x4*>(part + values + k * 256);
        }
        float to = m;
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (i0 + i >= rec.parts) ml[i].y = 0.0f;
            to = ml[i].y == 0.0f ? to : fmaxf(to, ml[i].x);         // 0: nothing seen
        }
        const float by = l == 0.0f ? 0.0f : not_zero(__builtin_amdgcn_exp2f(m - to));
        l = l == 0.0f ? 0.0f : l * by;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[k][e] = by == 0.0f ? 0.0f : acc[k][e] * by;
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const bool none = ml[i].y == 0.0f;
            const float pby = none ? 0.0f : not_zero(__builtin_amdgcn_exp2f(ml[i].x - to));
            l += none ? 0.0f : ml[i].y * pby;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[k][e] += pby == 0.0f ? 0.0f : v[i][k][e] * pby;
        }
        m = to;
    }
    const RowEnd e = row_end(m, l, a, row);
    char* const out = a.out.d + (int64_t)(seq.first + token) * a.out.token_bytes + (int64_t)h * a.out.head_bytes;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float o[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) o[x] = joined(e, acc[k][x], pr[k][x]);
        *reinterpret_cast<u32x2*>(out + 2 * (32 * d + 8 * k + 4 * hh)) = (u32x2){pack2<kBf16>(o[0], o[1]), pack2<kBf16>(o[2], o[3])};
    }
    if (d == 0 && hh == 0 && a.lse != nullptr) a.lse[row] = e.lse;
}

}  // namespace

}  // namespace sali
