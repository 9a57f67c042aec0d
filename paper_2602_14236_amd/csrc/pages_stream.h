// Attention of few new tokens a sequence (up to 32 rows: single tokens, drafts, short texts): a stream over the pages.
//
// Few rows make the products thin, so the kernel is bound by the bytes of K and V.  Every wave takes tiles of its own straight from memory into the
// operands of the 16x16x32 products, no LDS and no barrier between tiles; the next tile's K is asked for when this one's has been multiplied, V
// likewise, so that a tile (16 KB of 16-bit values) is always under way.
//
// The work of all sequences and K/V heads is one row of tiles, cut into equal stretches, one a block: whatever the lengths, all
// blocks have the same number of tiles, give or take one.  A block's stretch may end inside one pair of sequence and head and hold
// whole ones; its waves split each such segment, meet in LDS, and leave a result (whole pairs) or a partial one, of which a block has
// at most two, at its ends.  A second launch joins a pair's partial results.
//
// Measured: one token over 131072 keys, 8 heads of 128 values in 16 bits, 537 MB in 96 us, 5.6 TB/s (a copy of 2 GiB: 4.9); 48 sequences of up to 8192
// keys in 8 bits 96 us, 5.1 TB/s.  4 bits: 16 sequences under a window of 4096 keys 42 us, 2.2 TB/s; the 800 vector instructions a tile that unpack them
// keep the vector units busy for half of that, waves wait for a third of it, and neither is the bound alone.  Short texts are bound by the chain of a launch,
// the lengths, the page table, K, V and the joining of the waves: 10.8 us for 777 keys.
#pragma once

#include "pages_attn.h"

namespace sali {

namespace {

constexpr int kComputeUnits = 256;
constexpr int kStreamMostBlocks = 3 * kComputeUnits;

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
    float vs[kDim / 32];
};
template <int kDim>
struct StreamRaw<SALI_STORE_INT4, kDim> {
    u32x4 k[2];                             // head dim 64: half of it
    u32x2 v[kDim / 32];
    float ks[2];
    uint16_t kz[2];
    float vs[kDim / 32];
    uint16_t vz[kDim / 32];
};

__device__ __forceinline__ u32x4 stream16(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4*>(p)); }

template <int kStore, int kDim>
__device__ __forceinline__ void stream_load_k(const char* b0, const char* b1, int lane, StreamRaw<kStore, kDim>& r) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const char* b = j == 0 ? b0 : b1;
        if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
            for (int t = 0; t < kDim / 32; ++t) r.k[j][t] = stream16(b + (uint32_t)(t * 1024 + lane * 16));
        } else if constexpr (kStore == SALI_STORE_INT8) {
#pragma unroll
            for (int u = 0; u < kDim / 64; ++u) {
                r.k[j][u] = stream16(b + (uint32_t)(u * 1024 + lane * 16));
                r.ks[j][u] = *reinterpret_cast<const float*>(b + kAt.ks + (uint32_t)((2 * u + (lane >> 5)) * 64 + (lane & 15) * 4));
            }
        } else if constexpr (kDim == 128) {
            r.k[j] = stream16(b + (uint32_t)(lane * 16));
            r.ks[j] = *reinterpret_cast<const float*>(b + kAt.ks + (uint32_t)(lane * 4));
            r.kz[j] = *reinterpret_cast<const uint16_t*>(b + kAt.kz + (uint32_t)(lane * 2));
        } else {
            const uint32_t at = (uint32_t)((lane >> 5) * 16 + (lane & 15));
            const u32x2 c = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(b + at * 16 + (uint32_t)(lane >> 4 & 1) * 8));
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
        for (int f = 0; f < kDim / 16; ++f) r.v[f] = stream16(b + kAt.v + (a * kDim + 16 * f + i) * 16);
    } else {
#pragma unroll
        for (int g = 0; g < kDim / 32; ++g) {
            if constexpr (kStore == SALI_STORE_INT8) r.v[g] = stream16(b + kAt.v + (a * kDim + 32 * g + 2 * i) * 8);
            else r.v[g] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(b + kAt.v + ((a * (kDim / 32) + g) * 16 + i) * 8));
            const uint32_t token = g * 16 + 8 * a + (i & 7);
            r.vs[g] = *reinterpret_cast<const float*>(b + kAt.vs + token * 4);
            if constexpr (kStore == SALI_STORE_INT4) r.vz[g] = *reinterpret_cast<const uint16_t*>(b + kAt.vz + token * 2);
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
        return row_values8<kBf16>(lo, hi, r.vs[f / 2]);
    } else {
        const int shift = (f & 1) * 4;
        const uint32_t lo = r.v[f / 2].x, hi = r.v[f / 2].y;
        return row_values4<kBf16>(lo >> shift & 0x0F0F0F0Fu, hi >> shift & 0x0F0F0F0Fu, r.vs[f / 2], low_half<kBf16>(r.vz[f / 2]));
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

// The parts of a pair, as the launch that joins them finds them: the first in `slot`, the others the first segments of the following
// blocks.  A block leaves a record of the pair whose first part is its last segment, parts = 0 if there is none.
struct StreamRecord {
    int32_t seq, head, slot, parts;
};

// Rows r0 .. r0 + n_rows - 1 of a pair from its parts, by a block of kThreads: groups of threads that have two values of a row each share the parts,
// sixteen in flight; meanwhile the parts' references and sums give their weights (a wave a row).
template <int kDim, int kThreads>
constexpr int join_lds(int rows, int parts) { return rows * (parts + 2) + 2 * (kThreads > rows * (kDim / 2) ? kThreads : rows * (kDim / 2)); }      // floats
template <int kDim, bool kBf16, int kThreads>
__device__ __forceinline__ void join_parts(const PagesAttend& a, const StreamRecord& rec, const PageSeq& seq, int kernel_rows, int r0, int n_rows, int tid, float* lds) {
    constexpr int kPitch = kDim + 4, kPairs = kDim / 2, kFlight = 16;
    const int wave = tid >> 6, lane = tid & 63;
    float* const s_top = lds;
    float* const s_sum = lds + n_rows;
    float* const s_weight = lds + 2 * n_rows;               // [n_rows][parts]
    float* const s_part = s_weight + n_rows * rec.parts;    // [groups][n_rows][kDim]
    const int items = n_rows * kPairs, groups = max(1, kThreads / items);
    const int group = min(tid / items, groups - 1);
    // offsets in the area of partial results, which is far below 4 GB
    const char* const area = reinterpret_cast<const char*>(a.partial);
    const uint32_t slot_bytes = (uint32_t)kernel_rows * kPitch * 4u, first_at = (uint32_t)rec.slot * slot_bytes, others_at = (uint32_t)(rec.slot & ~1) * slot_bytes;
    auto row_of_part = [&](int part, int row) { return (part == 0 ? first_at : others_at + (uint32_t)part * (2u * slot_bytes)) + (uint32_t)(r0 + row) * (kPitch * 4u); };
    float2 v[kFlight];
    auto ask = [&](int item, int k) {
        const int row = item / kPairs;
        const uint32_t in_row = 16u + (uint32_t)(item % kPairs) * 8u;
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            v[i] = *reinterpret_cast<const float2*>(area + (row_of_part(min(group + groups * (k + i), rec.parts - 1), row) + in_row));
    };
    const bool helps = tid < items * groups;
    const int item0 = tid - group * items;
    if (helps) ask(min(item0, items - 1), 0);
    for (int x = wave; x < n_rows; x += kThreads / 64) {
        float top = -INFINITY, sum = 0.0f;
        for (int i = lane; i < rec.parts; i += 64) {
            const float2 ml = *reinterpret_cast<const float2*>(area + row_of_part(i, x));
            const float m = ml.x, l = ml.y;
            s_weight[x * rec.parts + i] = l == 0.0f ? -INFINITY : m;
            const float to = l == 0.0f ? top : fmaxf(top, m);
            if (l != 0.0f) sum = (sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f(top - to)) + l * __builtin_amdgcn_exp2f(m - to);
            top = to;
        }
        float all = top;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) all = fmaxf(all, __shfl_xor(all, off));
        sum = sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f(top - all);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
        for (int i = lane; i < rec.parts; i += 64) {
            const float m = s_weight[x * rec.parts + i];
            s_weight[x * rec.parts + i] = m == -INFINITY && sum == sum ? 0.0f : not_zero(__builtin_amdgcn_exp2f(m - all));
        }
        if (lane == 0) {
            s_top[x] = all;
            s_sum[x] = sum;
        }
    }
    __syncthreads();
    for (int item = item0; helps && item < items; item += kThreads) {
        if (item != item0) ask(item, 0);
        const float* const weight = s_weight + item / kPairs * rec.parts;
        float o0 = 0.0f, o1 = 0.0f;
        for (int k = 0; group + groups * k < rec.parts; k += kFlight) {
            if (k > 0) ask(item, k);
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                const int part = group + groups * (k + i);
                const float w = part < rec.parts ? weight[part] : 0.0f;
                const bool none = w == 0.0f;                // nothing seen
                o0 = __builtin_fmaf(none ? 0.0f : v[i].x, w, o0);
                o1 = __builtin_fmaf(none ? 0.0f : v[i].y, w, o1);
            }
        }
        s_part[(group * items + item) * 2] = o0;
        s_part[(group * items + item) * 2 + 1] = o1;
    }
    __syncthreads();
    for (int item = tid; item < items; item += kThreads) {
        float o0 = 0.0f, o1 = 0.0f;
        for (int g = 0; g < groups; ++g) {
            o0 += s_part[(g * items + item) * 2];
            o1 += s_part[(g * items + item) * 2 + 1];
        }
        const int x = item / kPairs, d = item % kPairs * 2, r = r0 + x;
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

// bytes of the kernel's leading arguments, where its struct lies
constexpr int kStreamArgsAt = 3 * 8 + 10 * 4;
static_assert(kStreamArgsAt % alignof(PagesAttend) == 0, "where the struct lies");

// What a block works on.
//   pairs: grid (K/V heads, sequences), a block the one pair; for short sequences, where parts and their joining would cost more than they bring.
//          us of pairs and of stretches: 8 sequences of 300 keys, 32 heads, 10.4 and 17.6; 1 of 1000, 8 heads, 10.4 and 12.1; 1 of 4000, 8 heads, 20.7
//          and 15.8; 64 of 300, 32 heads, 89 and 66
//   stretches: of all tiles; a launch of its own joins the parts of cut pairs (k_pages_stream_merge)
enum class StreamMode { pairs, stretches };
// Waves of a block, and waves a SIMD that their registers leave room for.  Stretches: small blocks, several of which share a compute unit, so that one
// walks on while another is between two pairs: 48 sequences in 8 bits 95 us, with one block of eight waves a compute unit 116.
constexpr int stream_waves(StreamMode mode) { return mode == StreamMode::pairs ? 8 : 4; }
constexpr int stream_occupancy(int store, int sets, StreamMode mode) { return store != SALI_STORE_16 && sets == 1 && mode == StreamMode::stretches ? 3 : 2; }

// The leading arguments come in registers: what the first loads depend on.
template <int kStore, int kDim, bool kBf16, int kSets, StreamMode kMode>
__global__ __launch_bounds__(64 * stream_waves(kMode)) __attribute__((amdgpu_waves_per_eu(stream_occupancy(kStore, kSets, kMode), stream_occupancy(kStore, kSets, kMode))))
void k_pages_stream(
    const int32_t* __restrict__ starts, const int32_t* __restrict__ lengths, const int32_t* __restrict__ tables, int n_seqs, int width, int n_tokens, int max_q,
    int max_kv, int blocks_log2, int window, int sinks, int group, int n_kv, PagesAttend a, int rows_max, int min_tiles) {
    constexpr int kStreamWaves = stream_waves(kMode), kRows = 16 * kSets, kSteps = kDim / 32, kFs = kDim / 16, kPitch = kDim + 4;
    constexpr bool kStretches = kMode != StreamMode::pairs;
    __shared__ __align__(16) float s_acc[kStreamWaves][kRows][kPitch];
    __shared__ float s_m[kStreamWaves][kRows], s_l[kStreamWaves][kRows];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, hh = lane >> 4;
    const int page_tokens = kBlockTokens << blocks_log2;
    const int64_t in_table = (int64_t)width * page_tokens, room = in_table < max_kv ? in_table : max_kv;
    auto read = [&](int s, bool& fits) -> PageSeq {
        const int first = starts[s], next = starts[s + 1], len = lengths[s];
        fits = page_seq_holds(first, next, len, n_tokens, max_q, room);
        return {first, fits ? next - first : 0, len};
    };
    auto view_of_seq = [&](const PageSeq& q) { return view_of<kTileTokens>(q.len - q.n, q.len - 1, window, sinks); };
    // the pages from `page0` on, one a lane
    int page0 = 0, page_of_lane = -1;

    int s, head, done = 0;                  // done: tiles of the pair before the block's
    PageSeq seq = {0, 0, 0};
    uint32_t at = 0, end = 0, total = 0, blocks = 1;
    StreamRecord record = {0, 0, 0, 0};
    const StartFalls falls_of_pair(starts, kStretches ? 0 : n_seqs, lane, 64);
    if constexpr (!kStretches) {
        head = blockIdx.x;
        s = blockIdx.y;
        if (width > 0) page_of_lane = tables[(int64_t)s * width + min(lane, width - 1)];      // on their way with the lengths
        bool fits;
        seq = read(s, fits);
        if (!fits && head == 0 && threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        if (!in_stream(seq, group, rows_max)) return;
        end = (uint32_t)view_of_seq(seq).tiles;
    } else {
        // the block's stretch: every wave finds it by itself, a sequence a lane
        page0 = -64;
        bool bad = false, falls = false;
        auto lane_seq = [&](int i) -> PageSeq {
            PageSeq q = {0, 0, 0};
            if (i >= n_seqs) return q;
            bool fits;
            q = read(i, fits);
            bad |= !fits;
            falls |= !fits && starts[i] > starts[i + 1];
            return q;
        };
        auto tiles_of = [&](const PageSeq& q) { return in_stream(q, group, rows_max) ? view_of_seq(q).tiles : 0; };
        const PageSeq first_mine = lane_seq(lane);
        const int first_tiles = tiles_of(first_mine);
        int own = first_tiles;
#pragma unroll 4
        for (int i = 64 + lane; i < n_seqs; i += 64) own += tiles_of(lane_seq(i));
        total = (uint32_t)__builtin_amdgcn_readlane(wave_scan(own), 63) * (uint32_t)n_kv;
        if (__builtin_amdgcn_ballot_w64(falls) != 0) total = 0;
        if (bad && blockIdx.x == 0 && wave == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        blocks = max(1u, min(gridDim.x, total / (uint32_t)min_tiles));
        if (blockIdx.x >= blocks || total == 0) {
            if (threadIdx.x == 0) reinterpret_cast<StreamRecord*>(late_arguments<kStreamArgsAt>().records)[blockIdx.x] = record;
            return;
        }
        const Stretches cut(total, blocks);
        at = __builtin_amdgcn_readfirstlane(cut.start(blockIdx.x));
        end = __builtin_amdgcn_readfirstlane(cut.start(blockIdx.x + 1));
        uint32_t before = 0;                // tiles a head of the sequences before it
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
            if (base >= n_seqs) {                           // the batch changed while it was read
                if (threadIdx.x == 0) reinterpret_cast<StreamRecord*>(late_arguments<kStreamArgsAt>().records)[blockIdx.x] = record;
                return;
            }
            q = lane_seq(base + lane);
            t = tiles_of(q);
        }
        const int tiles = view_of_seq(seq).tiles;
        head = (int)((at - before * (uint32_t)n_kv) / (uint32_t)tiles);
        done = (int)(at - before * (uint32_t)n_kv) - head * tiles;
    }

    bool first_segment = true;
    for (;;) {
        // the same for all lanes, and to be in scalar registers
        at = __builtin_amdgcn_readfirstlane(at);
        done = __builtin_amdgcn_readfirstlane(done);
        s = __builtin_amdgcn_readfirstlane(s);
        head = __builtin_amdgcn_readfirstlane(head);
        seq = {__builtin_amdgcn_readfirstlane(seq.first), __builtin_amdgcn_readfirstlane(seq.n), __builtin_amdgcn_readfirstlane(seq.len)};
        if (at >= end) break;
        const View view = view_of_seq(seq);
        const int todo = min(view.tiles - done, (int)(end - at));
        const int rows = seq.n * group;
        const int32_t* table = tables + (int64_t)s * width;
        const int pages = (seq.len + page_tokens - 1) >> (blocks_log2 + 4);
        const char* const heads = a.geom.pool + (uint64_t)head * a.geom.head_bytes;
        constexpr uint32_t block_bytes = block_layout(kStore, kDim).bytes;
        struct Tile {
            const char* b[2];
            int live[2];                     // tokens of the block that a row may see: none of a page that is none
        };
        auto locate = [&](int i) -> Tile {
            Tile t;
            const int tile = tile_at(view, i);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int block = 2 * tile + j, index = block >> blocks_log2;
                if ((unsigned)(index - page0) >= 64u) {
                    page0 = index;
                    page_of_lane = index + lane < pages ? table[index + lane] : -1;
                    asm volatile("" : "+v"(page_of_lane));      // waited for here: a wait behind the branch would be one for K and V too
                }
                int page = __builtin_amdgcn_readlane(page_of_lane, index - page0);
                t.live[j] = min(kBlockTokens, seq.len - block * kBlockTokens);
                if (t.live[j] <= 0) {
                    page = 0;                // behind the sequence's end
                } else if ((unsigned)page >= (unsigned)a.geom.n_pages) {
                    if (lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                    t.live[j] = 0;
                    page = 0;
                }
                t.b[j] = heads + (uint64_t)page * a.geom.page_bytes + (uint32_t)(block & ((1 << blocks_log2) - 1)) * block_bytes;
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
        if constexpr (!kStretches) {        // the starts are here since the page table is
            if (__builtin_amdgcn_ballot_w64(falls_of_pair.some()) != 0) {
                if (threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
                return;
            }
        }
        u32x4 q[kSets][kSteps];
        int pos[kSets];
#pragma unroll
        for (int c = 0; c < kSets; ++c) {
            int r = 16 * c + col;
            asm volatile("" : "+v"(r));     // not worked out ahead of time, which would take registers
            const int token = r / group, g = r - token * group;
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
            const bool masked = now.live[0] < kBlockTokens || now.live[1] < kBlockTokens || partly_hidden(view, window, sinks, j0, kTileTokens);
            if (masked) {
                // relative to the lane's first key, in place
                int first_key = j0 + 8 * (hh & 1) + 4 * (hh >> 1);
                asm volatile("" : "+v"(first_key));
#pragma unroll
                for (int c = 0; c < kSets; ++c) {
                    const Sight sight = sight_of(pos[c], first_key, window, sinks);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (now.live[j] <= 0 || !sight.has(16 * j + r)) s2[c][j][r] = -INFINITY;
                }
            }
            // the weights in two 16-bit numbers each, what the first one's rounding leaves in the second: the matrix cores have time for both
            u32x4 p[kSets], p_rest[kSets];
#pragma unroll
            for (int c = 0; c < kSets; ++c) {
                float top = fmaxf(fmaxf(fmaxf(s2[c][0][0], s2[c][0][1]), fmaxf(s2[c][0][2], s2[c][0][3])),
                                  fmaxf(fmaxf(s2[c][1][0], s2[c][1][1]), fmaxf(s2[c][1][2], s2[c][1][3])));
                top = reference_of<kBf16>(max_over_quarters(top), a.scale2);
                const float to = top > m[c] + Num<kBf16>::kLag ? top : m[c];
                if (__builtin_amdgcn_ballot_w64(to != m[c]) != 0) {
                    const float by = to != m[c] ? __builtin_amdgcn_exp2f(m[c] - to) : 1.0f;
                    l[c] *= by;
#pragma unroll
                    for (int f = 0; f < kFs; ++f) acc[c][f] *= by;
                    m[c] = to;
                }
                const float ref = m[c] == -INFINITY ? 0.0f : m[c];
                uint32_t w[2][2], rest[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float e[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s2[c][j][r], a.scale2, -ref));
                        l[c] += e[r];
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        w[j][r] = pack2<kBf16>(e[2 * r], e[2 * r + 1]);
                        rest[j][r] = pack2<kBf16>(e[2 * r] - low_half<kBf16>(w[j][r]), e[2 * r + 1] - high_half<kBf16>(w[j][r]));
                    }
                }
                // to the lanes that hold the same tokens of V: quarter hh takes tokens 8 (hh % 2) .. + 7 of block hh / 2
                const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                p[c] = (u32x4){(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
                const auto xr = __builtin_amdgcn_permlane32_swap(rest[0][0], rest[1][0], false, false);
                const auto yr = __builtin_amdgcn_permlane32_swap(rest[0][1], rest[1][1], false, false);
                p_rest[c] = (u32x4){(uint32_t)xr[0], (uint32_t)yr[0], (uint32_t)xr[1], (uint32_t)yr[1]};
            }
            // (16 bits: every tile, since what the second weight is multiplied with has to be finite in all of them)
            if (masked || kStore == SALI_STORE_16) {
                const int live = (hh < 2 ? now.live[0] : now.live[1]) - 8 * (hh & 1);
                if constexpr (kStore != SALI_STORE_16) {
#pragma unroll
                    for (int g = 0; g < kDim / 32; ++g) {
                        raw.vs[g] = (lane & 7) < live ? raw.vs[g] : 0.0f;
                        if constexpr (kStore == SALI_STORE_INT4) raw.vz[g] = (lane & 7) < live ? raw.vz[g] : 0;
                    }
                } else {
                    // the matrix cores look: 0 times an infinity or NaN is a NaN, the sum of all others times 0 is 0
                    f32x4 zeros = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int f = 0; f < kFs; ++f) {
                        if (masked) raw.v[f] = live_tokens(raw.v[f], live);
                        zeros = Num<kBf16>::mma16(raw.v[f], (u32x4){0u, 0u, 0u, 0u}, zeros);
                    }
                    const bool odd = !((zeros[0] + zeros[1]) + (zeros[2] + zeros[3]) == 0.0f);
                    if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                        u32x4 seen[kSets];
#pragma unroll
                        for (int c = 0; c < kSets; ++c) {
                            const Sight sight = sight_of(pos[c], j0 + 16 * (hh >> 1) + 8 * (hh & 1), window, sinks);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                seen[c][e] = (2 * e < live && sight.has(2 * e) ? (uint32_t)Num<kBf16>::kOne : 0u) |
                                             (2 * e + 1 < live && sight.has(2 * e + 1) ? (uint32_t)Num<kBf16>::kOne << 16 : 0u);
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
                for (int c = 0; c < kSets; ++c) acc[c][f] = Num<kBf16>::mma16(vf, p_rest[c], Num<kBf16>::mma16(vf, p[c], acc[c][f]));
            }
            stream_load_v<kStore, kDim>(next.b[0], next.b[1], lane, raw);
            now = next;
        }

        // ---- the waves meet
        // (from here on with a thread number that the compiler does not know: it would work out all of this before the loop and have no registers for it)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
#pragma unroll
        for (int c = 0; c < kSets; ++c) {
            const int r = 16 * c + (tid & 15);
            const float sum = sum_over_quarters(l[c]);
            if (r >= rows) continue;
            if constexpr (kStore == SALI_STORE_16)
                if ((up[c] | down[c]) != 0)
#pragma unroll
                    for (int f = 0; f < kFs; ++f)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[c][f][e] += found((up[c] >> (4 * f + e) & 1) != 0, (down[c] >> (4 * f + e) & 1) != 0);
            if ((tid >> 4 & 3) == 0) {
                s_m[wave][r] = m[c];
                s_l[wave][r] = sum;
            }
#pragma unroll
            for (int f = 0; f < kFs; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_acc[wave][r][stream_v_value<kStore>(f, 4 * (tid >> 4 & 3) + e)] = acc[c][f][e];
        }
        __syncthreads();
        const PagesAttend b = late_arguments<kStreamArgsAt>();
        const bool whole = todo == view.tiles;
        const int slot = 2 * (int)blockIdx.x + (first_segment ? 0 : 1);
        for (int idx = tid; idx < rows * (kDim / 4); idx += 64 * kStreamWaves) {
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
                const float by = not_zero(__builtin_amdgcn_exp2f(mw - top));
                sum += s_l[w][r] * by;
                o += *reinterpret_cast<const f32x4*>(&s_acc[w][r][d]) * by;
            }
            if (kStretches && !whole) {
                float* part = b.partial + ((size_t)slot * kRows + r) * kPitch;
                *reinterpret_cast<f32x4*>(part + 4 + d) = o;
                if (d == 0) *reinterpret_cast<float2*>(part) = make_float2(top, sum);
                continue;
            }
            const int token = r / group, h = head * group + (r - token * group);
            const int64_t row = (int64_t)(seq.first + token) * b.heads + h;
            const RowEnd e = row_end(top, sum, b, row);
            f32x4 pr = {0.0f, 0.0f, 0.0f, 0.0f};
            if (b.prior != nullptr) pr = *reinterpret_cast<const f32x4*>(b.prior + row * kDim + d);
            const u32x2 v = {pack2<kBf16>(joined(e, o[0], pr[0]), joined(e, o[1], pr[1])), pack2<kBf16>(joined(e, o[2], pr[2]), joined(e, o[3], pr[3]))};
            *reinterpret_cast<u32x2*>(b.out.d + (int64_t)(seq.first + token) * b.out.token_bytes + (int64_t)h * b.out.head_bytes + 2 * d) = v;
            if (d == 0 && b.lse != nullptr) b.lse[row] = e.lse;
        }
        if (kStretches && !whole && done == 0) {
            // the pair's first part, in the block's last segment; the following blocks have the others
            const Stretches cut(total, blocks);
            record = {s, head, slot, (int)(cut.of(at + (uint32_t)view.tiles - 1u) - blockIdx.x) + 1};
        }
        if constexpr (!kStretches) return;
        __syncthreads();

        at += todo;
        first_segment = false;
        done += todo;
        if (done == view.tiles && at < end) {
            done = 0;
            if (++head == n_kv) {
                head = 0;
                bool fits;
                do {
                    if (++s >= n_seqs) break;
                    seq = read(s, fits);
                } while (!in_stream(seq, group, rows_max));
                if (s >= n_seqs) break;
                page0 = -64;
            }
        }
    }
    if (threadIdx.x == 0) reinterpret_cast<StreamRecord*>(late_arguments<kStreamArgsAt>().records)[blockIdx.x] = record;
}

// Joins the parts of the pairs, four rows a block: grid (blocks of the stream, rows / 4)
template <int kDim, bool kBf16>
__global__ __launch_bounds__(256) void k_pages_stream_merge(PagesAttend a, int kernel_rows) {
    __shared__ float s_join[join_lds<kDim, 256>(4, kStreamMostBlocks)];
    const StreamRecord rec = reinterpret_cast<const StreamRecord*>(a.records)[blockIdx.x];
    if (rec.parts == 0) return;
    bool fits;
    const PageSeq seq = read_seq(a.seqs, a.geom, rec.seq, fits);
    const int r0 = 4 * (int)blockIdx.y;
    if (r0 >= seq.n * a.group) return;
    join_parts<kDim, kBf16, 256>(a, rec, seq, kernel_rows, r0, min(4, seq.n * a.group - r0), threadIdx.x, s_join);
}

}  // namespace

}  // namespace sali
