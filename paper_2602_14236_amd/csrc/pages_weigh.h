// What attention weight keys had: for every key of a sequence and K/V head, the sum of exp(s - lse) over the new tokens that see it and the query heads of the group (gfx950).
//
// Rows, scores, masks and tiles of 32 keys are those of attention (pages_attn.h); with lse at hand there is no maximum to find, no second product and
// nothing to join: keys stay with a wave, which walks the rows that see them and adds the weights up in fp32, always in the same order.
//
// Three kernels, by rows (new tokens times heads of a group, as far as the batch's sizes tell):
//   up to 32   k_pages_weigh_stream  bound by K's bytes: a wave has the rows' queries in registers and walks tiles, the next one's K on its way.  16 texts of up to 8192
//                                    keys, 8 heads of 128 in 8 bits, one token each: 88 MB in 24 us, 3.6 TB/s
//   up to 256  k_pages_weigh_few     the same with 32x32 products, the rows in LDS.  32 tokens, 4 heads each over 20001 and 10700 keys in 4 bits, 8 heads: 21.6 us, half of it
//                                    the chain of a launch, lengths, page table, K and the first results
//   more       k_pages_weigh_tile    keys in registers, rows through LDS, three steps of 64 on their way past the registers; in chunks where there are fewer keys than the chip
//                                    holds, whose sums a launch of its own joins.  8192 causal tokens, 32 heads over 8 of 128: 343 us, 800 TFLOP/s (a large library product: 1369).
//                                    What it waits for there: products alone 181 us, weights alone 229, LDS reads 122 of both; products of one half step and weights of
//                                    the one before are side by side, and two blocks of eight waves a compute unit.  64 keys a wave, half the reads of LDS: 351 to 364
//
// Under a window the first two walk all of a text's keys and leave out what is out of sight only then: 16 texts of 20000 keys in 16 bits, 8 heads, one token each, take 125 us
// with a window of 1024 as without one, 20 times the bytes that are in sight.
#pragma once

#include "pages_stream.h"

namespace sali {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// sum over the 16 lanes of a row, in all of them
__device__ __forceinline__ float sum_over_row(float v) {
#define SALI_ROR(n) __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + n, 0xF, 0xF, true))
    v += SALI_ROR(8);
    v += SALI_ROR(4);
    v += SALI_ROR(2);
    v += SALI_ROR(1);
#undef SALI_ROR
    return v;
}

// A sequence's blocks and weights, of one K/V head
struct WeighSeq {
    const int32_t* table;
    int32_t len, first;                     // tokens; the first new one's position
    // where a block of 16 tokens lies and its weights; a block that is none, or of a page that is none: weights NULL
    __device__ __forceinline__ const char* block(const PagesWeigh& a, int head, int block, int page, float*& weights) const {
        const int in_page = block & ((1 << a.geom.blocks_log2) - 1);
        const bool is = block * kBlockTokens < len && (unsigned)page < (unsigned)a.geom.n_pages;
        weights = is ? a.weights + (((int64_t)page * a.geom.n_kv + head) << (a.geom.blocks_log2 + 4)) + in_page * kBlockTokens : nullptr;
        return a.geom.pool + (uint64_t)(is ? page : 0) * a.geom.page_bytes + (uint64_t)head * a.geom.head_bytes + (uint32_t)in_page * (a.geom.head_bytes >> a.geom.blocks_log2);
    }
    // sums of four keys from position `at` on, the first of four of a block
    __device__ __forceinline__ void put(const PagesWeigh& a, float* weights, int at, f32x4 sum) const {
        if (weights == nullptr) return;
        float* const to = weights + (at & 15);
        if (at + 3 < first || (at >= first && at + 3 < len) || (!a.add && at + 3 < len)) {
            f32x4* const all = reinterpret_cast<f32x4*>(to);
            *all = a.add && at + 3 < first ? *all + sum : sum;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < len) to[e] = a.add && at + e < first ? to[e] + sum[e] : sum[e];
    }
};

// ---- few rows
constexpr int kWeighStreamWaves = 4;

// `blocks` thread blocks a sequence and head, a wave `each` tiles of 32 keys; up to 16 kSets rows
template <int kStore, int kDim, bool kBf16, int kSets>
__global__ __launch_bounds__(64 * kWeighStreamWaves) void k_pages_weigh_stream(PagesWeigh a, int blocks, int each) {
    constexpr int kSteps = kDim / 32;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, hh = lane >> 4;
    const int head = (int)(blockIdx.x % (uint32_t)a.geom.n_kv), nth = (int)(blockIdx.x / (uint32_t)a.geom.n_kv), s = nth / blocks, nth_of_seq = nth - s * blocks;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, lane, 64);
    const int lo = (nth_of_seq * kWeighStreamWaves + wave) * each, shift = a.geom.blocks_log2;
    // the page numbers of the wave's blocks, one a lane, on their way with the lengths
    int page_of_lane = -1;
    const int64_t index0 = (int64_t)(2 * lo) >> shift;
    if (index0 + lane < a.seqs.width) page_of_lane = a.seqs.table[(int64_t)s * a.seqs.width + index0 + lane];
    const PageSeq seq = load_seq(a.seqs, a.geom, s, nth_of_seq == 0 && head == 0 && threadIdx.x == 0);
    if (seq.n == 0) {
        if (nth_of_seq == 0 && head == 0 && __builtin_amdgcn_ballot_w64(falls.some()) != 0 && threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    const WeighSeq w = {nullptr, seq.len, seq.len - seq.n};
    const int tiles = (seq.len + kTileTokens - 1) / kTileTokens, hi = min(lo + each, tiles);
    if (lo >= hi) return;
    struct Tile {
        const char* b[2];
        float* w[2];
    };
    auto locate = [&](int tile) -> Tile {
        Tile t;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int block = 2 * tile + j, page = __builtin_amdgcn_readlane(page_of_lane, (int)((block >> shift) - index0));
            t.b[j] = w.block(a, head, block, page, t.w[j]);
            if (t.w[j] == nullptr && block * kBlockTokens < seq.len && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
        }
        return t;
    };
    StreamRaw<kStore, kDim> raw;
    Tile now = locate(lo);
    stream_load_k<kStore, kDim>(now.b[0], now.b[1], lane, raw);
    const int rows = seq.n * a.group;
    u32x4 q[kSets][kSteps];
    float lse2[kSets];
    int pos[kSets];                         // -1: a row that is none, or saw nothing
#pragma unroll
    for (int c = 0; c < kSets; ++c) {
        const int r = 16 * c + col, token = r / a.group, g = r - token * a.group;
        pos[c] = -1;
        lse2[c] = 0.0f;
#pragma unroll
        for (int t = 0; t < kSteps; ++t) q[c][t] = (u32x4){0u, 0u, 0u, 0u};
        if (r >= rows) continue;
        const float lse = a.lse[(int64_t)(seq.first + token) * a.heads + head * a.group + g];
        const char* const at = a.q.d + (int64_t)(seq.first + token) * a.q.token_bytes + (int64_t)(head * a.group + g) * a.q.head_bytes;
#pragma unroll
        for (int t = 0; t < kSteps; ++t) q[c][t] = load16(at + 2 * stream_k_value<kStore, kDim>(t, hh));
        lse2[c] = lse * kLog2e;
        if (lse != -INFINITY) pos[c] = w.first + token;
    }
    if (__builtin_amdgcn_ballot_w64(falls.some()) != 0) {
        if (threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    for (int tile = lo; tile < hi; ++tile) {
        const int j0 = tile * kTileTokens;
        const Tile next = locate(min(tile + 1, hi - 1));
        f32x4 x[kSets][2], sum[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int c = 0; c < kSets; ++c) x[c][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const u32x4 k = stream_k<kStore, kDim, kBf16>(raw, j, t);
#pragma unroll
                for (int c = 0; c < kSets; ++c) x[c][j] = Num<kBf16>::mma16(k, q[c][t], x[c][j]);
            }
        }
        stream_load_k<kStore, kDim>(next.b[0], next.b[1], lane, raw);
        // lane (row col, hh): tokens 8 (hh % 2) + 4 (hh / 2) .. + 3 of each block
        const int first_key = j0 + 8 * (hh & 1) + 4 * (hh >> 1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sum[j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < kSets; ++c) {
                const Sight sight = sight_of(pos[c], first_key, a.window, a.sinks);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[c][j][e], a.scale2, -lse2[c]));
                    sum[j][e] += pos[c] >= 0 && sight.has(16 * j + e) ? v : 0.0f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[j][e] = sum_over_row(sum[j][e]);
            if (col == 0) w.put(a, now.w[j], first_key + 16 * j, sum[j]);
        }
        now = next;
    }
}

// ---- more rows
constexpr int kWeighWaves = 8, kWeighKeys = 32 * kWeighWaves;
constexpr int kWeighRows = 64;              // of a step: two halves of 32
constexpr int kWeighBuffers = 4;            // steps' rows in LDS: one worked on, three on their way

// a wave's 32 keys, two blocks, as the A operand of 32x32x16 products: lane (place col % 16 of block col / 16, hh) has values 16 step + 8 hh .. + 7
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ void weigh_keys(const char* block, int place, int hh, u32x4* k) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
        for (int s = 0; s < kDim / 16; ++s) k[s] = load16(block + ((2 * s + hh) * 16 + place) * 16);
    } else {
#pragma unroll
        for (int g = 0; g < kDim / 32; ++g) {
            const float scale = *reinterpret_cast<const float*>(block + kAt.ks + (g * 16 + place) * 4);
            if constexpr (kStore == SALI_STORE_INT8) {
                const u32x2 c0 = *reinterpret_cast<const u32x2*>(block + (2 * g * 16 + place) * 16 + 8 * hh), c1 = *reinterpret_cast<const u32x2*>(block + ((2 * g + 1) * 16 + place) * 16 + 8 * hh);
                k[2 * g] = values8<kBf16>(c0.x, c0.y, scale);
                k[2 * g + 1] = values8<kBf16>(c1.x, c1.y, scale);
            } else {
                const float low = low_half<kBf16>(*reinterpret_cast<const uint16_t*>(block + kAt.kz + (g * 16 + place) * 2));
                const u32x2 c = *reinterpret_cast<const u32x2*>(block + (g * 16 + place) * 16 + 8 * hh);
                k[2 * g] = values4<kBf16>(c.x & 0x0F0F0F0Fu, c.y & 0x0F0F0F0Fu, scale, low);
                k[2 * g + 1] = values4<kBf16>(c.x >> 4 & 0x0F0F0F0Fu, c.y >> 4 & 0x0F0F0F0Fu, scale, low);
            }
            if (g % 2 == 1) asm volatile("" ::: "memory");                  // two groups at a time: all at once take registers that there are not
        }
    }
}

// kSteps products with 48 vector instructions between them
template <int kSteps>
__device__ __forceinline__ void side_by_side() {
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 48 / kSteps, 0);
    }
}

// Rows of the kernel: a token has as many as the group has heads, filled up to a divisor of 64 or a multiple of it, so that all rows of a step of 64 move on by the same.
__host__ __device__ inline int weigh_padded(int group) {
    if (group >= kWeighRows) return (group + kWeighRows - 1) / kWeighRows * kWeighRows;
    int n = 1;
    while (n < group) n *= 2;
    return n;
}

// A step's rows in LDS, as loads of 1024 bytes leave them: load n brings the rows n, n + kLoads, .. (kLoads loads a step), and the loads lie 16 bytes further apart than they are
// long, so that 16 rows' pieces are on different banks.
template <int kDim>
struct WeighLayout {
    static constexpr int kLoads = kWeighRows * 2 * kDim / 1024, kPitch = 1024 + 16, kBytes = kLoads * kPitch, kPieces = kDim / 8;
    static __device__ __forceinline__ int row_of(int load, int lane) { return load + kLoads * (lane / kPieces); }
    static __device__ __forceinline__ int at(int row) { return row % kLoads * kPitch + row / kLoads * (2 * kDim); }
};
// 16 bytes (or 4) a lane from memory to LDS, from `to` on, past the registers.  (Not the compiler's own form, before whose readers it waits for all loads.)
__device__ __forceinline__ void weigh_bring16(const void* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "m0", "memory");
}
__device__ __forceinline__ void weigh_bring4(const void* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "m0", "memory");
}
// All of the wave's loads but the last kLater are done, and its reads of LDS; then all waves of the block
template <int kLater>
__device__ __forceinline__ void weigh_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLater) : "memory");
}

// How the rows of a group lie in steps of 64: as many tokens as there is room for; filled up with rows that are none; or a token over several steps, filled up too
enum class WeighRows { even, filled, wide };

// `blocks` thread blocks of 256 keys a sequence and head, times `chunks` of `chunk_steps` steps of 64 rows.  With several chunks the sums go to `partial`,
// [chunk][sequence, head, block][256].
template <int kStore, int kDim, bool kBf16, WeighRows kKind>
__global__ __launch_bounds__(64 * kWeighWaves) __attribute__((amdgpu_waves_per_eu(4))) void k_pages_weigh_tile(PagesWeigh a, int blocks, int chunks, int chunk_steps) {
    constexpr int kSteps = kDim / 16;
    constexpr int kOwn = WeighLayout<kDim>::kLoads / kWeighWaves;           // loads of a wave and step
    constexpr bool kWide = kKind == WeighRows::wide;
    typedef WeighLayout<kDim> L;
    __shared__ __align__(16) uint8_t s_q[kWeighBuffers][L::kBytes];
    __shared__ float s_lse[kWeighBuffers][kWeighRows];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
    const uint32_t units = gridDim.x / (uint32_t)chunks, unit = blockIdx.x % units;
    const int chunk = chunks - 1 - (int)(blockIdx.x / units);               // rows that see most keys first
    const int head = (int)(unit % (uint32_t)a.geom.n_kv), nth = (int)(unit / (uint32_t)a.geom.n_kv), s = nth / blocks, nth_of_seq = nth - s * blocks;
    const bool notes = chunk == 0 && nth_of_seq == 0 && head == 0;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, lane, 64);
    const PageSeq seq = load_seq(a.seqs, a.geom, s, notes && threadIdx.x == 0);
    if (__builtin_amdgcn_ballot_w64(falls.some()) != 0) {
        if (notes && threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    const int key0 = nth_of_seq * kWeighKeys;
    if (seq.n == 0 || key0 >= seq.len) return;
    const WeighSeq w = {a.seqs.table + (int64_t)s * a.seqs.width, seq.len, seq.len - seq.n};
    const int group = a.group, padded = kKind == WeighRows::even ? group : weigh_padded(group);
    const int by_token = kWide ? 1 : kWeighRows / padded, phases = kWide ? padded / kWeighRows : 1;        // tokens of a step, steps of a token
    // The sequence's steps from the first row on: the first with a token from `t` on, the first one behind those whose tokens lie all before `t`, and the end
    auto step_from = [&](int t) { return (int64_t)t / by_token * phases; };
    auto step_behind = [&](int64_t t) { return (t + by_token - 1) / by_token * phases; };
    // steps that see some of the block's keys: from the token at position key0 on, and under a window up to the last one that has the block's last key in its window
    int64_t end = step_behind(seq.n);
    if (a.window > 0 && key0 >= a.sinks) end = min(end, step_behind(max((int64_t)0, (int64_t)key0 + kWeighKeys - 1 + a.window - w.first)));
    const int64_t step0 = max(step_from(max(0, key0 - w.first)), (int64_t)chunk * chunk_steps);
    const int steps = (int)max((int64_t)0, min(end, (int64_t)(chunk + 1) * chunk_steps) - step0);
    const int j0 = key0 + 32 * wave;

    // ---- rows on their way to LDS: kOwn + 1 loads a wave and step (all waves bring the log-sums); a thread has the addresses of its next ones
    auto row_of_step = [&](int r, int& of_group) {                          // row r of a step: tokens behind its first one, and head of the group (wide: behind the phase's first)
        of_group = kWide ? r : r & (padded - 1);
        return kWide ? 0 : r / padded;
    };
    // (Instead of a row that is none another one, which nobody looks at: one of the last head, or of the last token.)
    auto place = [&](int r, int64_t step, int64_t& token, int& of_group) {
        token = row_of_step(r, of_group) + (kWide ? step / phases : step * by_token);
        token = min(token, (int64_t)seq.n - 1);
        if constexpr (kWide) of_group += (int)(step % phases) * kWeighRows;
        if constexpr (kKind != WeighRows::even) of_group = min(of_group, group - 1);
    };
    const char* from[kOwn];
    const float* lse_from;
    auto address = [&](int64_t step) {
        int64_t token;
        int g;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            place(L::row_of(wave + kWeighWaves * i, lane), step, token, g);
            from[i] = a.q.d + (seq.first + token) * a.q.token_bytes + (int64_t)(head * group + g) * a.q.head_bytes + 16 * (lane % L::kPieces);
        }
        place(lane, step, token, g);
        lse_from = a.lse + (seq.first + token) * a.heads + head * group + g;
    };
    const int64_t q_by = by_token * a.q.token_bytes, lse_by = (int64_t)by_token * a.heads;
    const int whole = (int)min((int64_t)steps, (kWide ? (int64_t)seq.n * phases : (int64_t)(seq.n / by_token)) - step0);     // steps without tokens behind the last one
    const uint32_t q_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&s_q[0][0] + (uint32_t)(L::kPitch * wave);
    const uint32_t lse_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&s_lse[0][0];
    int asked = 0;
    auto ask = [&]() {                      // of step `asked`; behind the last one that one again, for nothing, so that what is on its way has always the same number
        const uint32_t buf = (uint32_t)asked % kWeighBuffers;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) weigh_bring16(from[i], q_at + buf * L::kBytes + (uint32_t)(i * L::kPitch * kWeighWaves));
        weigh_bring4(lse_from, lse_at + buf * (4 * kWeighRows));
        ++asked;
        if (!kWide && asked < whole) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) from[i] += q_by;
            lse_from += lse_by;
        } else if (asked < steps) {
            address(step0 + asked);
        }
    };

    // where the wave's block b of 16 keys lies, and its weights
    auto block_of = [&](int b, float*& to) {
        const int block = j0 / kBlockTokens + b;
        const int page = block * kBlockTokens < seq.len ? __builtin_amdgcn_readfirstlane(w.table[block >> a.geom.blocks_log2]) : -1;
        return w.block(a, head, block, page, to);
    };
    u32x4 k[kSteps];
    {
        const char* at[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float* to;
            at[b] = block_of(b, to);
            if (to == nullptr && j0 + kBlockTokens * b < seq.len && chunk == 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
        }
        weigh_keys<kStore, kDim, kBf16>(col < 16 ? at[0] : at[1], col & 15, hh, k);
#pragma unroll
        for (int t = 0; t < kSteps; ++t) asm volatile("" : "+v"(k[t]));     // waited for here, before loads are on their way whose number matters
    }
    f32x16 sum;
#pragma unroll
    for (int x = 0; x < 16; ++x) sum[x] = 0.0f;

    if (steps > 0) {
        address(step0);
#pragma unroll
        for (int i = 0; i < kWeighBuffers - 1; ++i) ask();
    }
    int step = 0;
    float lse2[2] = {0.0f, 0.0f};           // of the lane's rows
    auto begin = [&]() {                    // the step's rows are there, and all waves are through with the step before, whose buffer is the next one's
        weigh_meet<(kWeighBuffers - 2) * (kOwn + 1)>();
        ask();
        const float* const l = s_lse[(uint32_t)step % kWeighBuffers] + col;
        lse2[0] = l[0] * kLog2e;
        lse2[1] = l[32] * kLog2e;
    };
    auto queries = [&](int half, int t) { return load16(s_q[(uint32_t)step % kWeighBuffers] + L::at(col) + 16 * hh + 32 / L::kLoads * half * (2 * kDim) + 32 * t); };
    auto add = [&](const f32x16& st, float lse2, bool is) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
            sum[e] += kKind == WeighRows::even || is ? v : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(sum[e]));        // here, and not moved behind the barrier
    };
    int row_head[2], behind[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) behind[i] = row_of_step(32 * i + col, row_head[i]);
    auto is_head = [&](int i) { return kKind == WeighRows::even || (kWide ? (int)((step0 + step) % phases) * kWeighRows : 0) + row_head[i] < group; };
    // steps all of whose rows see all of the wave's keys
    int64_t plain_end = whole;
    if (a.window > 0 && j0 + 32 > a.sinks) plain_end = min(plain_end, ((int64_t)max(0, j0 + a.window - w.first)) / by_token * phases - step0);
    const int64_t plain_from = step_behind(max(0, j0 + 31 - w.first)) - step0;
    while (step < steps) {
        begin();
        if (step >= plain_from && step < plain_end && __builtin_amdgcn_ballot_w64(fminf(lse2[0], lse2[1]) == -INFINITY) == 0) {
            // Products and weights of different rows side by side: the weights of a step's second half wait for the next products
            f32x16 held;
            float held_lse2 = INFINITY;                                     // weights of 0
            bool held_is = true, more;
#pragma unroll
            for (int e = 0; e < 16; ++e) held[e] = 0.0f;
            do {
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[t], queries(0, t), st);
                add(held, held_lse2, held_is);
                side_by_side<kSteps>();
#pragma unroll
                for (int e = 0; e < 16; ++e) held[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) held = Num<kBf16>::mma32(k[t], queries(1, t), held);
                add(st, lse2[0], is_head(0));
                side_by_side<kSteps>();
                held_lse2 = lse2[1];
                held_is = is_head(1);
                more = ++step < plain_end;
                if (more) {
                    begin();
                    more = __builtin_amdgcn_ballot_w64(fminf(lse2[0], lse2[1]) == -INFINITY) == 0;
                    if (!more) break;       // with the step begun
                }
            } while (more);
            add(held, held_lse2, held_is);
            if (step >= plain_end) continue;
        }
        const int token = (int)(kWide ? (step0 + step) / phases : (step0 + step) * by_token);       // the step's first one
        if (w.first + token + by_token - 1 >= j0 && !(a.window > 0 && j0 >= a.sinks && w.first + token - a.window >= j0 + 31)) {
            int first_key = j0 + 8 * hh;
            asm volatile("" : "+v"(first_key));
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int t = token + behind[half];
                const Sight sight = sight_of(w.first + t, first_key, a.window, a.sinks);
                const bool some = t < seq.n && is_head(half) && lse2[half] != -INFINITY;         // a row that saw nothing has no weights
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[t], queries(half, t), st);
                // lane (row col, hh): register e has token 8 hh + e % 8 of block e / 8
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2[half]));
                    asm("" : "+v"(v));      // a choice, not a branch
                    sum[e] += some && sight.has(16 * (e / 8) + e % 8) ? v : 0.0f;
                }
            }
        }
        ++step;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // nothing is on its way to the block's LDS when it ends
    // ---- over the 32 rows' lanes
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t u = __builtin_bit_cast(uint32_t, sum_over_row(sum[e]));
        const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        sum[e] = __builtin_bit_cast(float, (uint32_t)both[0]) + __builtin_bit_cast(float, (uint32_t)both[1]);
    }
    // (the lane's number worked out again, with what the compiler does not know: through the loop it has no registers for it)
    uint32_t all = ~0u;
    asm volatile("" : "+s"(all));
    const int end_lane = __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
    if ((end_lane & 31) != 0) return;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        float* to;
        block_of(b, to);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 8 * b + 4 * i, at = 32 * wave + 16 * b + 8 * (end_lane >> 5) + 4 * i;
            const f32x4 four = {sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            if (chunks > 1) *reinterpret_cast<f32x4*>(a.partial + ((int64_t)chunk * units + unit) * kWeighKeys + at) = four;
            else w.put(a, to, key0 + at, four);
        }
    }
}

// ---- rows that fit LDS: up to 256, for all of a thread block's keys.  A wave walks `each` tiles of 32 keys, the next one's on their way; no barrier but the one for the rows.
constexpr int kWeighFewWaves = 4, kWeighFewSteps = 4;
template <int kStore, int kDim>
struct WeighRaw {                           // a lane's share of 32 keys, as weigh_keys makes operands of it
    u32x4 c[kStore == SALI_STORE_16 ? kDim / 16 : (kStore == SALI_STORE_INT8 ? kDim / 32 : kDim / 64)];
    float scale[kStore == SALI_STORE_16 ? 1 : kDim / 32];
    uint16_t low[kStore == SALI_STORE_INT4 ? kDim / 32 : 1];
};
template <int kStore, int kDim>
__device__ __forceinline__ void weigh_load(const char* block, int place, int hh, WeighRaw<kStore, kDim>& r) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
        for (int s = 0; s < kDim / 16; ++s) r.c[s] = stream16(block + ((2 * s + hh) * 16 + place) * 16);
    } else {
        // pieces of two steps each (8 bits: step s; 4 bits: steps 2 s and 2 s + 1), this half's 8 bytes
#pragma unroll
        for (int s = 0; s < (kStore == SALI_STORE_INT8 ? kDim / 32 : kDim / 64); ++s) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(block + (2 * s * 16 + place) * 16 + 8 * hh), y = *reinterpret_cast<const u32x2*>(block + ((2 * s + 1) * 16 + place) * 16 + 8 * hh);
            r.c[s] = (u32x4){x.x, x.y, y.x, y.y};
        }
#pragma unroll
        for (int g = 0; g < kDim / 32; ++g) {
            r.scale[g] = *reinterpret_cast<const float*>(block + kAt.ks + (g * 16 + place) * 4);
            if constexpr (kStore == SALI_STORE_INT4) r.low[g] = *reinterpret_cast<const uint16_t*>(block + kAt.kz + (g * 16 + place) * 2);
        }
    }
}
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ u32x4 weigh_operand(const WeighRaw<kStore, kDim>& r, int t) {
    if constexpr (kStore == SALI_STORE_16) {
        return r.c[t];
    } else if constexpr (kStore == SALI_STORE_INT8) {
        const u32x4& c = r.c[t / 2];
        return values8<kBf16>(t & 1 ? c.z : c.x, t & 1 ? c.w : c.y, r.scale[t / 2]);
    } else {
        const int g = t / 2, shift = 4 * (t & 1);
        const u32x4& c = r.c[g / 2];
        return values4<kBf16>((g & 1 ? c.z : c.x) >> shift & 0x0F0F0F0Fu, (g & 1 ? c.w : c.y) >> shift & 0x0F0F0F0Fu, r.scale[g], low_half<kBf16>(r.low[g]));
    }
}

// `blocks` thread blocks a sequence and head; `lds_steps`: steps of 64 rows that there is LDS for
template <int kStore, int kDim, bool kBf16, WeighRows kKind>
__global__ __launch_bounds__(64 * kWeighFewWaves) __attribute__((amdgpu_waves_per_eu(3))) void k_pages_weigh_few(PagesWeigh a, int blocks, int each, int lds_steps) {
    typedef WeighLayout<kDim> L;
    constexpr int kSteps = kDim / 16, kOwn = L::kLoads / kWeighFewWaves;
    constexpr bool kWide = kKind == WeighRows::wide;
    extern __shared__ __align__(16) uint8_t s_few[];        // [step][L::kBytes], then the log-sums [step][64]
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
    const int head = (int)(blockIdx.x % (uint32_t)a.geom.n_kv), nth = (int)(blockIdx.x / (uint32_t)a.geom.n_kv), s = nth / blocks, nth_of_seq = nth - s * blocks;
    const bool notes = nth_of_seq == 0 && head == 0;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, lane, 64);
    const int lo = (nth_of_seq * kWeighFewWaves + wave) * each, shift = a.geom.blocks_log2;
    // the page numbers of the wave's blocks, one a lane, on their way with the lengths
    int page_of_lane = -1;
    const int64_t index0 = (int64_t)(2 * lo) >> shift;
    if (index0 + lane < a.seqs.width) page_of_lane = a.seqs.table[(int64_t)s * a.seqs.width + index0 + lane];
    const PageSeq seq = load_seq(a.seqs, a.geom, s, notes && threadIdx.x == 0);
    if (__builtin_amdgcn_ballot_w64(falls.some()) != 0) {
        if (notes && threadIdx.x == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    const int tiles = (int)(((int64_t)seq.len + kTileTokens - 1) / kTileTokens), hi = min(lo + each, tiles);
    if (seq.n == 0 || nth_of_seq * kWeighFewWaves * each >= tiles) return;
    const WeighSeq w = {nullptr, seq.len, seq.len - seq.n};
    const int group = a.group, padded = kKind == WeighRows::even ? group : weigh_padded(group);
    const int by_token = kWide ? 1 : kWeighRows / padded, phases = kWide ? padded / kWeighRows : 1;
    const int steps = min(lds_steps, (seq.n + by_token - 1) / by_token * phases);
    // ---- the rows, as the other kernel has them
    auto row_of = [&](int r, int step, int& token, int& of_group) {
        of_group = kWide ? step % phases * kWeighRows + r : r & (padded - 1);
        token = kWide ? step / phases : step * by_token + r / padded;
    };
    auto address = [&](int r, int step, int64_t& token, int& of_group) {
        int t;
        row_of(r, step, t, of_group);
        token = seq.first + min(t, seq.n - 1);
        of_group = min(of_group, group - 1);
    };
    const uint32_t q_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)s_few, lse_at = q_at + (uint32_t)(lds_steps * L::kBytes);
    for (int step = 0; step < steps; ++step) {
        int64_t token;
        int g;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int load = wave + kWeighFewWaves * i;
            address(L::row_of(load, lane), step, token, g);
            weigh_bring16(a.q.d + token * a.q.token_bytes + (int64_t)(head * group + g) * a.q.head_bytes + 16 * (lane % L::kPieces),
                          q_at + (uint32_t)(step * L::kBytes + load * L::kPitch));
        }
        address(lane, step, token, g);
        if (step % kWeighFewWaves == wave) weigh_bring4(a.lse + token * a.heads + head * group + g, lse_at + (uint32_t)(4 * kWeighRows * step));
    }
    struct Tile {
        const char* b[2];
        float* w[2];
    };
    auto locate = [&](int tile) -> Tile {
        Tile t;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int block = 2 * tile + j, page = __builtin_amdgcn_readlane(page_of_lane, (int)((block >> shift) - index0));
            t.b[j] = w.block(a, head, block, page, t.w[j]);
            if (t.w[j] == nullptr && block * kBlockTokens < seq.len && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
        }
        return t;
    };
    WeighRaw<kStore, kDim> raw;
    Tile now = {};
    if (lo < hi) {
        now = locate(lo);
        weigh_load<kStore, kDim>(col < 16 ? now.b[0] : now.b[1], col & 15, hh, raw);
    }
    weigh_meet<0>();
    for (int tile = lo; tile < hi; ++tile) {
        const int j0 = tile * kTileTokens;
        u32x4 k[kSteps];
#pragma unroll
        for (int t = 0; t < kSteps; ++t) k[t] = weigh_operand<kStore, kDim, kBf16>(raw, t);
        const Tile next = locate(min(tile + 1, hi - 1));
        weigh_load<kStore, kDim>(col < 16 ? next.b[0] : next.b[1], col & 15, hh, raw);
        f32x16 sum;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
        const bool early = j0 + kTileTokens - 1 <= w.first && a.window == 0;       // all rows see all of the tile
        const bool out_of_sight = a.window > 0 && j0 >= a.sinks && j0 + kTileTokens - 1 <= w.first - a.window;
        for (int half = 0; half < 2 * steps && !out_of_sight; ++half) {
            const int step = half >> 1, r = 32 * (half & 1) + col;
            const uint8_t* const q = s_few + step * L::kBytes + L::at(col) + 32 / L::kLoads * (half & 1) * (2 * kDim) + 16 * hh;
            const float lse = *reinterpret_cast<const float*>(s_few + lds_steps * L::kBytes + 4 * (kWeighRows * step + r)), lse2 = lse * kLog2e;
            f32x16 st;
#pragma unroll
            for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
            for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[t], load16(q + 32 * t), st);
            int token, g;
            row_of(r, step, token, g);
            const bool some = token < seq.n && g < group && lse != -INFINITY;      // a row that saw nothing has no weights
            if (early && __builtin_amdgcn_ballot_w64(!some) == 0) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
            } else {
                int first_key = j0 + 8 * hh;
                asm volatile("" : "+v"(first_key));
                const Sight sight = sight_of(w.first + token, first_key, a.window, a.sinks);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
                    asm("" : "+v"(v));      // a choice, not a branch
                    sum[e] += some && sight.has(16 * (e / 8) + e % 8) ? v : 0.0f;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t u = __builtin_bit_cast(uint32_t, sum_over_row(sum[e]));
            const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            sum[e] = __builtin_bit_cast(float, (uint32_t)both[0]) + __builtin_bit_cast(float, (uint32_t)both[1]);
        }
        if (col == 0)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int e = 8 * b + 4 * i;
                    w.put(a, now.w[b], j0 + 16 * b + 8 * hh + 4 * i, (f32x4){sum[e], sum[e + 1], sum[e + 2], sum[e + 3]});
                }
        now = next;
    }
}

// The chunks' sums, in their order: a thread four keys
__global__ __launch_bounds__(kWeighKeys / 4) void k_pages_weigh_merge(PagesWeigh a, int blocks, int chunks) {
    const uint32_t units = gridDim.x, unit = blockIdx.x;
    const int head = (int)(unit % (uint32_t)a.geom.n_kv), nth = (int)(unit / (uint32_t)a.geom.n_kv), s = nth / blocks;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, threadIdx.x, 64);
    const PageSeq seq = load_seq(a.seqs, a.geom, s, false);
    const int at = (nth - s * blocks) * kWeighKeys + 4 * (int)threadIdx.x;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = 0; c < chunks; ++c) sum += *reinterpret_cast<const f32x4*>(a.partial + ((int64_t)c * units + unit) * kWeighKeys + 4 * threadIdx.x);
    if (__builtin_amdgcn_ballot_w64(falls.some()) != 0 || seq.n == 0 || at >= seq.len) return;
    const WeighSeq w = {a.seqs.table + (int64_t)s * a.seqs.width, seq.len, seq.len - seq.n};
    float* to;
    w.block(a, head, at / kBlockTokens, w.table[(at / kBlockTokens) >> a.geom.blocks_log2], to);
    w.put(a, to, at, sum);
}

}  // namespace

}  // namespace sali
