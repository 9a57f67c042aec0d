// What attention weight keys had: for every key of a sequence and K/V head, the sum of exp(s - lse) over the new tokens that see it and the query heads of the group (gfx950).
//
// Rows, scores, masks and tiles of 32 keys are those of attention (pages_attn.h); with lse at hand there is no maximum to find, no second product and
// nothing to join: keys stay with a wave, which walks the rows that see them and adds the weights up in fp32, always in the same order.
//
// Few rows (single tokens, drafts): the stream, bound by K's bytes.  A wave has its rows' queries in registers and walks tiles, the next one's K on its way.
// More: the rows' queries come through LDS, 32 at a time, and a wave has 64 keys in registers, so that a query read from LDS is multiplied twice.
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
constexpr int kWeighWaves = 4, kWeighKeys = 32 * kWeighWaves;
constexpr int kWeighRows = 64;              // of a step: two products'

// a wave's 32 keys, two blocks, as the A operand of 32x32x16 products: lane (place col % 16 of block col / 16, hh) has values 16 step + 8 hh .. + 7
template <int kStore, int kDim, bool kBf16>
__device__ __forceinline__ void weigh_keys(const char* block, int place, int hh, u32x4* k) {
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
        for (int s = 0; s < kDim / 16; ++s) k[s] = load16(block + ((2 * s + hh) * 16 + place) * 16);
    } else {
        u32x2 c[kDim / 16];
        float scale[kDim / 32], low[kDim / 32];
#pragma unroll
        for (int g = 0; g < kDim / 32; ++g) {
            scale[g] = *reinterpret_cast<const float*>(block + kAt.ks + (g * 16 + place) * 4);
            low[g] = 0.0f;
            if constexpr (kStore == SALI_STORE_INT4) low[g] = low_half<kBf16>(*reinterpret_cast<const uint16_t*>(block + kAt.kz + (g * 16 + place) * 2));
        }
        constexpr int kLoads = kStore == SALI_STORE_INT8 ? kDim / 16 : kDim / 32;
#pragma unroll
        for (int s = 0; s < kLoads; ++s) c[s] = *reinterpret_cast<const u32x2*>(block + (s * 16 + place) * 16 + 8 * hh);
#pragma unroll
        for (int s = 0; s < kDim / 16; ++s) {
            if constexpr (kStore == SALI_STORE_INT8) k[s] = values8<kBf16>(c[s].x, c[s].y, scale[s / 2]);
            else k[s] = values4<kBf16>(c[s / 2].x >> (4 * (s & 1)) & 0x0F0F0F0Fu, c[s / 2].y >> (4 * (s & 1)) & 0x0F0F0F0Fu, scale[s / 2], low[s / 2]);
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

// `blocks` thread blocks of 128 keys a sequence and head, times `chunks` of `chunk_rows` rows.  With several chunks the sums go to `partial`, [chunk][sequence, head, block][128].
// kPad: some rows are none.
template <int kStore, int kDim, bool kBf16, bool kPad>
__global__ __launch_bounds__(64 * kWeighWaves) __attribute__((amdgpu_waves_per_eu(3))) void k_pages_weigh_tile(PagesWeigh a, int blocks, int chunks, int64_t chunk_rows) {
    constexpr int kSteps = kDim / 16, kPieces = kDim / 8, kPitch = 16 * kWeighRows + 16;
    constexpr int kOwn = kWeighRows * kPieces / (64 * kWeighWaves);         // pieces of 16 bytes that a thread brings
    __shared__ __align__(16) uint8_t s_q[2][kPieces * kPitch];
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
    const int group = a.group, padded = kPad ? weigh_padded(group) : group;
    const int64_t rows = (int64_t)seq.n * padded;
    // rows that see some of the block's keys: from the one at position key0 on, and under a window up to the last one that has the block's last key in its window
    int64_t lo = (int64_t)max(0, key0 - w.first) * padded, hi = rows;
    if (a.window > 0 && key0 >= a.sinks) hi = max((int64_t)0, min(rows, ((int64_t)key0 + kWeighKeys - 1 + a.window - w.first) * padded));
    lo = max(lo & ~(int64_t)(kWeighRows - 1), (int64_t)chunk * chunk_rows);
    hi = min(hi, (int64_t)(chunk + 1) * chunk_rows);
    const int steps = (int)max((int64_t)0, (hi - lo + kWeighRows - 1) / kWeighRows);
    const int j0 = key0 + 32 * wave;
    u32x4 k[kSteps];
    float* to[2];                           // of the wave's blocks of 16 keys
    {
        const char* at[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int block = j0 / kBlockTokens + b;
            const int page = block * kBlockTokens < seq.len ? w.table[block >> a.geom.blocks_log2] : -1;
            at[b] = w.block(a, head, block, page, to[b]);
            if (to[b] == nullptr && block * kBlockTokens < seq.len && chunk == 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
        }
        weigh_keys<kStore, kDim, kBf16>(col < 16 ? at[0] : at[1], col & 15, hh, k);
        // waited for here: in the loop a wait for them would be one for the next queries too
#pragma unroll
        for (int t = 0; t < kSteps; ++t) asm volatile("" : "+v"(k[t]));
    }
    f32x16 sum;
#pragma unroll
    for (int x = 0; x < 16; ++x) sum[x] = 0.0f;

    // A step's rows: those of 64 / padded tokens, or 64 of a token's.  A thread has the addresses of the pieces that it brings and of its own rows' log-sums; all move on by the same.
    const int by_token = padded >= kWeighRows ? 1 : kWeighRows / padded, phases = padded > kWeighRows ? padded / kWeighRows : 1;
    const int64_t q_step = by_token * a.q.token_bytes, lse_step = (int64_t)by_token * a.heads;
    int phase = (int)(lo % padded) / kWeighRows, token0 = (int)(lo / padded);       // 64 rows of the first token's from 64 phase on
    auto of_step = [&](int r, int& of_group) {                              // of the step's row r: tokens behind its first one, head of the group without the phase
        of_group = padded >= kWeighRows ? r : r & (padded - 1);
        return padded >= kWeighRows ? 0 : r / padded;
    };
    const char* from[kOwn];
    const float* lse_from[2];
    int behind[2], row_head[2];             // of the lane's rows
    // (Instead of a row that is none another one, which nobody looks at.)
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        int g;
        const int t = of_step(((int)threadIdx.x + 64 * kWeighWaves * i) / kPieces, g);
        from[i] = a.q.d + (int64_t)(seq.first + token0 + t) * a.q.token_bytes + (int64_t)(head * group + 64 * phase + (kPad ? min(g, group - 1 - 64 * phase) : g)) * a.q.head_bytes +
                  16 * ((int)threadIdx.x % kPieces);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        behind[i] = of_step(32 * i + col, row_head[i]);
        lse_from[i] = a.lse + (int64_t)(seq.first + token0 + behind[i]) * a.heads + head * group + 64 * phase + (kPad ? min(row_head[i], group - 1 - 64 * phase) : row_head[i]);
    }
    u32x4 x[kOwn];
    float lse[2];
    int asked_token = token0, asked_phase = phase;
    auto ask = [&]() {
        // tokens behind the last one: the last one's rows
        const int most = seq.n - 1 - asked_token;
        if (by_token - 1 <= most) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) x[i] = load16(from[i]);
#pragma unroll
            for (int i = 0; i < 2; ++i) lse[i] = *lse_from[i];
        } else {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                int g;
                const int t = of_step(((int)threadIdx.x + 64 * kWeighWaves * i) / kPieces, g);
                x[i] = load16(from[i] - (int64_t)max(0, t - most) * a.q.token_bytes);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) lse[i] = *(lse_from[i] - (int64_t)max(0, behind[i] - most) * a.heads);
        }
        // on to the next rows
        int64_t q_by = q_step, lse_by = lse_step;
        if (phases > 1) {
            const bool next = ++asked_phase == phases;
            // 64 heads on; from the last ones back to the token's first (where rows are filled up, those of the last phase stay within the group)
            const int heads = next ? -(phases - 1) * kWeighRows : kWeighRows;
            if (next) asked_phase = 0;
            q_by = (next ? a.q.token_bytes : 0) + heads * a.q.head_bytes;
            lse_by = (next ? a.heads : 0) + heads;
            asked_token += next ? 1 : 0;
            if constexpr (kPad) {
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int g = ((int)threadIdx.x + 64 * kWeighWaves * i) / kPieces;
                    from[i] = a.q.d + (int64_t)(seq.first + asked_token) * a.q.token_bytes + (int64_t)(head * group + min(64 * asked_phase + g, group - 1)) * a.q.head_bytes +
                              16 * ((int)threadIdx.x % kPieces);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) lse_from[i] = a.lse + (int64_t)(seq.first + asked_token) * a.heads + head * group + min(64 * asked_phase + 32 * i + col, group - 1);
                return;
            }
        } else {
            asked_token += by_token;
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) from[i] += q_by;
#pragma unroll
        for (int i = 0; i < 2; ++i) lse_from[i] += lse_by;
    };
    // A step's beginning: its rows to LDS, the next ones' on their way.  What the step has: its first row's token and phase, and the log-sums of the lane's rows
    int left = steps, buf = 1, token = 0, next_token = token0;
    int step_phase = 0, next_phase = phase;
    float lse2[2] = {0.0f, 0.0f};
    auto begin = [&]() {
        buf ^= 1;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int p = (int)threadIdx.x + 64 * kWeighWaves * i;
            *reinterpret_cast<u32x4*>(s_q[buf] + p % kPieces * kPitch + p / kPieces * 16) = x[i];
        }
        token = next_token;
        step_phase = next_phase;
        lse2[0] = lse[0] * kLog2e;
        lse2[1] = lse[1] * kLog2e;
        next_token = asked_token;
        next_phase = asked_phase;
        if (left > 1) ask();
        __syncthreads();                    // the rows are there, and all waves are through with the other buffer
    };
    // Is the lane's row one, whatever its log-sum?
    auto is_row = [&](int i) { return token + behind[i] < seq.n && (!kPad || 64 * step_phase + row_head[i] < group); };
    // Do all of the step's rows see all of the wave's keys, and have they seen something?  (Rows that fill up groups do not count.)
    auto plain = [&]() {
        const int first_pos = w.first + token, last_pos = first_pos + by_token - 1;
        if (first_pos < j0 + 31 || token + by_token > seq.n || !(a.window == 0 || last_pos - a.window < j0 || j0 + 32 <= a.sinks)) return false;
        return __builtin_amdgcn_ballot_w64(fminf(lse2[0], lse2[1]) == -INFINITY) == 0;
    };
    auto add = [&](f32x16& to, const f32x16& st, float lse2, bool is) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
            to[e] += !kPad || is ? v : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(to[e]));        // here, and not moved behind the barrier
    };
    auto queries = [&](int half, int t) { return load16(s_q[buf] + (2 * t + hh) * kPitch + half * 512 + col * 16); };
    if (left > 0) {
        ask();
        begin();
    }
    while (left > 0) {
        if (plain()) {
            // Products and weights of different rows side by side: the weights of a step's second half wait for the next products
            f32x16 held;
            float held_lse2 = INFINITY;             // weights of 0
            bool held_is = true;
#pragma unroll
            for (int e = 0; e < 16; ++e) held[e] = 0.0f;
            do {
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[t], queries(0, t), st);
                add(sum, held, held_lse2, held_is);
                side_by_side<kSteps>();
#pragma unroll
                for (int e = 0; e < 16; ++e) held[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) held = Num<kBf16>::mma32(k[t], queries(1, t), held);
                add(sum, st, lse2[0], is_row(0));
                side_by_side<kSteps>();
                held_lse2 = lse2[1];
                held_is = is_row(1);
                if (--left == 0) break;
                begin();
            } while (plain());
            add(sum, held, held_lse2, held_is);
            if (left == 0) break;
        }
        if (w.first + token + by_token - 1 >= j0 && !(a.window > 0 && j0 >= a.sinks && w.first + token - a.window >= j0 + 31)) {
            int first_key = j0 + 8 * hh;
            asm volatile("" : "+v"(first_key));
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const Sight sight = sight_of(w.first + token + behind[half], first_key, a.window, a.sinks);
                const bool some = is_row(half) && lse2[half] != -INFINITY;     // a row that saw nothing has no weights
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[t], queries(half, t), st);
                // lane (row col, hh): register e has token 8 hh + e % 8 of block e / 8
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2[half]));
                    sum[e] += some && sight.has(16 * (e / 8) + e % 8) ? v : 0.0f;
                }
            }
        }
        if (--left > 0) begin();
    }
    // ---- over the 32 rows' lanes
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t u = __builtin_bit_cast(uint32_t, sum_over_row(sum[e]));
        const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        sum[e] = __builtin_bit_cast(float, (uint32_t)both[0]) + __builtin_bit_cast(float, (uint32_t)both[1]);
    }
    if (col != 0) return;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 8 * b + 4 * i;
            const f32x4 four = {sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            if (chunks > 1) *reinterpret_cast<f32x4*>(a.partial + ((int64_t)chunk * units + unit) * kWeighKeys + 32 * wave + 16 * b + 8 * hh + 4 * i) = four;
            else w.put(a, to[b], j0 + 16 * b + 8 * hh + 4 * i, four);
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
