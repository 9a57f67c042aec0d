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
        for (int t = 0; t < kSteps; ++t) {
            const u32x4 v = load16(at + 2 * stream_k_value<kStore, kDim>(t, hh));
#pragma unroll
            for (int e = 0; e < 4; ++e) q[c][t][e] = (v[e] & a.q_keep) ^ a.q_flip;
        }
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
constexpr int kWeighWaves = 4, kWeighKeys = 64 * kWeighWaves;
constexpr int kWeighRows = 32;              // of a step

// a wave's 64 keys as the A operand of 32x32x16 products: two sets of two blocks; lane (place col % 16 of block col / 16, hh) has values 16 step + 8 hh .. + 7
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

// `blocks` thread blocks of 256 keys a sequence and head, times `chunks` of `chunk_rows` rows.  With several chunks the sums go to `partial`, [chunk][sequence, head, block][256].
template <int kStore, int kDim, bool kBf16>
__global__ __launch_bounds__(64 * kWeighWaves) __attribute__((amdgpu_waves_per_eu(2))) void k_pages_weigh_tile(PagesWeigh a, int blocks, int chunks, int chunk_rows) {
    constexpr int kSteps = kDim / 16, kPieces = kDim / 8, kPitch = 16 * kWeighRows + 16;
    constexpr int kOwn = kWeighRows * kPieces / (64 * kWeighWaves);         // pieces of 16 bytes that a thread brings
    __shared__ __align__(16) uint8_t s_q[2][kPieces * kPitch];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
    const uint32_t units = gridDim.x / (uint32_t)chunks, unit = blockIdx.x % units;
    const int chunk = (int)(blockIdx.x / units);
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
    const int rows = seq.n * a.group, group = a.group;
    // rows that see some of the block's keys: from the one at position key0 on, and under a window up to the last one that has the block's last key in its window
    int lo = max(0, key0 - w.first) * group, hi = rows;
    if (a.window > 0 && key0 >= a.sinks) hi = (int)max((int64_t)0, min((int64_t)rows, ((int64_t)key0 + kWeighKeys - 1 + a.window - w.first) * group));
    lo = max(lo & ~(kWeighRows - 1), chunk * chunk_rows);
    hi = min(hi, (int)min((int64_t)0x7FFFFFFF, (int64_t)(chunk + 1) * chunk_rows));
    const int j0 = key0 + 64 * wave;
    u32x4 k[2][kSteps];
    float* to[4];                           // of the wave's blocks of 16 keys
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int block = j0 / kBlockTokens + b;
        const int page = block * kBlockTokens < seq.len ? w.table[block >> a.geom.blocks_log2] : -1;
        w.block(a, head, block, page, to[b]);
        if (to[b] == nullptr && block * kBlockTokens < seq.len && chunk == 0 && lane == 0) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
    }
    if (lo < hi) {
#pragma unroll
        for (int set = 0; set < 2; ++set) {
            const int block = j0 / kBlockTokens + 2 * set + (col >> 4);
            const int page = block * kBlockTokens < seq.len ? w.table[block >> a.geom.blocks_log2] : -1;
            float* unused;
            weigh_keys<kStore, kDim, kBf16>(w.block(a, head, block, page, unused), col & 15, hh, k[set]);
        }
        // waited for here: in the loop a wait for them would be one for the next queries too
#pragma unroll
        for (int set = 0; set < 2; ++set)
#pragma unroll
            for (int t = 0; t < kSteps; ++t) asm volatile("" : "+v"(k[set][t]));
    }
    f32x16 sum[2];
#pragma unroll
    for (int set = 0; set < 2; ++set)
#pragma unroll
        for (int x = 0; x < 16; ++x) sum[set][x] = 0.0f;

    // Rows, which move on by 32 a step: by tokens and heads of the group.  A lane has the addresses of the pieces that it brings and of its own row's log-sum.
    const int by_token = kWeighRows / group, by_head = kWeighRows - by_token * group;
    const int64_t q_step = by_token * a.q.token_bytes + by_head * a.q.head_bytes, q_wrap = a.q.token_bytes - group * a.q.head_bytes;
    const int lse_step = by_token * a.heads + by_head, lse_wrap = a.heads - group;
    struct Row {
        int token, of_group;
    };
    auto row_at = [&](int r) -> Row { return {(int)((uint32_t)r / (uint32_t)group), (int)((uint32_t)r % (uint32_t)group)}; };
    // does it go on to another token than by_token further?
    auto move_on = [&](Row& r) {
        r.token += by_token;
        r.of_group += by_head;
        const bool wraps = r.of_group >= group;
        r.of_group -= wraps ? group : 0;
        r.token += wraps ? 1 : 0;
        return wraps;
    };
    Row bring[kOwn], mine = row_at(lo + col), first_row = row_at(lo), last_row = row_at(lo + kWeighRows - 1);
    const char* from[kOwn];
    const float* lse_from = a.lse + (int64_t)(seq.first + mine.token) * a.heads + head * group + mine.of_group;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        bring[i] = row_at(lo + ((int)threadIdx.x + 64 * kWeighWaves * i) / kPieces);
        from[i] = a.q.d + (int64_t)(seq.first + bring[i].token) * a.q.token_bytes + (int64_t)(head * group + bring[i].of_group) * a.q.head_bytes + 16 * ((int)threadIdx.x % kPieces);
    }
    u32x4 x[kOwn];
    float lse = -INFINITY;
    Row asked = mine;                       // the row whose log-sum is on its way
    // (Behind the sequence's last row another one instead, which nobody looks at: without branches the step is one stretch of code.)
    const char* const some_row = a.q.d + (int64_t)seq.first * a.q.token_bytes + (int64_t)(head * group) * a.q.head_bytes;
    const float* const some_lse = a.lse + (int64_t)seq.first * a.heads + head * group;
    auto ask = [&]() {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            x[i] = load16(bring[i].token < seq.n ? from[i] : some_row);
            from[i] += q_step + (move_on(bring[i]) ? q_wrap : 0);
        }
        lse = *(asked.token < seq.n ? lse_from : some_lse);
        lse_from += lse_step + (move_on(asked) ? lse_wrap : 0);
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int p = (int)threadIdx.x + 64 * kWeighWaves * i, c = p % kPieces, r = p / kPieces;
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (x[i][e] & a.q_keep) ^ a.q_flip;
            *reinterpret_cast<u32x4*>(s_q[buf] + c * kPitch + r * 16) = v;
        }
    };
    // A step's beginning: its rows to LDS, the next ones' on their way.  What the step's lanes have:
    int r0 = lo, buf = 1, pos = 0, first_pos = 0, last_pos = 0;             // positions of its first and last token (the last may lie behind the sequence's last)
    bool some = false;
    float lse2 = 0.0f;
    auto begin = [&]() {
        buf ^= 1;
        put(buf);
        pos = w.first + mine.token;
        some = mine.token < seq.n && lse != -INFINITY;
        lse2 = lse * kLog2e;
        move_on(mine);
        ask();
        first_pos = w.first + first_row.token;
        last_pos = w.first + last_row.token;
        move_on(first_row);
        move_on(last_row);
        __syncthreads();                    // the rows are there, and all waves are through with the other buffer
    };
    // do all of the step's rows see all of the wave's keys?
    auto plain = [&]() {
        return first_pos >= j0 + 63 && (a.window == 0 || last_pos - a.window < j0 || j0 + 64 <= a.sinks) && __builtin_amdgcn_ballot_w64(!some) == 0;
    };
    auto add = [&](f32x16& to, const f32x16& st, float lse2) {
#pragma unroll
        for (int e = 0; e < 16; ++e) to[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(to[e]));        // here, and not moved behind the barrier
    };
    auto queries = [&](int t) { return load16(s_q[buf] + (2 * t + hh) * kPitch + col * 16); };
    if (lo < hi) {
        ask();
        begin();
    }
    while (r0 < hi) {
        if (plain()) {
            // Products and weights of different sets side by side: the second set's weights wait for the next step's products of the first
            f32x16 held;
            float held_lse2 = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) held[e] = -INFINITY;
            do {
                u32x4 q[kSteps];
#pragma unroll
                for (int t = 0; t < kSteps; ++t) q[t] = queries(t);
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[0][t], q[t], st);
                add(sum[1], held, held_lse2);
                side_by_side<kSteps>();
#pragma unroll
                for (int e = 0; e < 16; ++e) held[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) held = Num<kBf16>::mma32(k[1][t], q[t], held);
                add(sum[0], st, lse2);
                side_by_side<kSteps>();
                held_lse2 = lse2;
                r0 += kWeighRows;
                if (r0 >= hi) break;
                begin();
            } while (plain());
            add(sum[1], held, held_lse2);
            if (r0 >= hi) break;
        }
        if (last_pos >= j0 && !(a.window > 0 && j0 >= a.sinks && first_pos - a.window >= j0 + 63)) {
            int first_key = j0 + 8 * hh;
            asm volatile("" : "+v"(first_key));
            const Sight sight = sight_of(pos, first_key, a.window, a.sinks);
#pragma unroll
            for (int set = 0; set < 2; ++set) {
                f32x16 st;
#pragma unroll
                for (int e = 0; e < 16; ++e) st[e] = 0.0f;
#pragma unroll
                for (int t = 0; t < kSteps; ++t) st = Num<kBf16>::mma32(k[set][t], queries(t), st);
                // lane (row col, hh): register e has token 8 hh + e % 8 of the set's block e / 8
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], a.scale2, -lse2));
                    sum[set][e] += some && sight.has(32 * set + 16 * (e / 8) + e % 8) ? v : 0.0f;
                }
            }
        }
        r0 += kWeighRows;
        if (r0 < hi) begin();
    }
    // ---- over the 32 rows' lanes
#pragma unroll
    for (int set = 0; set < 2; ++set)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t u = __builtin_bit_cast(uint32_t, sum_over_row(sum[set][e]));
            const auto both = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            sum[set][e] = __builtin_bit_cast(float, (uint32_t)both[0]) + __builtin_bit_cast(float, (uint32_t)both[1]);
        }
    if (col != 0) return;
    if (chunks > 1) {
        f32x4* const part = reinterpret_cast<f32x4*>(a.partial + ((int64_t)chunk * units + unit) * kWeighKeys + 64 * wave + 8 * hh);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) part[4 * b + i] = *(reinterpret_cast<const f32x4*>(&sum[b / 2]) + 2 * (b % 2) + i);
        return;
    }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 8 * (b % 2) + 4 * i;
            w.put(a, to[b], j0 + 16 * b + 8 * hh + 4 * i, (f32x4){sum[b / 2][e], sum[b / 2][e + 1], sum[b / 2][e + 2], sum[b / 2][e + 3]});
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
