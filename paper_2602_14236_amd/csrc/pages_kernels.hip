// Writing K/V rows of text tokens into pages, quantised on the way, and reading them back (gfx950).  Layout of a block: sali.h.
//
// Per group of 32 values, every step one IEEE fp32 operation (this file is compiled with -ffp-contract=off), as in the frame cache:
//   INT8  m = max |x|           scale = m / 127        code = rne(x * (127 / m))              value = code * scale
//   INT4  low = min x           m = max (x - low)      scale = m / 15     code = rne((x - low) * (15 / m))    value = code * scale + low, rounded once
// and the value is then rounded to the pool's 16-bit type.
//
// Both kernels move every byte once and are bound by memory; a block of 256 threads has one 16-token block of one K/V head, or in long batches of up to eight
// heads one after the other.  Rows are contiguous along the head's values, the layout has eight tokens of one value side by side (V) or a token's
// pieces 16 tokens apart (K), so the block is turned over in LDS between 16-byte accesses on both sides: its rows (or their codes), padded so that
// a column's reads fall on different banks.  Codes are made and expanded on the side of the rows, where a group lies in four adjacent lanes.
// Blocks that the new tokens do not fill are written value by value, so that no byte of another token is touched.
// Measured: 2048 tokens of 32 heads in 16 bits, written and read back, 134 MB in 25 us (the caches hold them); three of 12001 and
// 40 heads in 4 bits 1.37 GB in 262 us, 5.2 TB/s (229 us with the same rows again; a copy of 2 GiB through the caches: 4.9).

#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace sali {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// Blocks of 256 threads, twice what the compute units hold: where there are more, a block takes several heads, the next one's data on its way meanwhile.
// Three texts of 12001 tokens, 40 heads, written in 4 bits and read back, through the caches: 296 us, a head a block 380; 32 single tokens 8.1 us, always eight heads a block 19.
constexpr int kEnoughBlocks = 4096;
// Bytes of rows, half of what the last cache holds, from which on they go past the caches: longer ones would only push each other out.  Written and read back, us with and
// without: 10000 tokens of 32 heads (164 MB) 105 and 132 in 16 bits, 83 and 96 in 4, three texts of 12001 tokens and 40 heads in 4 bits 229 and 292; 4096 of 32 heads
// (67 MB) 46 and 43.
constexpr int64_t kPastCaches = 128 << 20;

template <bool kBf16>
struct Half;
template <>
struct Half<false> {
    typedef _Float16 type;
    static constexpr uint32_t kExponent = 0x7C00u;
};
template <>
struct Half<true> {
    typedef __bf16 type;
    static constexpr uint32_t kExponent = 0x7F80u;
};

template <bool kBf16>
union Piece {                               // 16 bytes
    u32x4 u;
    typename Half<kBf16>::type h[8];
    uint16_t b16[8];
    uint8_t b8[16];
};

// rounded to fp32 first, then to 16 bits (a fused instruction would round once)
template <typename T>
__device__ __forceinline__ T rounded_after_f32(float v) {
    asm volatile("" : "+v"(v));
    return (T)v;
}

template <int kCtrl>
__device__ __forceinline__ uint32_t quad_move(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xF, 0xF, true); }
template <int kCtrl>
__device__ __forceinline__ float quad_move(float v) { return __builtin_bit_cast(float, quad_move<kCtrl>(__builtin_bit_cast(uint32_t, v))); }
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E;                 // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kFirst = 0x00, kSecond = 0x55, kThird = 0xAA, kFourth = 0xFF;     // [n,n,n,n]

// is one of the eight values infinite or NaN?  (An exponent of all ones and one more carries into the sign's place.)
template <bool kBf16>
__device__ __forceinline__ bool not_finite(const u32x4& v) {
    constexpr uint32_t kExponents = Half<kBf16>::kExponent * 0x10001u, kOnes = (0x8000u - Half<kBf16>::kExponent) * 0x10001u;
    return ((((v.x & kExponents) + kOnes) | ((v.y & kExponents) + kOnes) | ((v.z & kExponents) + kOnes) | ((v.w & kExponents) + kOnes)) & 0x80008000u) != 0u;
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

// The last sequence whose first slot is not past `slot`, -1 if a start of the batch falls; all threads of the block.  All starts are looked at, since a fall
// anywhere is the whole batch's: up to 256 by every wave for itself, more by all four together and through LDS.  (Us of an append of single tokens, this
// and a search that looks at some of them: 64 of them, 8 heads, 4.3 and 4.3; 200 7.7 and 7.4; 300 10.6 and 9.7; 4096, one head, 22.7 and 14.7.  65: 4.5, through LDS 4.7.)
__device__ __forceinline__ int seq_of_slot(const PageSeqs& q, int64_t slot) {
    __shared__ int s_before[4], s_falls[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), last = q.n_seqs - 1;
    if (last == 0) return 0;
    int before = 0;                         // sequences whose first slot is not past it (the last one counted several times)
    bool falls = false;
    auto look = [&](int first, int next, int i) {
        falls |= first > next;
        before += (int)__popcll(__ballot(max(first, 0) / kBlockTokens <= (int)slot - 2 * i));       // first_slot(first, i) <= slot
    };
    // sequences base + thread + step k
    auto looks = [&](int base, int thread, int step, auto flight) {
        constexpr int kFlight = decltype(flight)::value;
        int first[kFlight], next[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int i = min(base + step * k + thread, last);
            first[k] = q.start[i];
            next[k] = q.start[i + 1];
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) look(first[k], next[k], base + step * k + thread);
    };
    if (q.n_seqs <= 256) {
        if (q.n_seqs <= 64) looks(0, lane, 64, std::integral_constant<int, 1>{});
        else looks(0, lane, 64, std::integral_constant<int, 4>{});
        if (__ballot(falls) != 0) return -1;
    } else {
        for (int base = 0; base < q.n_seqs; base += 1024) looks(base, threadIdx.x, 256, std::integral_constant<int, 4>{});
        const bool any = __ballot(falls) != 0;
        if (lane == 0) {
            s_before[wave] = before;
            s_falls[wave] = any ? 1 : 0;
        }
        __syncthreads();
        if ((s_falls[0] | s_falls[1] | s_falls[2] | s_falls[3]) != 0) return -1;
        before = s_before[0] + s_before[1] + s_before[2] + s_before[3];
    }
    return __builtin_amdgcn_readfirstlane(max(min(before, q.n_seqs) - 1, 0));
}

// What a thread block has: a 16-token block of a sequence, for a run of K/V heads; which tokens of it are the batch's, where their rows and
// the first head's block lie
struct BlockWork {
    char* block;                            // of head 0; NULL: no such page
    int32_t row0;                           // row of the block's token 0 (it may lie before the new tokens)
    int32_t t0, t1;                         // the new tokens of the block
    int32_t head, heads_end;
};
__device__ __forceinline__ bool find_work(const PageGeom& g, const PageSeqs& q, int heads_each, BlockWork& w) {
    const int64_t slot = blockIdx.x;
    const int s = seq_of_slot(q, slot);
    if (s < 0) {
        if (threadIdx.x == 0) atomicOr(q.status, SALI_FAULT_BATCH);
        return false;
    }
    const PageSeq seq = load_seq(q, g, s, threadIdx.x == 0);
    const int pos0 = seq.len - seq.n;                       // position of the first new token
    const int block = block_of_slot(seq, s, slot);
    if (block < 0) return false;
    w.head = (int)blockIdx.y * heads_each;
    w.heads_end = min(w.head + heads_each, g.n_kv);
    w.t0 = max(0, pos0 - block * kBlockTokens);
    w.t1 = min(kBlockTokens, seq.len - block * kBlockTokens);
    w.row0 = seq.first + (block * kBlockTokens - pos0);
    const int page = q.table[(int64_t)s * q.width + (block >> g.blocks_log2)];
    w.block = nullptr;
    if (page >= 0 && page < g.n_pages) {
        const int in_page = block & ((1 << g.blocks_log2) - 1);
        w.block = g.pool + (uint64_t)page * g.page_bytes + (uint32_t)in_page * (g.head_bytes >> g.blocks_log2);
    } else if (threadIdx.x == 0) {
        atomicOr(q.status, SALI_FAULT_PAGE);
    }
    return true;
}

// LDS: the 16 rows of K, then those of V, as values or as codes; a row's length in bytes with what keeps columns on different banks
template <int kStore, int kDim>
struct Rows {
    static constexpr int kBytes = kStore == SALI_STORE_16 ? 2 * kDim : (kStore == SALI_STORE_INT8 ? kDim : kDim / 2);
    static constexpr int kPitch = kBytes + 16;
    static constexpr int kGroups = kDim / kGroup;
};

// kOnce: see kPastCaches
template <int kStore, int kDim, bool kBf16, bool kOnce>
__global__ __launch_bounds__(256) void k_pages_append(PageGeom g, PageSeqs seqs, RowsIn k, RowsIn v, int heads_each) {
    typedef Rows<kStore, kDim> R;
    constexpr int kPieces = kDim / 8, kItems = 32 * kPieces;            // 16-byte pieces of a row, of all rows
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    __shared__ __align__(16) uint8_t s_rows[32 * R::kPitch];
    __shared__ float s_scale[kStore == SALI_STORE_16 ? 1 : 32 * R::kGroups];
    __shared__ uint16_t s_low[kStore == SALI_STORE_INT4 ? 32 * R::kGroups : 1];
    BlockWork w;
    if (!find_work(g, seqs, heads_each, w) || w.block == nullptr) return;

    Piece<kBf16> x[kItems / 256];
    auto ask = [&](int head) {
#pragma unroll
        for (int i = 0; i < kItems / 256; ++i) {
            const int item = (int)threadIdx.x + 256 * i, row = item / kPieces, c = item % kPieces, t = row & 15;
            const RowsIn& in = row < 16 ? k : v;
            x[i].u = (u32x4){0u, 0u, 0u, 0u};
            if (t < w.t0 || t >= w.t1) continue;
            const u32x4* const from = reinterpret_cast<const u32x4*>(in.d + (int64_t)(w.row0 + t) * in.token_bytes + (int64_t)head * in.head_bytes + c * 16);
            if constexpr (kOnce) x[i].u = __builtin_nontemporal_load(from);
            else x[i].u = *from;
        }
    };
    ask(w.head);
    bool bad = false;
    for (int head = w.head; head < w.heads_end; ++head) {
        char* const block = w.block + (uint64_t)head * g.head_bytes;
        if (head > w.head) __syncthreads();                     // the head before is out of LDS
        constexpr int kOwn = kItems / 256;
        if constexpr (kStore == SALI_STORE_16) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int item = (int)threadIdx.x + 256 * i, row = item / kPieces, c = item % kPieces;
                bad |= not_finite<kBf16>(x[i].u);
                *reinterpret_cast<u32x4*>(s_rows + row * R::kPitch + c * 16) = x[i].u;
            }
        } else {
            constexpr float kSteps = kStore == SALI_STORE_INT8 ? 127.0f : 15.0f;
            float f[kOwn][8], m[kOwn], low[kOwn];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[i][e] = (float)x[i].h[e];
                low[i] = 0.0f;
                if constexpr (kStore == SALI_STORE_INT8) {
                    float top = fabsf(f[i][0]);
#pragma unroll
                    for (int e = 1; e < 8; ++e) top = fmaxf(top, fabsf(f[i][e]));
                    top = fmaxf(top, quad_move<kSwap1>(top));
                    m[i] = fmaxf(top, quad_move<kSwap2>(top));
                } else {
                    float least = f[i][0], high = f[i][0];
#pragma unroll
                    for (int e = 1; e < 8; ++e) {
                        least = fminf(least, f[i][e]);
                        high = fmaxf(high, f[i][e]);
                    }
                    least = fminf(least, quad_move<kSwap1>(least));
                    least = fminf(least, quad_move<kSwap2>(least));
                    high = fmaxf(high, quad_move<kSwap1>(high));
                    high = fmaxf(high, quad_move<kSwap2>(high));
                    // rounding keeps the order of numbers, so the largest of the rounded differences is this one
                    m[i] = high - least;
                    low[i] = least;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[i][e] = f[i][e] - least;
                }
            }
            // one division for the quad's four (two groups' steps / m and m / steps): a lane has one of them
            const float of = (threadIdx.x & 2) != 0 ? m[kOwn - 1] : m[0];
            const float quotient = (threadIdx.x & 1) != 0 ? of / kSteps : kSteps / of;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int item = (int)threadIdx.x + 256 * i, row = item / kPieces, c = item % kPieces;
                const float inv = i == 0 ? quad_move<kFirst>(quotient) : quad_move<kThird>(quotient);
                const float step = i == 0 ? quad_move<kSecond>(quotient) : quad_move<kFourth>(quotient);
                // a group with an infinity or NaN, or one too wide or too small for fp32 steps, is stored as zeros: every value of the pages is finite
                uint32_t odd = not_finite<kBf16>(x[i].u) || !(m[i] <= 3.402823466e38f) ? 1u : 0u;
                odd |= quad_move<kSwap1>(odd);
                odd |= quad_move<kSwap2>(odd);
                bad |= odd != 0u;
                const bool some = odd == 0u && m[i] > 0.0f && inv <= 3.402823466e38f;
                if ((c & 3) == 0) {
                    s_scale[row * R::kGroups + c / 4] = some ? step : 0.0f;
                    if constexpr (kStore == SALI_STORE_INT4) {
                        Piece<kBf16> z;
                        z.h[0] = (typename Half<kBf16>::type)(odd == 0u ? low[i] : 0.0f);       // exact: one of the values
                        s_low[row * R::kGroups + c / 4] = z.b16[0];
                    }
                }
                // |f| <= m, so the products lie within the steps (give or take a rounding) and need no clamp; adding 1.5 2^23 rounds to the nearest
                // even whole number and leaves it in the low byte, in two's complement
                uint32_t q[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = __builtin_bit_cast(uint32_t, f[i][e] * inv + 12582912.0f);
                const uint32_t keep = some ? 0xFFFFFFFFu : 0u;
                const u32x2 code = {low_bytes(q[0], q[1], q[2], q[3]) & keep, low_bytes(q[4], q[5], q[6], q[7]) & keep};
                if constexpr (kStore == SALI_STORE_INT8) {
                    *reinterpret_cast<u32x2*>(s_rows + row * R::kPitch + c * 8) = code;
                } else {
                    // lanes 0, 1 of a quad hold values 0 .. 15 of the group, lanes 2, 3 the others, which go to the high halves of the same bytes
                    const uint32_t a = quad_move<kSwap2>(code.x) << 4 | code.x, b = quad_move<kSwap2>(code.y) << 4 | code.y;
                    if ((c & 2) == 0) *reinterpret_cast<u32x2*>(s_rows + row * R::kPitch + (c / 4) * 16 + (c & 1) * 8) = (u32x2){a, b};
                }
            }
        }
        __syncthreads();
        if (head + 1 < w.heads_end) ask(head + 1);              // on its way while this one is written

        // K: pieces of 16 bytes, [piece of the row][place]
#pragma unroll
        for (int i = 0; i < (R::kBytes + 255) / 256; ++i) {
            const int p = (int)threadIdx.x + 256 * i, t = token_of_place(p & 15);
            if (p < R::kBytes && t >= w.t0 && t < w.t1)
                *reinterpret_cast<u32x4*>(block + p * 16) = *reinterpret_cast<const u32x4*>(s_rows + t * R::kPitch + (p >> 4) * 16);
        }
        // V: for each half of the block and each element of a row (a value, a code, a byte of two codes) those of eight tokens
        constexpr int kElem = kStore == SALI_STORE_16 ? 2 : 1, kElems = R::kBytes / kElem;
#pragma unroll
        for (int i = 0; i < (2 * kElems + 255) / 256; ++i) {
            const int p = (int)threadIdx.x + 256 * i, a = p / kElems, e = p % kElems;
            if (p >= 2 * kElems) continue;
            Piece<kBf16> o;
            o.u = (u32x4){0u, 0u, 0u, 0u};
            const uint8_t* column = s_rows + (16 + 8 * a) * R::kPitch + e * kElem;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if constexpr (kElem == 2) o.b16[t] = *reinterpret_cast<const uint16_t*>(column + t * R::kPitch);
                else o.b8[t] = column[t * R::kPitch];
            }
            char* dst = block + kAt.v + (uint32_t)p * (8 * kElem);
            if (w.t0 <= 8 * a && w.t1 >= 8 * a + 8) {
                if constexpr (kElem == 2) *reinterpret_cast<u32x4*>(dst) = o.u;
                else *reinterpret_cast<u32x2*>(dst) = (u32x2){o.u.x, o.u.y};
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    if (8 * a + t < w.t0 || 8 * a + t >= w.t1) continue;
                    if constexpr (kElem == 2) reinterpret_cast<uint16_t*>(dst)[t] = o.b16[t];
                    else reinterpret_cast<uint8_t*>(dst)[t] = o.b8[t];
                }
            }
        }
        if constexpr (kStore != SALI_STORE_16) {
            const int p = (int)threadIdx.x;                     // [K, V][group][16]
            if (p < 32 * R::kGroups) {
                const int side = p / (16 * R::kGroups), group = p / 16 % R::kGroups, t = side == 0 ? token_of_place(p & 15) : p & 15;
                if (t >= w.t0 && t < w.t1) {
                    const int from = (16 * side + t) * R::kGroups + group;
                    reinterpret_cast<float*>(block + kAt.ks)[p] = s_scale[from];
                    if constexpr (kStore == SALI_STORE_INT4) reinterpret_cast<uint16_t*>(block + kAt.kz)[p] = s_low[from];
                }
            }
        }
    }
    if (bad) atomicOr(seqs.status, SALI_FAULT_NONFINITE);
}

// kOnce: see kPastCaches
template <int kStore, int kDim, bool kBf16, bool kOnce>
__global__ __launch_bounds__(256) void k_pages_read(PageGeom g, PageSeqs seqs, RowsOut k, RowsOut v, int heads_each) {
    typedef Rows<kStore, kDim> R;
    typedef typename Half<kBf16>::type T;
    constexpr int kPieces = kDim / 8, kItems = 32 * kPieces;
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    constexpr int kElem = kStore == SALI_STORE_16 ? 2 : 1, kElems = R::kBytes / kElem;
    constexpr int kKLoads = (R::kBytes + 255) / 256, kVLoads = (2 * kElems + 255) / 256;
    __shared__ __align__(16) uint8_t s_rows[32 * R::kPitch];
    __shared__ float s_scale[kStore == SALI_STORE_16 ? 1 : 32 * R::kGroups];
    __shared__ uint16_t s_low[kStore == SALI_STORE_INT4 ? 32 * R::kGroups : 1];
    BlockWork w;
    if (!find_work(g, seqs, heads_each, w)) return;
    u32x4 kp[kKLoads];
    Piece<kBf16> vp[kVLoads];
    float scale_in = 0.0f;
    uint16_t low_in = 0;
    auto ask = [&](int head) {
        if (w.block == nullptr) return;
        const char* const block = w.block + (uint64_t)head * g.head_bytes;
#pragma unroll
        for (int i = 0; i < kKLoads; ++i) {
            const int p = (int)threadIdx.x + 256 * i;
            if (p < R::kBytes) kp[i] = *reinterpret_cast<const u32x4*>(block + p * 16);
        }
#pragma unroll
        for (int i = 0; i < kVLoads; ++i) {
            const int p = (int)threadIdx.x + 256 * i;
            if (p >= 2 * kElems) continue;
            const char* src = block + kAt.v + (uint32_t)p * (8 * kElem);
            if constexpr (kElem == 2) {
                vp[i].u = *reinterpret_cast<const u32x4*>(src);
            } else {
                const u32x2 c = *reinterpret_cast<const u32x2*>(src);
                vp[i].u = (u32x4){c.x, c.y, 0u, 0u};
            }
        }
        if constexpr (kStore != SALI_STORE_16) {
            const int p = (int)threadIdx.x;
            if (p < 32 * R::kGroups) {
                scale_in = reinterpret_cast<const float*>(block + kAt.ks)[p];
                if constexpr (kStore == SALI_STORE_INT4) low_in = reinterpret_cast<const uint16_t*>(block + kAt.kz)[p];
            }
        }
    };
    ask(w.head);
    for (int head = w.head; head < w.heads_end; ++head) {
        if (head > w.head) __syncthreads();                     // the head before is out of LDS
        if (w.block != nullptr) {
            if constexpr (kStore != SALI_STORE_16) {
                const int p = (int)threadIdx.x;
                if (p < 32 * R::kGroups) {
                    const int side = p / (16 * R::kGroups), group = p / 16 % R::kGroups, t = side == 0 ? token_of_place(p & 15) : p & 15;
                    const int to = (16 * side + t) * R::kGroups + group;
                    s_scale[to] = scale_in;
                    if constexpr (kStore == SALI_STORE_INT4) s_low[to] = low_in;
                }
            }
#pragma unroll
            for (int i = 0; i < kKLoads; ++i) {
                const int p = (int)threadIdx.x + 256 * i;
                if (p < R::kBytes) *reinterpret_cast<u32x4*>(s_rows + token_of_place(p & 15) * R::kPitch + (p >> 4) * 16) = kp[i];
            }
#pragma unroll
            for (int i = 0; i < kVLoads; ++i) {
                const int p = (int)threadIdx.x + 256 * i, a = p / kElems, e = p % kElems;
                if (p >= 2 * kElems) continue;
                uint8_t* column = s_rows + (16 + 8 * a) * R::kPitch + e * kElem;
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    if constexpr (kElem == 2) *reinterpret_cast<uint16_t*>(column + t * R::kPitch) = vp[i].b16[t];
                    else column[t * R::kPitch] = vp[i].b8[t];
                }
            }
        }
        __syncthreads();
        if (head + 1 < w.heads_end) ask(head + 1);              // on its way while this one is written
#pragma unroll
        for (int i = 0; i < kItems / 256; ++i) {
            const int item = (int)threadIdx.x + 256 * i, row = item / kPieces, c = item % kPieces, t = row & 15;
            if (t < w.t0 || t >= w.t1) continue;
            Piece<kBf16> o;
            o.u = (u32x4){0u, 0u, 0u, 0u};
            if (w.block != nullptr) {
                if constexpr (kStore == SALI_STORE_16) {
                    o.u = *reinterpret_cast<const u32x4*>(s_rows + row * R::kPitch + c * 16);
                } else {
                    const float scale = s_scale[row * R::kGroups + c / 4];
                    Piece<kBf16> code;
                    if constexpr (kStore == SALI_STORE_INT8) {
                        const u32x2 q = *reinterpret_cast<const u32x2*>(s_rows + row * R::kPitch + c * 8);
                        code.u = (u32x4){q.x, q.y, 0u, 0u};
#pragma unroll
                        for (int e = 0; e < 8; ++e) o.h[e] = rounded_after_f32<T>((float)(int)(int8_t)code.b8[e] * scale);
                    } else {
                        Piece<kBf16> z;
                        z.b16[0] = s_low[row * R::kGroups + c / 4];
                        const float low = (float)z.h[0];
                        const u32x2 q = *reinterpret_cast<const u32x2*>(s_rows + row * R::kPitch + (c / 4) * 16 + (c & 1) * 8);
                        const int shift = (c & 2) * 2;          // values 16 .. 31 of a group lie in the high halves
                        code.u = (u32x4){q.x >> shift & 0x0F0F0F0Fu, q.y >> shift & 0x0F0F0F0Fu, 0u, 0u};
#pragma unroll
                        for (int e = 0; e < 8; ++e) o.h[e] = rounded_after_f32<T>(__builtin_fmaf((float)code.b8[e], scale, low));
                    }
                }
            }
            const RowsOut& out = row < 16 ? k : v;
            u32x4* const to = reinterpret_cast<u32x4*>(out.d + (int64_t)(w.row0 + t) * out.token_bytes + (int64_t)head * out.head_bytes + c * 16);
            if constexpr (kOnce) __builtin_nontemporal_store(o.u, to);
            else *to = o.u;
        }
    }
}

template <typename F>
hipError_t by_type(int dtype, int store, int dim, const F& go) {
    auto with_dim = [&](auto bf16, auto st) {
        if (dim == 64) go(bf16, st, std::integral_constant<int, 64>{});
        else go(bf16, st, std::integral_constant<int, 128>{});
    };
    auto with_store = [&](auto bf16) {
        if (store == SALI_STORE_16) with_dim(bf16, std::integral_constant<int, SALI_STORE_16>{});
        else if (store == SALI_STORE_INT8) with_dim(bf16, std::integral_constant<int, SALI_STORE_INT8>{});
        else with_dim(bf16, std::integral_constant<int, SALI_STORE_INT4>{});
    };
    if (dtype == SALI_DTYPE_BF16) with_store(std::true_type{});
    else with_store(std::false_type{});
    return hipGetLastError();
}

// Heads of a thread block: as many as leave a few rounds of blocks for the compute units.  Finding the work is a chain of four trips to memory; a block that
// walks several heads has the next one's data on its way meanwhile.
struct Shares {
    int heads_each;
    bool once;
    dim3 grid;
};
Shares shares(const PageGeom& g, const PageSeqs& q, int dim) {
    const int64_t slots = q.n_tokens / kBlockTokens + 2ll * q.n_seqs;
    const int64_t most = slots * g.n_kv / kEnoughBlocks;
    const int each = (int)std::max<int64_t>(1, std::min<int64_t>(most, std::min(g.n_kv, 8)));
    return {each, 4ll * dim * g.n_kv * q.n_tokens >= kPastCaches, dim3((unsigned)slots, (unsigned)((g.n_kv + each - 1) / each))};
}

}  // namespace

hipError_t launch_pages_append(int dtype, int store, int dim, const PageGeom& g, const PageSeqs& seqs, const RowsIn& k, const RowsIn& v, hipStream_t s) {
    const Shares sh = shares(g, seqs, dim);
    return by_type(dtype, store, dim, [&](auto bf16, auto st, auto d) {
        auto go = [&](auto once) {
            hipLaunchKernelGGL((k_pages_append<decltype(st)::value, decltype(d)::value, decltype(bf16)::value, decltype(once)::value>), sh.grid, dim3(256), 0, s, g, seqs, k, v,
                               sh.heads_each);
        };
        if (sh.once) go(std::true_type{});
        else go(std::false_type{});
    });
}

hipError_t launch_pages_read(int dtype, int store, int dim, const PageGeom& g, const PageSeqs& seqs, const RowsOut& k, const RowsOut& v, hipStream_t s) {
    const Shares sh = shares(g, seqs, dim);
    return by_type(dtype, store, dim, [&](auto bf16, auto st, auto d) {
        auto go = [&](auto once) {
            hipLaunchKernelGGL((k_pages_read<decltype(st)::value, decltype(d)::value, decltype(bf16)::value, decltype(once)::value>), sh.grid, dim3(256), 0, s, g, seqs, k, v,
                               sh.heads_each);
        };
        if (sh.once) go(std::true_type{});
        else go(std::false_type{});
    });
}

}  // namespace sali
