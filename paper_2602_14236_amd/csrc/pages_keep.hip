// Cutting a text down: which tokens stay, by their attention weights, and moving their rows together (gfx950).

#include <algorithm>
#include <type_traits>

#include "pages_stream.h"

namespace sali {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kDigits[3] = {21, 10, 0};     // lowest bit of each digit: 11, 11 and 10 bits
constexpr int kBins = 2048;
constexpr int kInLds = 32768;               // keys that stay in LDS

// Weights as whole numbers in the same order: a NaN above all, tokens of no page below all.
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0xFFFFFFFFu;
    const uint32_t u = __builtin_bit_cast(uint32_t, w == 0.0f ? 0.0f : w);
    return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}

// A block a sequence and K/V head.  The weight that the last of the tokens that stay has is found digit by digit, highest first, in a histogram of the tokens that are alike so
// far; then every wave takes a stretch of tokens, counts those above and at that weight, and writes the places of those that stay behind what the waves before it have.
// Bound by its chain of passes over LDS: three texts of up to 24001 tokens, 8 heads, in 27 us, where their weights are 1.7 MB.  Keys are kept there once read (48 us
// with loads of one weight), several on their way together and without branches (33 us with them).  Keys behind those that LDS has room for are fetched again in every pass, page and
// weight one after the other: 32768 tokens of 8 heads 34 us, 131072 255.
__global__ __launch_bounds__(kSelectThreads) void k_pages_select(PagesSelect a) {
    __shared__ uint32_t s_keys[kInLds];
    __shared__ uint32_t s_bins[kBins];
    __shared__ uint32_t s_wave[2][kSelectWaves];
    __shared__ uint32_t s_found[2];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int s = (int)(blockIdx.x / (uint32_t)a.geom.n_kv), head = (int)(blockIdx.x % (uint32_t)a.geom.n_kv);
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, tid, kSelectThreads);
    const PageSeq seq = load_seq(a.seqs, a.geom, s, head == 0 && tid == 0);
    if (__syncthreads_or(falls.some() ? 1 : 0) != 0) {
        if (tid == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    bool fits;
    read_seq(a.seqs, a.geom, s, fits);
    if (!fits) return;
    int32_t* const out = a.keep + ((int64_t)s * a.geom.n_kv + head) * a.budget;
    const int n = seq.n, base = seq.len - seq.n;
    if (n <= a.budget) {
        each_from(tid, a.budget, kSelectThreads, [&](uint32_t i) { out[i] = i < (uint32_t)n ? (int)i : -1; });
        return;
    }
    const int shift = a.geom.blocks_log2 + 4, page_tokens = 1 << shift;
    const int32_t* const table = a.seqs.table + (int64_t)s * a.seqs.width;
    auto page_at = [&](int pos) {
        const int page = table[pos >> shift];
        return (unsigned)page < (unsigned)a.geom.n_pages ? page : -1;
    };
    auto weights_at = [&](int page, int pos) { return a.weights + ((((int64_t)page * a.geom.n_kv + head) << shift) + (pos & (page_tokens - 1))); };
    auto key_in_pages = [&](int i) -> uint32_t {            // of the i-th of the sequence's new tokens
        const int page = page_at(base + i);
        if (page >= 0) return key_of(*weights_at(page, base + i));
        atomicOr(a.seqs.status, SALI_FAULT_PAGE);
        return 0u;
    };
    // sum over the waves before this one
    auto before_wave = [&](const uint32_t* of_wave) {
        const int upto = wave_scan(lane < kSelectWaves ? (int)of_wave[lane] : 0);
        return wave == 0 ? 0u : (uint32_t)__builtin_amdgcn_readlane(upto, wave - 1);
    };
    // those that are chosen from: first .. first + m - 1
    const int first = a.sinks, m = n - a.sinks - a.recent;
    uint32_t room = (uint32_t)(a.budget - a.sinks - a.recent);
    // (Where all are in LDS, reading them takes no branch, and several are on their way together.)
    auto choose = [&](auto all_in_lds) {
        auto key = [&](int j) {
            if constexpr (decltype(all_in_lds)::value) return s_keys[j];
            else return j < kInLds ? s_keys[j] : key_in_pages(first + j);
        };
        uint32_t at = 0xFFFFFFFFu, ties = 0;                    // keys above `at` stay, and the first `ties` of those at it
        if (room > 0) {
            // four at a time, aligned as the pages are, and several of them on their way together
            const int pos_end = base + first + min(m, kInLds), quad0 = (base + first) & ~3;
            constexpr int kFlight = 8;
            for (int64_t pos0 = quad0; pos0 < pos_end; pos0 += 4 * kFlight * kSelectThreads) {
                int page[kFlight];
                f32x4 w[kFlight];
#pragma unroll
                for (int i = 0; i < kFlight; ++i) {
                    const int64_t pos = pos0 + 4 * (kSelectThreads * i + tid);
                    page[i] = pos < pos_end ? page_at((int)pos) : -2;
                }
#pragma unroll
                for (int i = 0; i < kFlight; ++i)
                    w[i] = page[i] >= 0 ? *reinterpret_cast<const f32x4*>(weights_at(page[i], (int)(pos0 + 4 * (kSelectThreads * i + tid)))) : (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < kFlight; ++i) {
                    if (page[i] == -1) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                    const int64_t pos = pos0 + 4 * (kSelectThreads * i + tid);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (pos + e >= base + first && pos + e < pos_end) s_keys[(int)(pos + e) - base - first] = page[i] >= 0 ? key_of(w[i][e]) : 0u;
                }
            }
            uint32_t prefix = 0;
            for (int d = 0; d < 3; ++d) {
                const int low = kDigits[d], high = d == 0 ? 32 : kDigits[d - 1];
                for (int b = tid; b < kBins; b += kSelectThreads) s_bins[b] = 0;
                __syncthreads();
                // several keys on their way together: the loop is a chain of trips to LDS
                constexpr int kKeys = 4;
                each_from(tid, m, kKeys * kSelectThreads, [&](uint32_t j0) {
                    uint32_t k[kKeys];
#pragma unroll
                    for (int i = 0; i < kKeys; ++i) k[i] = key((int)min(j0 + (uint32_t)(kSelectThreads * i), (uint32_t)m - 1u));
#pragma unroll
                    for (int i = 0; i < kKeys; ++i)
                        if (j0 + (uint32_t)(kSelectThreads * i) < (uint32_t)m && (d == 0 || k[i] >> high == prefix))
                            atomicAdd(&s_bins[k[i] >> low & (kBins - 1) & ((1u << (high - low)) - 1u)], 1u);
                });
                __syncthreads();
                // tokens from the highest bin down: thread t has bins kBins - 1 - 2 t and the one below
                const uint32_t upper = s_bins[kBins - 1 - 2 * tid], lower = s_bins[kBins - 2 - 2 * tid];
                uint32_t sum = (uint32_t)wave_scan((int)(upper + lower));
                if (lane == 63) s_wave[0][wave] = sum;
                __syncthreads();
                sum += before_wave(s_wave[0]);
                const uint32_t before = sum - upper - lower;
                if (before < room && sum >= room) {
                    const bool in_upper = before + upper >= room;
                    s_found[0] = (uint32_t)(kBins - 1 - 2 * tid - (in_upper ? 0 : 1));
                    s_found[1] = room - before - (in_upper ? 0u : upper);
                }
                __syncthreads();
                prefix = prefix << (high - low) | s_found[0];
                room = s_found[1];
            }
            at = prefix;
            ties = room;
        }
        // every wave a stretch of the sequence's tokens
        const int stretch = ((n + kSelectWaves - 1) / kSelectWaves + 63) & ~63, lo = (int)min((int64_t)n, (int64_t)stretch * wave), hi = (int)min((int64_t)n, (int64_t)lo + stretch);
        constexpr int kLooks = 8;               // of a lane, on their way together
        auto each = [&](auto look) {
            for (int64_t i0 = lo; i0 < hi; i0 += 64 * kLooks) {
                uint32_t k[kLooks];
#pragma unroll
                for (int x = 0; x < kLooks; ++x) {
                    const int64_t i = i0 + 64 * x + lane;
                    k[x] = decltype(all_in_lds)::value || ties > 0 ? key((int)min(max(i - first, (int64_t)0), (int64_t)m - 1)) : 0u;
                }
#pragma unroll
                for (int x = 0; x < kLooks; ++x) {
                    const int64_t i = i0 + 64 * x + lane;
                    const bool from = i >= first && i < first + m;
                    look((int)i, i < hi && (!from || (ties > 0 && k[x] > at)), ties > 0 && i < hi && from && k[x] == at);
                }
            }
        };
        uint32_t sure = 0, tied = 0;
        each([&](int, bool stays, bool tie) {
            sure += (uint32_t)__popcll(__ballot(stays));
            tied += (uint32_t)__popcll(__ballot(tie));
        });
        __syncthreads();                                        // s_wave has been read
        if (lane == 0) {
            s_wave[0][wave] = sure;
            s_wave[1][wave] = tied;
        }
        __syncthreads();
        sure = before_wave(s_wave[0]);
        tied = before_wave(s_wave[1]);
        uint32_t next = sure + min(tied, ties);
        const uint64_t lanes_before = (1ull << lane) - 1ull;
        each([&](int i, bool stays, bool tie) {
            const uint64_t all_ties = __ballot(tie);
            stays |= tie && tied + (uint32_t)__popcll(all_ties & lanes_before) < ties;
            tied += (uint32_t)__popcll(all_ties);
            const uint64_t all = __ballot(stays);
            if (stays) out[next + (uint32_t)__popcll(all & lanes_before)] = i;
            next += (uint32_t)__popcll(all);
        });
    };
    if (m <= kInLds) choose(std::true_type{});
    else choose(std::false_type{});
}

// ---- moving rows
// A block of 16 tokens falls apart into strips that move by themselves: a group of 32 values of K or of V, with its scales; and the weights.  A thread block takes one strip of a
// sequence and K/V head (into other pages a strip of K with that of V), kTokens tokens at a time, as they are stored: K's pieces of 16 bytes from place to place, V's values eight tokens at a time.
//
// In place, a row never moves to a higher position, so rows that are still to be read lie behind all that have been written if the chunks are taken in their
// order, each read whole before it is written: one thread block walks a strip.  Into other pages chunks are blocks of their own.
//
// Bound by the lines that rows lie in: those that stay are spread, so that nearly all of the source is touched.  4096 of up to 24001 tokens, three texts, 8 heads of 128 in 16
// bits: 171 MB read and 51 written in 41 us, 5.4 TB/s (57 where a block takes a strip of K or of V alone: half as much for the same chain of lengths, list, tables
// and rows; 43 with V's values asked for behind branches; chunks of 128 or blocks of 128 threads 40).  In place, 32 drafts of 16 tokens: 9 us, a launch and its chain of list, tables, rows;
// the three texts 91 us (37 elsewhere, the call alone): a chunk waits for the one before.
constexpr int kKeepThreads = 256;

template <int kStore, int kDim>
struct Strip {
    static constexpr int kGroups = kDim / 32;
    static constexpr int kPieces = kStore == SALI_STORE_16 ? 4 : (kStore == SALI_STORE_INT8 ? 2 : 1);       // of K, 16 bytes
    static constexpr int kElem = kStore == SALI_STORE_16 ? 2 : 1;                                           // bytes of V's values, codes or pairs of codes
    static constexpr int kElems = kStore == SALI_STORE_INT4 ? 16 : 32;
};

// kTokens: of a chunk
template <int kStore, int kDim, bool kInPlace, int kTokens>
__global__ __launch_bounds__(kKeepThreads) void k_pages_keep(PagesKeep a, int chunks) {
    typedef Strip<kStore, kDim> S;
    constexpr BlockLayout kAt = block_layout(kStore, kDim);
    constexpr int kKItems = kTokens * S::kPieces, kVItems = kTokens / 8 * S::kElems;
    constexpr int kKOwn = (kKItems + kKeepThreads - 1) / kKeepThreads, kVOwn = (kVItems + kKeepThreads - 1) / kKeepThreads;
    constexpr uint64_t kNone = ~0ull, kZeros = ~0ull - 1;
    __shared__ uint64_t s_from[kTokens];                    // where the token's block lies, bits 0 to 3 its place there; kNone: nothing moves, kZeros: of no page
    __shared__ uint64_t s_to[kTokens / 16];
    const int tid = threadIdx.x;
    constexpr bool kBoth = !kInPlace;                       // a strip is a group of K and that of V
    constexpr int kStrips = kBoth ? S::kGroups : 2 * S::kGroups;
    const uint32_t n_strips = kStrips + (a.weights != nullptr ? 1 : 0), in_heads = blockIdx.x / (uint32_t)a.geom.n_kv, in_strips = in_heads / n_strips;
    const int head = (int)(blockIdx.x - in_heads * (uint32_t)a.geom.n_kv), strip = (int)(in_heads - in_strips * n_strips);
    const int s = (int)(in_strips / (uint32_t)chunks), nth = (int)(in_strips - (uint32_t)s * (uint32_t)chunks);
    const bool notes = strip == 0;
    const StartFalls falls(a.seqs.start, a.seqs.n_seqs, tid, kKeepThreads);
    const PageSeq seq = load_seq(a.seqs, a.geom, s, notes && tid == 0);
    if (__syncthreads_or(falls.some() ? 1 : 0) != 0) {
        if (tid == 0) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
        return;
    }
    if (seq.n == 0) return;
    const int shift = a.geom.blocks_log2 + 4, base = seq.len - seq.n, base0 = base & ~15;
    const int32_t* const keep = a.keep + ((int64_t)s * a.keep_heads + (a.keep_heads > 1 ? head : 0)) * a.width;
    const int32_t* const table = a.seqs.table + (int64_t)s * a.seqs.width;
    const int32_t* const to_table = a.to + (int64_t)s * a.to_width;
    const uint32_t block_bytes = a.geom.head_bytes >> a.geom.blocks_log2;
    const bool weights = strip == kStrips, keys = kBoth || strip < S::kGroups, values = kBoth || strip >= S::kGroups;    // what moves: the weights, else K, V
    const int group = strip % S::kGroups;
    // byte of a token's block of the strip's head, or the number of its first weight
    auto block_at = [&](int page, int pos) -> uint64_t {
        const uint32_t in_page = (uint32_t)(pos & ((1 << shift) - 1));
        if (weights) return (((uint64_t)(uint32_t)page * (uint32_t)a.geom.n_kv + (uint32_t)head) << shift) + (in_page & ~15u);
        return (uint64_t)(uint32_t)page * a.geom.page_bytes + (uint64_t)head * a.geom.head_bytes + (uint64_t)(in_page >> 4) * block_bytes;
    };
    const int64_t last = min((int64_t)base + a.width, (int64_t)seq.len);             // positions that rows move to: base .. last - 1, as many as the region has at the most
    const int step = kInPlace ? 1 : chunks;
    for (int64_t chunk = kInPlace ? 0 : nth; base0 + chunk * kTokens < last; chunk += step) {
        const int pos0 = (int)(base0 + chunk * kTokens);
        // ---- where rows lie and go
        bool some = false;
        for (int t = tid; t < kTokens; t += kKeepThreads) {
            const int64_t pos = (int64_t)pos0 + t, i = pos - base;
            uint64_t from = kNone;
            if (i >= 0 && pos < last) {
                const int k = keep[i];
                const int64_t to_page_nth = pos >> shift;
                if (k >= 0 && (k >= seq.n || (kInPlace && k < i) || to_page_nth >= a.to_width)) {
                    if (notes) atomicOr(a.seqs.status, SALI_FAULT_BATCH);
                } else if (k >= 0) {
                    const int page = table[(base + k) >> shift], to_page = to_table[to_page_nth];
                    const bool is = (unsigned)page < (unsigned)a.geom.n_pages, to_is = (unsigned)to_page < (unsigned)a.geom.n_pages;
                    if (notes && !(is && to_is)) atomicOr(a.seqs.status, SALI_FAULT_PAGE);
                    if (to_is) from = is ? block_at(page, base + k) | (uint64_t)((base + k) & 15) : kZeros;
                }
            }
            s_from[t] = from;
            some |= from != kNone;
            if ((t & 15) == 0) {
                const int64_t nth = pos >> shift;
                const int to_page = pos < last && nth < a.to_width ? to_table[nth] : -1;
                s_to[t / 16] = (unsigned)to_page < (unsigned)a.geom.n_pages ? block_at(to_page, (int)pos) : kNone;
            }
        }
        if (__syncthreads_or(some ? 1 : 0) == 0) {
            __syncthreads();
            continue;
        }
        // ---- read
        const char* const pool = a.geom.pool;
        constexpr int kX = kBoth ? kKOwn + kVOwn : (kKOwn > kVOwn ? kKOwn : kVOwn), kFirstV = kBoth ? kKOwn : 0, kSides = kBoth ? 2 : 1, kOwn = kTokens / kKeepThreads + 1;
        u32x4 x[kX];
        uint32_t scale[kSides * kOwn];
        uint16_t low[kSides * kOwn];
        auto from_of = [&](int t, int& place) -> uint64_t {
            const uint64_t f = s_from[t];
            place = (int)(f & 15u);
            return f >= kZeros ? f : f & ~15ull;
        };
        if (weights) {
            for (int t = tid, i = 0; t < kTokens; t += kKeepThreads, ++i) {
                const uint64_t f = s_from[t];
                scale[i] = f < kZeros ? reinterpret_cast<const uint32_t*>(a.weights)[f] : 0u;
            }
        } else {
            if (keys) {
#pragma unroll
                for (int i = 0; i < kKOwn; ++i) {
                    const int p = tid + kKeepThreads * i;
                    int place;
                    x[i] = (u32x4){0u, 0u, 0u, 0u};
                    if (p >= kKItems) continue;
                    const uint64_t f = from_of(p % kTokens, place);
                    if (f < kZeros) x[i] = *reinterpret_cast<const u32x4*>(pool + f + ((group * S::kPieces + p / kTokens) * 16 + place_of_token(place)) * 16);
                }
            }
            if (values) {
#pragma unroll
                for (int i = 0; i < kVOwn; ++i) {
                    const int p = tid + kKeepThreads * i, e = p % S::kElems, octet = p / S::kElems;
                    u32x4& v = x[kFirstV + i];
                    v = (u32x4){0u, 0u, 0u, 0u};
                    if (p >= kVItems) continue;
                    // (Into other pages all are asked for, of nothing the pool's first, so that they are on their way together; of a draft most stay where they are.)
                    uint32_t of[8];
                    bool is[8];
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        int place;
                        const uint64_t f = from_of(8 * octet + t, place);
                        is[t] = f < kZeros;
                        const char* const at = pool + (is[t] ? f : 0) + kAt.v + (((place >> 3) * (S::kGroups * S::kElems) + group * S::kElems + e) * 8 + (place & 7)) * S::kElem;
                        of[t] = 0u;
                        if (kInPlace && !is[t]) continue;
                        if constexpr (S::kElem == 2) of[t] = *reinterpret_cast<const uint16_t*>(at);
                        else of[t] = *reinterpret_cast<const uint8_t*>(at);
                    }
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[S::kElem == 2 ? t / 2 : t / 4] |= (is[t] ? of[t] : 0u) << (8 * S::kElem * (t % (4 / S::kElem)));
                }
            }
            if constexpr (kStore != SALI_STORE_16)
#pragma unroll
                for (int side = 0; side < kSides; ++side)
                    for (int t = tid, i = side * kOwn; t < kTokens; t += kKeepThreads, ++i) {
                        int place;
                        const uint64_t f = from_of(t, place);
                        const bool v = kBoth ? side == 1 : values;
                        scale[i] = 0u;
                        low[i] = 0;
                        if (f >= kZeros) continue;
                        const uint32_t at = (uint32_t)(group * 16 + (v ? place : place_of_token(place)));
                        scale[i] = *reinterpret_cast<const uint32_t*>(pool + f + (v ? kAt.vs : kAt.ks) + at * 4);
                        if constexpr (kStore == SALI_STORE_INT4) low[i] = *reinterpret_cast<const uint16_t*>(pool + f + (v ? kAt.vz : kAt.kz) + at * 2);
                    }
        }
        if constexpr (kInPlace) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                          // all of the chunk is here before any of it is written
            __syncthreads();
        }
        // ---- write
        char* const pool_to = a.geom.pool;
        if (weights) {
            for (int t = tid, i = 0; t < kTokens; t += kKeepThreads, ++i)
                if (s_from[t] != kNone) reinterpret_cast<uint32_t*>(a.weights)[s_to[t / 16] + (uint64_t)(t & 15)] = scale[i];
        } else {
            if (keys) {
#pragma unroll
                for (int i = 0; i < kKOwn; ++i) {
                    const int p = tid + kKeepThreads * i, t = p % kTokens;
                    if (p >= kKItems || s_from[t] == kNone) continue;
                    *reinterpret_cast<u32x4*>(pool_to + s_to[t / 16] + ((group * S::kPieces + p / kTokens) * 16 + place_of_token(t & 15)) * 16) = x[i];
                }
            }
            if (values) {
#pragma unroll
                for (int i = 0; i < kVOwn; ++i) {
                    const int p = tid + kKeepThreads * i, e = p % S::kElems, octet = p / S::kElems;
                    const u32x4 v = x[kFirstV + i];
                    if (p >= kVItems) continue;
                    uint32_t moves = 0;
#pragma unroll
                    for (int t = 0; t < 8; ++t) moves |= (s_from[8 * octet + t] != kNone ? 1u : 0u) << t;
                    if (moves == 0u) continue;
                    char* const at = pool_to + s_to[octet / 2] + kAt.v + ((octet & 1) * (S::kGroups * S::kElems) + group * S::kElems + e) * (8 * S::kElem);
                    if (moves == 0xFFu) {
                        if constexpr (S::kElem == 2) *reinterpret_cast<u32x4*>(at) = v;
                        else *reinterpret_cast<u32x2*>(at) = (u32x2){v.x, v.y};
                        continue;
                    }
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        if ((moves >> t & 1u) == 0u) continue;
                        if constexpr (S::kElem == 2) reinterpret_cast<uint16_t*>(at)[t] = (uint16_t)(v[t / 2] >> (16 * (t & 1)));
                        else reinterpret_cast<uint8_t*>(at)[t] = (uint8_t)(v[t / 4] >> (8 * (t & 3)));
                    }
                }
            }
            if constexpr (kStore != SALI_STORE_16)
#pragma unroll
                for (int side = 0; side < kSides; ++side)
                    for (int t = tid, i = side * kOwn; t < kTokens; t += kKeepThreads, ++i) {
                        if (s_from[t] == kNone) continue;
                        char* const block = pool_to + s_to[t / 16];
                        const bool v = kBoth ? side == 1 : values;
                        const uint32_t at = (uint32_t)(group * 16 + (v ? t & 15 : place_of_token(t & 15)));
                        *reinterpret_cast<uint32_t*>(block + (v ? kAt.vs : kAt.ks) + at * 4) = scale[i];
                        if constexpr (kStore == SALI_STORE_INT4) *reinterpret_cast<uint16_t*>(block + (v ? kAt.vz : kAt.kz) + at * 2) = low[i];
                    }
        }
        if constexpr (!kInPlace) return;
        __syncthreads();                                    // s_from and s_to have been read
    }
}

}  // namespace

hipError_t launch_pages_select(const PagesSelect& a, hipStream_t s) {
    hipLaunchKernelGGL(k_pages_select, dim3((unsigned)(a.seqs.n_seqs * a.geom.n_kv)), dim3(kSelectThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_keep(int store, int dim, const PagesKeep& a, hipStream_t s) {
    const int chunks = (int)keep_chunks(a.seqs, a.width, a.in_place != 0);
    const int strips = a.in_place ? keep_strips(dim, a.weights != nullptr) : dim / 32 + (a.weights != nullptr ? 1 : 0);
    const dim3 grid((unsigned)(a.seqs.n_seqs * (int64_t)chunks * a.geom.n_kv * strips));
    auto go = [&](auto st, auto d) {
        auto launch = [&](auto in_place, auto tokens) {
            hipLaunchKernelGGL((k_pages_keep<decltype(st)::value, decltype(d)::value, decltype(in_place)::value, decltype(tokens)::value>), grid, dim3(kKeepThreads), 0, s, a, chunks);
        };
        // in place a chunk waits for the one before: large ones, where there are several (drafts of 16 tokens: 8.7 us with chunks of 64, 14.9 with 256)
        if (!a.in_place) launch(std::false_type{}, std::integral_constant<int, kKeepTokens>{});
        else if (std::min(a.width, a.seqs.max_q) + kBlockTokens - 1 <= kKeepTokens) launch(std::true_type{}, std::integral_constant<int, kKeepTokens>{});
        else launch(std::true_type{}, std::integral_constant<int, 256>{});
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
