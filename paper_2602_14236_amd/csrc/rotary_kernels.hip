// Rotary positions: queries and keys of new tokens turned by the angles that their positions on one to four axes give (gfx950).
//
// Pair i of a row (its values i and i + pairs, or 2 i and 2 i + 1) turns by a = position[axis of i] * frequency[i]:
//     y1 = x1 cos a - x2 sin a,    y2 = x2 cos a + x1 sin a,
// in fp32, rounded once to the 16-bit type.  Angles in 64 bits, since 32 lose a radian's sixth place from position 10 on: turns = a / 2 pi, less the nearest whole number,
// and sine and cosine of what is left in fp32.
//
// Every row is read and written once, which is what bounds long calls; a block has one token (or part of its heads, where there are few tokens), whose angles it
// works out once for all heads, in LDS, while its first rows are on their way.  20002 tokens, 40 and 40 heads of 128, 820 MB: 147 us, 5.6 TB/s (a plain copy of 2 GiB:
// 4.8 by the library, 6.5 by the best kernel); 4608 tokens, 32 and 32 heads, 151 MB, out of the caches: 23.7 us; a step of 32 tokens 3.3 us, a launch's chain of trips, of 14.5
// that the call takes the host.  Slower: heads of long calls over several blocks, one piece a thread (157 to 165 us: the angles again in each), all pieces of a thread on
// their way together (151 us, and 69 for 62 in rows of 40 heads).
//
// Pairs half a row apart whose number is no multiple of eight go value by value, two bytes an access, what does not turn too: 12 pairs in the first of these calls 671 us.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace sali {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRotaryThreads = 256, kMostRotaryThreads = 512;
// Bytes of rows, half of what the last cache holds, from which on they go past the caches: longer ones would only push each other out.  With the append of the keys
// and a reader of the queries behind it, 138 MB take 109 us past them and 115 through them, 410 MB 327 and 326; alone 410 MB take 147 and 159.  Shorter ones are still there
// for what reads them: 92 MB 71 us, outputs past the caches 74.
constexpr int64_t kPastCaches = 128 << 20;

template <bool kBf16>
struct Row16;
template <>
struct Row16<false> {
    typedef _Float16 T;
};
template <>
struct Row16<true> {
    typedef __bf16 T;
};
template <bool kBf16>
union Eight {
    u32x4 u;
    typename Row16<kBf16>::T h[8];
};

// two values of a pair; `by`: cosine and sine
template <bool kBf16>
__device__ __forceinline__ void turn(typename Row16<kBf16>::T& a, typename Row16<kBf16>::T& b, float2 by) {
    const float x = (float)a, y = (float)b;
    a = (typename Row16<kBf16>::T)(x * by.x - y * by.y);
    b = (typename Row16<kBf16>::T)(y * by.x + x * by.y);
}

// kAdjacent: pairs 2 i, 2 i + 1.  kPieces: else, pairs come in whole pieces of eight values (pairs a multiple of 8), two pieces at a time; otherwise value by value.
// kOnce: see kPastCaches
template <bool kBf16, bool kAdjacent, bool kPieces, bool kOnce>
__global__ __launch_bounds__(kMostRotaryThreads) void k_rotate(Rotate r) {
    typedef typename Row16<kBf16>::T T;
    __shared__ float2 s_turn[64];
    const int threads = (int)blockDim.x;
    const int token = blockIdx.x;
    // what a thread does for a head: two pieces that turn together, one piece (adjacent; what does not turn), or one pair, or one value that does not turn
    const int turning = kAdjacent ? r.dim / 8 : (kPieces ? r.pairs / 8 : r.pairs);
    const int still = kAdjacent ? 0 : (kPieces ? (r.dim - 2 * r.pairs) / 8 : r.dim - 2 * r.pairs);
    const int of_head = turning + still, total = (r.q_heads + r.k_heads) * of_head;
    const int each = (total + (int)gridDim.y - 1) / (int)gridDim.y, end = min(total, each * ((int)blockIdx.y + 1));
    int item = each * (int)blockIdx.y + (int)threadIdx.x;
    struct Place {
        const char* from;
        char* to;
        int at;                             // of the head's items
    };
    auto place = [&](int item) -> Place {
        const int head = item / of_head, at = item - head * of_head;
        if (head < r.q_heads)
            return {r.q.d + (int64_t)token * r.q.token_bytes + (int64_t)head * r.q.head_bytes, r.q_out.d + (int64_t)token * r.q_out.token_bytes + (int64_t)head * r.q_out.head_bytes, at};
        const int h = head - r.q_heads;
        return {r.k.d + (int64_t)token * r.k.token_bytes + (int64_t)h * r.k.head_bytes, r.k_out.d + (int64_t)token * r.k_out.token_bytes + (int64_t)h * r.k_out.head_bytes, at};
    };
    auto get = [](const char* from) -> u32x4 {
        if constexpr (kOnce) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from));
        else return *reinterpret_cast<const u32x4*>(from);
    };
    auto put = [](char* to, u32x4 v) {
        if constexpr (kOnce) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
        else *reinterpret_cast<u32x4*>(to) = v;
    };
    constexpr int kFlight = kPieces ? 2 : 1;        // items of a thread on their way together
    Eight<kBf16> a[kFlight], b[kFlight];
    Place p[kFlight];
    auto ask = [&](int first) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (first + threads * i >= end) continue;
            p[i] = place(first + threads * i);
            if constexpr (kAdjacent) {
                a[i].u = get(p[i].from + 16 * p[i].at);
            } else if constexpr (kPieces) {
                const bool turns = p[i].at < turning;
                a[i].u = get(p[i].from + 16 * (turns ? p[i].at : p[i].at + turning));
                if (turns) b[i].u = get(p[i].from + 16 * (p[i].at + turning));
            } else {
                const bool turns = p[i].at < turning;
                a[i].h[0] = *reinterpret_cast<const T*>(p[i].from + 2 * (turns ? p[i].at : p[i].at + turning));
                if (turns) b[i].h[0] = *reinterpret_cast<const T*>(p[i].from + 2 * (p[i].at + turning));
            }
        }
    };
    ask(item);
    if ((int)threadIdx.x < r.pairs) {
        const int i = threadIdx.x;
        int axis = 0;
#pragma unroll
        for (int x = 0; x < 3; ++x) axis += i >= r.until[x] ? 1 : 0;
        const double turns = (double)r.position[(int64_t)axis * r.axis_stride + token] * r.frequency[i] * 0.15915494309189533577;
        const float left = (float)(turns - rint(turns));
        float sine, cosine;
        sincospif(2.0f * left, &sine, &cosine);
        s_turn[i] = make_float2(cosine, r.inverse ? -sine : sine);
    }
    __syncthreads();
    for (; item < end; item += kFlight * threads) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (item + threads * i >= end) continue;
            const int at = p[i].at;
            if constexpr (kAdjacent) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (4 * at + e < r.pairs) turn<kBf16>(a[i].h[2 * e], a[i].h[2 * e + 1], s_turn[4 * at + e]);
                put(p[i].to + 16 * at, a[i].u);
            } else if constexpr (kPieces) {
                if (at < turning) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) turn<kBf16>(a[i].h[e], b[i].h[e], s_turn[8 * at + e]);
                    put(p[i].to + 16 * at, a[i].u);
                    put(p[i].to + 16 * (at + turning), b[i].u);
                } else {
                    put(p[i].to + 16 * (at + turning), a[i].u);
                }
            } else if (at < turning) {
                turn<kBf16>(a[i].h[0], b[i].h[0], s_turn[at]);
                *reinterpret_cast<T*>(p[i].to + 2 * at) = a[i].h[0];
                *reinterpret_cast<T*>(p[i].to + 2 * (at + turning)) = b[i].h[0];
            } else {
                *reinterpret_cast<T*>(p[i].to + 2 * (at + turning)) = a[i].h[0];
            }
        }
        ask(item + kFlight * threads);
    }
}

}  // namespace

hipError_t launch_rotate(int dtype, const Rotate& r, hipStream_t s) {
    const bool pieces = r.pairs % 8 == 0;
    const int total = (r.q_heads + r.k_heads) * (r.adjacent ? r.dim / 8 : (pieces ? (r.dim - r.pairs) / 8 : r.dim - r.pairs));
    // few tokens: their heads over several blocks, a thread's work each
    const int splits = r.n_tokens >= 1024 ? 1 : std::max(1, std::min((total + kRotaryThreads - 1) / kRotaryThreads, 1024 / r.n_tokens));
    const dim3 grid((unsigned)r.n_tokens, (unsigned)splits);
    // else blocks whose threads have an even number of items, as they come in twos, or one (1280 items by 320 threads: 147 us, by 256: 154)
    const int most = total / kRotaryThreads, each = most < 2 ? 1 : most & ~1;
    const int threads = splits > 1 || r.n_tokens > kMostBlocks / 2 ? kRotaryThreads : std::min(kMostRotaryThreads, ((total + each - 1) / each + 63) & ~63);
    const bool once = 2ll * r.dim * (r.q_heads + r.k_heads) * r.n_tokens >= kPastCaches;
    auto go = [&](auto bf16, auto adjacent, auto whole) {
        if (once) hipLaunchKernelGGL((k_rotate<decltype(bf16)::value, decltype(adjacent)::value, decltype(whole)::value, true>), grid, dim3((unsigned)threads), 0, s, r);
        else hipLaunchKernelGGL((k_rotate<decltype(bf16)::value, decltype(adjacent)::value, decltype(whole)::value, false>), grid, dim3((unsigned)threads), 0, s, r);
    };
    auto by_layout = [&](auto bf16) {
        if (r.adjacent) go(bf16, std::true_type{}, std::true_type{});
        else if (pieces) go(bf16, std::false_type{}, std::true_type{});
        else go(bf16, std::false_type{}, std::false_type{});
    };
    if (dtype == SALI_DTYPE_BF16) by_layout(std::true_type{});
    else by_layout(std::false_type{});
    return hipGetLastError();
}

}  // namespace sali
