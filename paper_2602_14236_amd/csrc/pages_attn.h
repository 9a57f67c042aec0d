// Causal attention of new tokens over paged K/V (gfx950): what the kernels share.  The layout of a block of 16 tokens stands in sali.h.
//
// Rows.  For one sequence and K/V head the queries are rows r = token * group + head in group, so the heads of a group share every key that is
// read, and a call of one token a sequence has group rows.  Keys are taken 32 at a time (two blocks).  The scores are computed transposed,
// S^T = K Q^T: the matrix cores then leave a query's scores of 4 or 8 consecutive tokens in one lane, which is the operand that the second product,
// out^T = V^T P^T, wants, so weights never leave their lane's registers.  K's places and V's pairs of 8 tokens are laid
// out in memory as those operands: every load is 16 bytes a lane of contiguous memory, ready for use.
//
// Softmax.  Scores are kept in units of log 2 (scale2 = scale * log2 e).  Each row has a reference m and a sum of
// exp2(s - m).  The reference is set kRaise below the row's maximum and follows it only when that has grown by more than kLag, so the weights of
// 16 bits reach from 2^kRaise to 2^(kRaise + kLag) and nothing has to be rescaled most of the time.  fp16 has nothing below 2^-24: with weights at 1
// and below, many weak keys under a strong one (a first token that takes most of the weight) lost their bits or vanished, 20 % of the result at a distance of
// 17; from 2^10 on that happens 2^34 below the strongest.  bfloat16 has the exponents of fp32, as its values have: weights are lowered there, to about
// what a text's normalised weights are, so that 2^24 equal ones of the largest values have a sum (2^16 that lie kLag above the reference).
// Values down to 2^-112 give the results of larger ones but for single last places.  Nothing seen: m = -inf, sum 0.
//
// Masked keys.  Scores outside a row's view become -inf, whatever they were, and their weights 0.  A weight of 0 does not take
// out an infinity or NaN in V.  What no token has written (past a sequence's end, pages that are none) is set to zero before the product, by
// position; quantised values are finite wherever they were written.  16-bit rows are looked at, in the stream always: values that are not finite are set to zero for the product, two more products count, for
// every output, the infinities of each sign in its view (a NaN counts for both), and what was found is added to the result at the end.  Tiles look at keys that
// not all of their rows see; where all do, the product shows what is there, an infinity, or a NaN where its weight was rounded to zero, and a
// piece of work with a NaN in its results is done again with a look at all keys.
#pragma once

#include <type_traits>

#include "pages.h"

namespace sali {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));

constexpr float kLn2 = 0.69314718055994530942f;

// the 16-bit types and their matrix products
template <bool kBf16>
struct Num;
template <>
struct Num<false> {
    typedef _Float16 T;
    typedef half8 V8;
    static constexpr uint32_t kExp = 0x7C007C00u, kExpOne = 0x04000400u;
    static constexpr uint16_t kOne = 0x3C00u;
    static constexpr float kRaise = 10.0f, kLag = 5.0f;         // weights up to 2^15
    static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
};
template <>
struct Num<true> {
    typedef __bf16 T;
    typedef bhalf8 V8;
    static constexpr uint32_t kExp = 0x7F807F80u, kExpOne = 0x00800080u;
    static constexpr uint16_t kOne = 0x3F80u;
    static constexpr float kRaise = -24.0f, kLag = 8.0f;         // and down to 2^-126
    static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
};

// two fp32 numbers as a pair of 16-bit ones, rounded to nearest
template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef typename Num<kBf16>::T T;
    typedef T T2 __attribute__((ext_vector_type(2)));
    const T2 v = {(T)a, (T)b};
    return __builtin_bit_cast(uint32_t, v);
}
// the same where a and b are products or sums: those are rounded to fp32 first
template <bool kBf16>
__device__ __forceinline__ uint32_t pack2_after_f32(float a, float b) {
    asm("" : "+v"(a), "+v"(b));
    return pack2<kBf16>(a, b);
}
template <bool kBf16>
__device__ __forceinline__ float low_half(uint32_t w) {
    return (float)__builtin_bit_cast(typename Num<kBf16>::T, (uint16_t)w);
}
template <bool kBf16>
__device__ __forceinline__ float high_half(uint32_t w) {
    return (float)__builtin_bit_cast(typename Num<kBf16>::T, (uint16_t)(w >> 16));
}

// eight 8-bit codes, signed, times one scale or each times its own
__device__ __forceinline__ float code8(uint32_t w, int i) { return (float)(int)(int8_t)(w >> (8 * i) & 0xFFu); }
// eight 4-bit codes, in the low halves of the bytes of two words (already masked)
__device__ __forceinline__ float code4(uint32_t w, int i) { return (float)(w >> (8 * i) & 0xFFu); }

// 8 codes of one token (K)
template <bool kBf16>
__device__ __forceinline__ u32x4 values8(uint32_t a, uint32_t b, float scale) {
    u32x4 r;
    r.x = pack2_after_f32<kBf16>(code8(a, 0) * scale, code8(a, 1) * scale);
    r.y = pack2_after_f32<kBf16>(code8(a, 2) * scale, code8(a, 3) * scale);
    r.z = pack2_after_f32<kBf16>(code8(b, 0) * scale, code8(b, 1) * scale);
    r.w = pack2_after_f32<kBf16>(code8(b, 2) * scale, code8(b, 3) * scale);
    return r;
}
template <bool kBf16>
__device__ __forceinline__ u32x4 values4(uint32_t a, uint32_t b, float scale, float low) {
    u32x4 r;
    r.x = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 0), scale, low), __builtin_fmaf(code4(a, 1), scale, low));
    r.y = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 2), scale, low), __builtin_fmaf(code4(a, 3), scale, low));
    r.z = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 0), scale, low), __builtin_fmaf(code4(b, 1), scale, low));
    r.w = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 2), scale, low), __builtin_fmaf(code4(b, 3), scale, low));
    return r;
}
// 8 tokens' codes of one value (V).  The 16 lanes of a row take values of one group, so lane i of them brings the scale (and smallest value) of token
// i % 8 and the others take it from there, as an operand.
template <int kLane>
__device__ __forceinline__ float from_row(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x150 + kLane, 0xF, 0xF, true));        // row_newbcast
}
template <bool kBf16>
__device__ __forceinline__ u32x4 row_values8(uint32_t a, uint32_t b, float s) {
    asm("" : "+v"(s));         // used once a lane each, so that it is an operand and not a move
    u32x4 r;
    r.x = pack2_after_f32<kBf16>(code8(a, 0) * from_row<0>(s), code8(a, 1) * from_row<1>(s));
    r.y = pack2_after_f32<kBf16>(code8(a, 2) * from_row<2>(s), code8(a, 3) * from_row<3>(s));
    r.z = pack2_after_f32<kBf16>(code8(b, 0) * from_row<4>(s), code8(b, 1) * from_row<5>(s));
    r.w = pack2_after_f32<kBf16>(code8(b, 2) * from_row<6>(s), code8(b, 3) * from_row<7>(s));
    return r;
}
// (moves here, since a multiply-add takes no such operand; the two halves of a group's bytes share them)
template <bool kBf16>
__device__ __forceinline__ u32x4 row_values4(uint32_t a, uint32_t b, float s, float z) {
    u32x4 r;
    r.x = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 0), from_row<0>(s), from_row<0>(z)), __builtin_fmaf(code4(a, 1), from_row<1>(s), from_row<1>(z)));
    r.y = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 2), from_row<2>(s), from_row<2>(z)), __builtin_fmaf(code4(a, 3), from_row<3>(s), from_row<3>(z)));
    r.z = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 0), from_row<4>(s), from_row<4>(z)), __builtin_fmaf(code4(b, 1), from_row<5>(s), from_row<5>(z)));
    r.w = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 2), from_row<6>(s), from_row<6>(z)), __builtin_fmaf(code4(b, 3), from_row<7>(s), from_row<7>(z)));
    return r;
}
// the same where a lane has all of them
struct Scales8 {
    f32x4 a, b;
};
template <bool kBf16>
__device__ __forceinline__ u32x4 values4(uint32_t a, uint32_t b, const Scales8& s, const u32x4& z) {
    u32x4 r;
    const uint32_t z0 = z.x, z1 = z.y, z2 = z.z, z3 = z.w;
    r.x = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 0), s.a[0], low_half<kBf16>(z0)), __builtin_fmaf(code4(a, 1), s.a[1], high_half<kBf16>(z0)));
    r.y = pack2_after_f32<kBf16>(__builtin_fmaf(code4(a, 2), s.a[2], low_half<kBf16>(z1)), __builtin_fmaf(code4(a, 3), s.a[3], high_half<kBf16>(z1)));
    r.z = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 0), s.b[0], low_half<kBf16>(z2)), __builtin_fmaf(code4(b, 1), s.b[1], high_half<kBf16>(z2)));
    r.w = pack2_after_f32<kBf16>(__builtin_fmaf(code4(b, 2), s.b[2], low_half<kBf16>(z3)), __builtin_fmaf(code4(b, 3), s.b[3], high_half<kBf16>(z3)));
    return r;
}

__device__ __forceinline__ u32x4 load16(const void* p) { return *static_cast<const u32x4*>(p); }

// lanes 32 and 16 apart
__device__ __forceinline__ float max_over_halves(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_over_halves(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float max_over_quarters(float v) {
    v = max_over_halves(v);
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_over_quarters(float v) {
    v = sum_over_halves(v);
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// the reference that a row's largest score asks for
template <bool kBf16>
__device__ __forceinline__ float reference_of(float top, float scale2) {
    top *= scale2;
    asm("" : "+v"(top));                    // not one instruction, for which the constant would stay in a vector register
    return top - Num<kBf16>::kRaise;
}

// V's values of 8 tokens: those that are finite, and 1 where an infinity of either sign (or a NaN) stands
template <bool kBf16>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {        // bits 15 and 31
    return ((w & 0x7FFF7FFFu) + Num<kBf16>::kExpOne) & 0x80008000u;
}
template <bool kBf16>
__device__ __forceinline__ bool any_not_finite(const u32x4& v) {
    return (not_finite<kBf16>(v.x) | not_finite<kBf16>(v.y) | not_finite<kBf16>(v.z) | not_finite<kBf16>(v.w)) != 0;
}
// the words of a piece of 8 tokens with those from `live` on set to zero
__device__ __forceinline__ u32x4 live_tokens(const u32x4& v, int live) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (2 * i < live ? v[i] & 0xFFFFu : 0u) | (2 * i + 1 < live ? v[i] & 0xFFFF0000u : 0u);
    return r;
}
__device__ __forceinline__ Scales8 live_tokens(const Scales8& s, int live) {
    Scales8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.a[i] = i < live ? s.a[i] : 0.0f;
        r.b[i] = i + 4 < live ? s.b[i] : 0.0f;
    }
    return r;
}
template <bool kBf16>
__device__ __forceinline__ void take_apart(const u32x4 v, u32x4& finite, u32x4& plus, u32x4& minus) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = v[i], bad = not_finite<kBf16>(w), mask = (bad >> 15) * 0xFFFFu;
        // a NaN has bits below the exponent
        const uint32_t below = w & ~(Num<kBf16>::kExp | 0x80008000u);
        const uint32_t nan = ((below & 0xFFFFu) != 0 ? 0xFFFFu : 0u) | (below >> 16 != 0 ? 0xFFFF0000u : 0u);
        const uint32_t neg = (w >> 15 & 0x00010001u) * 0xFFFFu, one = Num<kBf16>::kOne | (uint32_t)Num<kBf16>::kOne << 16;
        finite[i] = w & ~mask;
        plus[i] = mask & (nan | ~neg) & one;
        minus[i] = mask & (nan | neg) & one;
    }
}

// A factor that joins results, of what sees something: the smallest number where fp32 has none that is small enough, so that an infinity stays one.
__device__ __forceinline__ float not_zero(float by) { return fmaxf(by, 1.4e-45f); }

// A row's result from its sum (out and lse still apart): joined with the prior and rounded.  `out` is one value of the unnormalised sum.
struct RowEnd {
    float lse, by_own, by_prior;            // out = out * by_own + prior * by_prior
};
__device__ __forceinline__ RowEnd row_end(float m, float l, const PagesAttend& a, int64_t row) {
    RowEnd r = {-INFINITY, 0.0f, 0.0f};
    const bool some = l > 0.0f || l != l;   // a NaN stays one
    float lse = some ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;      // log2
    float own = some ? 1.0f / l : 0.0f;
    if (a.prior == nullptr) {
        r.lse = lse;
        r.by_own = own;
        return r;
    }
    const float lp = a.prior_lse[row], top = fmaxf(lse, lp);
    if (top == -INFINITY && lse == lse && lp == lp) return r;
    const float w1 = expf(lse - top), w2 = expf(lp - top), sum = w1 + w2;
    r.lse = top + logf(sum);
    r.by_own = some ? not_zero(own * (w1 / sum)) : 0.0f;
    r.by_prior = w2 / sum;
    return r;
}
// what values that are not finite add to a result
__device__ __forceinline__ float found(bool up, bool down) { return (up ? INFINITY : 0.0f) + (down ? -INFINITY : 0.0f); }
// a weight of zero takes out whatever the other factor is: what sees nothing
__device__ __forceinline__ float joined(const RowEnd& e, float own, float prior) {
    const float a = e.by_own == 0.0f ? 0.0f : own * e.by_own;
    return e.by_prior == 0.0f ? a : __builtin_fmaf(prior, e.by_prior, a);
}

// The kernel's struct argument once more, which lies kAt bytes into its arguments: what is only needed in one place is not to take registers elsewhere
template <int kAt>
__device__ __forceinline__ PagesAttend late_arguments() {
#ifdef __HIP_DEVICE_COMPILE__
    typedef const __attribute__((address_space(4))) char* Constant;
    Constant p = (Constant)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const __attribute__((address_space(4))) PagesAttend*)(p + kAt);
#else
    return {};                              // the host's pass over this file
#endif
}

}  // namespace

}  // namespace sali
