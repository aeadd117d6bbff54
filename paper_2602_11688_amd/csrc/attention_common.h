// Device helpers of the cache and attention kernels: number formats, matrix instructions, pages.
#pragma once
#include <hip/hip_runtime.h>

#include "attention.h"

namespace gorgo {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using short4_t = __attribute__((ext_vector_type(4))) short;
using float2_t = __attribute__((ext_vector_type(2))) float;
using float4_t = __attribute__((ext_vector_type(4))) float;
using float16_t = __attribute__((ext_vector_type(16))) float;
using uint2_t = __attribute__((ext_vector_type(2))) unsigned;
using uint4_t = __attribute__((ext_vector_type(4))) unsigned;

// The two 16-bit types: eight values are four registers, uint4_t where they are only moved.
// Weights are 2^(score - largest score + RAISE), rounded to the type for the second product.  The maximum that they are taken against is
// renewed only where a score passes it by SLACK, which makes rescaling what has been added up rare: weights end at 2^(RAISE + SLACK),
// and 32 bits lose nothing by that.  bf16 has exponents enough on either side: the 2^31 weights that a row can have at most add up to
// 2^(31 + SLACK + RAISE) = 1/2 at most, so that no sum of weights times finite values overflows.  fp16 has so few exponents that
// weights are moved to their end (2^15): down to 2^-25 of the largest they keep all their bits, and below they are rounded in steps of
// 2^-35 of it.  (A SLACK of 2 would reach two powers
// further: heads of 64 with a window of 4096 take 654 us with 8, 661 with 4, 673 with 2.)
struct Bf16 {
    static constexpr float RAISE = -40.0f, SLACK = 8.0f;
    using x8 = bf16x8;
    static constexpr unsigned EXPONENT = 0x7f80u;
    static __device__ unsigned pack(float a, float b) {          // to nearest, ties to even
        return __builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){a, b}, bf16x2));
    }
    static __device__ float16_t mfma32(x8 a, x8 b, float16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ float4_t mfma16(x8 a, x8 b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
    static constexpr float RAISE = 11.0f, SLACK = 4.0f;
    using x8 = f16x8;
    static constexpr unsigned EXPONENT = 0x7c00u;
    static __device__ unsigned pack(float a, float b) {
        return __builtin_bit_cast(unsigned, __builtin_convertvector((float2_t){a, b}, f16x2));
    }
    static __device__ float16_t mfma32(x8 a, x8 b, float16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ float4_t mfma16(x8 a, x8 b, float4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

template <class T>
__device__ typename T::x8 as_x8(uint4_t x) { return __builtin_bit_cast(typename T::x8, x); }

// Four codes of 8 bits to four bf16 values, times a power of two: exact (four significant bits, bf16's own exponents).
__device__ inline uint2_t widen(unsigned codes, float power) {
    uint2_t r;
    r.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, false));
    r.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, true));
    return r;
}
__device__ inline uint4_t widen8(unsigned lo, unsigned hi, float power) {
    const uint2_t a = widen(lo, power), b = widen(hi, power);
    return (uint4_t){a.x, a.y, b.x, b.y};
}
__device__ inline float power_of(unsigned scale_byte) { return __builtin_bit_cast(float, scale_byte << 23); }

// Column of a 4 x 16 block of 16-bit values in LDS: sixteen lanes give the addresses of its rows' quarters (lane i row i / 4,
// values 4 * (i % 4) on), lane i gets column i.
__device__ inline uint2_t column4(const char* lds) {
    return __builtin_bit_cast(
        uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(lds)));
}

// The same of an 8 x 16 block of bytes: lane i gives the address of half a row (row i / 2, bytes 8 * (i % 2) on).
__device__ inline uint2_t column8(const char* lds) {
    using int2_t = __attribute__((ext_vector_type(2))) int;
    return __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) int2_t*)(lds)));
}

// Memory that nobody writes while the kernel runs, for scalar loads at uniform indexes.
using constant_i32 = __attribute__((address_space(4))) const int32_t;
__device__ inline constant_i32* constant(const int32_t* p) { return (constant_i32*)(uintptr_t)p; }

__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float log2_(float x) { return __builtin_amdgcn_logf(x); }

// What the two halves of a wavefront hold (of lanes i and i ^ 32), and what lanes i and i ^ 16 do.
struct Two {
    float a, b;
};
__device__ inline Two halves(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];                 // (a bit cast of a vector's element takes the first one)
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ inline Two sixteens(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];                 // (a bit cast of a vector's element takes the first one)
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ inline float both_max(float x) {
    const Two t = halves(x);
    return fmaxf(t.a, t.b);
}
__device__ inline float both_sum(float x) {
    const Two t = halves(x);
    return t.a + t.b;
}
// Of what lanes i, i ^ 16, i ^ 32 and i ^ 48 hold.
__device__ inline float quarters_max(float x) {
    const Two t = sixteens(both_max(x));
    return fmaxf(t.a, t.b);
}
__device__ inline float quarters_sum(float x) {
    const Two t = sixteens(both_sum(x));
    return t.a + t.b;
}

// A running maximum before any key: finite, so that exp2(-inf - it) is 0, and no finite score lies below it.
constexpr float NO_MAX = -__FLT_MAX__;
// An exponent is one fused step, score * scale - maximum: its only rounding is the maximum's, which all weights of a row share.  From
// here on that rounding grows to powers of two that 32 bits (and 16, for the weights) do not hold, and exponents are taken as the
// difference of two rounded products instead, which is 0 for the largest.  (A branch that is seldom taken: differences everywhere would be an
// instruction more for each score.)
constexpr float FAR_OUT = 4194304.0f;
__device__ inline bool far_out(float top) { return __any(__builtin_fabsf(top) >= FAR_OUT && top != NO_MAX); }

// What a row's exponents are taken against from now on: `top` so far, and the largest of its new scores.  (Far out the steps of 32
// bits are no smaller than RAISE, and weights end at 1.)
template <class T>
__device__ float renewed(float top, float largest) { return fmaxf(top, __builtin_fabsf(largest) < FAR_OUT ? largest - T::RAISE : largest); }
// Natural logarithm of a row's sum of powers of e, from its sum of weights: without the raise that both have, near 0 no bits are lost to it.
template <class T>
__device__ float log_of_sum(float top, float sum) {
    constexpr float LOWER = T::RAISE < 0 ? (float)((uint64_t)1 << (int)-T::RAISE) : 1.0f / (float)((uint64_t)1 << (int)T::RAISE);
    return sum != 0.0f ? ((top + T::RAISE) + log2_(sum * LOWER)) * 0.6931471805599453f : -__builtin_inff();
}

__device__ inline int32_t quotient(const Divider& d, int32_t x) { return (int32_t)(((uint64_t)(uint32_t)x * d.multiplier) >> (31 + d.shift)); }

// Position of a row of the cache; page ids outside the pages hold no key.
__device__ inline int32_t page_of(const BatchArgs& b, const CacheArgs& c, int32_t s, int32_t index) {
    const int32_t id = b.table[(int64_t)s * b.columns + index];
    return (uint32_t)id < (uint32_t)c.pages ? id : -1;
}

// Tokens of a sequence; of less than none there are none, so that positions fit 32 bits whatever `lengths` holds.
__device__ inline int32_t length_of(const BatchArgs& b, int32_t s) { return max(b.lengths[s], 0); }

// New tokens of a sequence: [begin, end) of the packed rows, whatever `first` holds.
struct Span {
    int32_t begin, end;
};
__device__ inline Span span_of(const BatchArgs& b, int32_t s) {
    if (!b.first) return {min(s, b.tokens), min(s + 1, b.tokens)};
    const int32_t begin = min(max(b.first[s], 0), b.tokens);
    return {begin, min(max(b.first[s + 1], begin), b.tokens)};
}

}  // namespace gorgo
