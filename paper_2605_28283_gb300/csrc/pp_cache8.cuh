// The cache in 8 bits: e4m3 codes and their scales.
//
// Why powers of two: a block's scale may grow with a later entry, and its
// codes are then rounded again.  At a power of two that moves exponents only
// (nothing is lost but what falls below 2^-9 of the new scale), where scales of
// amax / 448 would round every code again at each step; e4m3 has the same four
// significant bits at any magnitude, so the factor of up to two costs no
// precision.  And code * scale is exact in bf16.
#pragma once

#include "pp_batch.cuh"

namespace pp {

constexpr float kTopCode = 448.0f;
constexpr int kLeastExponent = -60;

// Two codes of fp32 values, the first in the low byte: to nearest, ties to
// even; 448 at most.
PP_DEVINL uint32_t to_codes(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
// Values of the two codes in the low 16 bits (exact).
PP_DEVINL float2 from_codes(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// The value as it is to be held: what is not finite becomes NaN.
PP_DEVINL float to_hold(float x) { return isfinite(x) ? x : __uint_as_float(0x7fffffffu); }
// Its part in a block's largest magnitude.
PP_DEVINL float magnitude(float x) { return isfinite(x) ? fabsf(x) : 0.f; }

// The smallest power of two s >= 2^-60 with 448 s >= amax (finite, >= 0):
// 448 = 1.75 * 2^8.
PP_DEVINL float scale_for(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return __uint_as_float((uint32_t)(max(e, kLeastExponent) + 127) << 23);
}

// The largest code whose value at this scale is a finite number: 448 below
// scales of 2^119, 240 at 2^120, where 256 would be 2^128.
constexpr float kLargeScale = 0x1p119f;
PP_DEVINL float top_code(float scale) {
    if (scale < kLargeScale) return kTopCode;
    // the quotient rounded down, to the four significant bits of a code
    return fminf(__uint_as_float(__float_as_uint(__fdiv_rd(3.402823466e38f, scale)) & 0xfff00000u), kTopCode);
}
// x within [-top, top] (NaN stays).
PP_DEVINL float within(float x, float top) { return fabsf(x) > top ? copysignf(top, x) : x; }

// Scale of a block whose entries to be written reach amax; `old` is that of
// entries that stay (`stays`).
PP_DEVINL float block_scale(float amax, float old, bool stays) {
    return stays && !(amax > kTopCode * old) ? old : scale_for(amax);
}

PP_DEVINL long long scale_index(const BatchArgs& B, const ScaleArgs& S, int n_kv_heads, int page, int h, int entry) {
    const unsigned off = (unsigned)entry % (unsigned)B.page_size;
    return ((long long)page * n_kv_heads + h) * S.blocks + (off >> S.shift);
}

}  // namespace pp
