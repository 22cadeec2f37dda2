// Vectors of a head's elements, and the angle of a rotated pair: shared by the
// kernels that move heads (rotation, norms, append).
#pragma once

#include "pp_common.cuh"

namespace pp {

// ------------------------------------------------------------------ access
// V consecutive elements of type T in one load or store.
template <int BYTES>
struct Raw;
template <>
struct Raw<16> {
    using type = uint4;
};
template <>
struct Raw<8> {
    using type = uint2;
};
template <>
struct Raw<4> {
    using type = unsigned;
};

template <typename T, int V>
struct Vec {
    typename Raw<sizeof(T) * V>::type raw;
    // read and written once: first to leave L2 (4 % of a prompt's time)
    PP_DEVINL void load(const char* p) { raw = __ldcs(reinterpret_cast<const decltype(raw)*>(p)); }
    PP_DEVINL void store(char* p) const { __stcs(reinterpret_cast<decltype(raw)*>(p), raw); }
    PP_DEVINL float get(int i) const {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&raw)[sizeof(T) == 4 ? i : i / 2];
        if (sizeof(T) == 4) return __uint_as_float(w);
        return i & 1 ? bf16hi(w) : bf16lo(w);
    }
    PP_DEVINL void set2(int i, float a, float b) {  // elements i (even) and i + 1
        uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
        if (sizeof(T) == 4) {
            w[i] = __float_as_uint(a);
            w[i + 1] = __float_as_uint(b);
        } else {
            w[i / 2] = Elem<__nv_bfloat16>::pair(a, b);
        }
    }
};

// cp.async of 4, 8 or 16 bytes.
template <int BYTES>
PP_DEVINL void cp_async_small(void* dst, const void* src) {
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(BYTES) : "memory");
}

// cos and sin of pos * f (f in radians) at any 32-bit position: the frequency
// is taken in units of 2^-64 turn, where the product with the position wraps
// at whole turns by itself, so that the angle is rounded only once, when the
// rest becomes a float.  1 / 2 pi to 64 bits leaves at most 2^-30 turn at the
// largest position (for f up to 1).
PP_DEVINL float2 cos_sin(int pos, float f) {
    constexpr unsigned long long kInv2Pi = 2935890503282001226ull;  // 2^64 / 2 pi
    const unsigned bits = __float_as_uint(f), ex = bits >> 23 & 0xffu;
    const unsigned long long m = (bits & 0x7fffffu) | (ex ? 0x800000u : 0u);
    const int shift = 150 - (int)(ex ? ex : 1u);  // |f| = m 2^-shift
    const unsigned long long hi = __umul64hi(m, kInv2Pi), lo = m * kInv2Pi;
    unsigned long long turn = shift >= 64 ? hi >> min(shift - 64, 63)
                              : shift > 0 ? hi << (64 - shift) | lo >> shift
                                          : lo << min(-shift, 63);
    if (bits >> 31) turn = 0ull - turn;
    turn *= (unsigned long long)(long long)pos;
    const float half = (float)(int)(turn >> 32) * 0x1p-31f;  // the angle in units of pi, -1 to 1
    float s, c;
    sincospif(half, &s, &c);
    return make_float2(c, s);
}

}  // namespace pp
