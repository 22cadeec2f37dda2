// tcgen05 helpers for e4m3 operands (kind::f8f6f4): a tile row of 128 bytes
// holds 128 elements, one instruction covers K = 32, so that the shared-memory
// descriptors of the 16-bit kernels serve as they are (32 bytes of K a step;
// an N-major operand's atoms are 128 elements of N x 8 of K).
#pragma once

#include "pp_tc_attn.cuh"

namespace pp {

// D fp32, A and B e4m3, M = 128, N a multiple of 16 up to 256; B "N-major" or not.
PP_DEVINL uint32_t idesc_f8_m128(int n, bool b_n_major) {
    return (1u << 4) | ((b_n_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

PP_DEVINL void umma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// A in TMEM: lane = row, four e4m3 a column.
PP_DEVINL void umma_f8_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Warp-collective: lane i writes 8 consecutive columns of row (lane base + i).
PP_DEVINL void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

}  // namespace pp
