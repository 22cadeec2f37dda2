// tcgen05 helpers of the attention kernel beyond pp_tc.cuh: an A operand in
// TMEM, a B operand whose N runs along the contiguous dimension (values as
// they lie in the cache: [token][element]), and TMEM stores.
#pragma once

#include "pp_tc.cuh"

namespace pp {

// Instruction descriptor with B "N-major" (bit 16).
PP_DEVINL constexpr uint32_t idesc_bf16_m128_bn(int n) { return idesc_bf16_m128(n) | (1u << 16); }

// Shared-memory descriptor of an N-major operand with the 128-byte swizzle:
// atoms of 64 elements of N (128 B) x 8 of K (128 B apart); the next 8 of K
// lie 1024 B further, the next 64 of N `group_bytes` further.
PP_DEVINL uint64_t sdesc_sw128_n(const void* p, uint32_t group_bytes) {
    const uint32_t a = smem_u32(p);
    uint64_t d = (uint64_t)((a & 0x3ffffu) >> 4);
    d |= (uint64_t)(group_bytes >> 4) << 16;  // leading byte offset: next 64 of N
    d |= (uint64_t)(1024u >> 4) << 32;        // stride byte offset: next 8 of K
    d |= (uint64_t)1u << 46;                  // descriptor version
    d |= (uint64_t)2u << 61;                  // 128-byte swizzle
    return d;
}

// D[128 x N] (+)= A[128 x 16] * B, A in TMEM: lane = row, two bf16 a column.
PP_DEVINL void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Warp-collective: lane i writes 16 consecutive columns of row (lane base + i).
PP_DEVINL void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
PP_DEVINL void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 4-D tiled tensor copy global -> shared; boxes past an extent read zeros.
PP_DEVINL void tma_load_4d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, "
        "{%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}

// The same in three dimensions.
PP_DEVINL void tma_load_3d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, "
        "{%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}

// Fetch a tensor map ahead of its first use.
PP_DEVINL void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// Wait for a barrier's phase, for at most limit_ns; false when it gave up.  On
// expiry PP_ERR_TIMEOUT is recorded, over an earlier code: the call's results
// are lost.  Waits that have lasted over 1 ms give up once that is recorded,
// and only then: a bad page or length recorded by this call or an earlier one
// leaves the other sequences to be computed, and a wait of several ms is
// regular (the rows of q wait for a whole item: 1 ms at 64 thousand entries).
// The first wait of a CTA that gives up sets *lost (shared memory), and the
// CTA's other waits give up after one try each.
struct Waits {
    unsigned* status;
    uint64_t limit_ns;
    volatile unsigned* lost;
};
static __device__ __noinline__ bool attn_wait_slow(uint64_t* bar, uint32_t parity, Waits w) {
    const uint64_t t0 = globaltimer_ns();
    while (!mbar_try_wait(bar, parity)) {
        if (*w.lost) return false;
        const uint64_t dt = globaltimer_ns() - t0;
        const bool expired = dt > w.limit_ns;
        if (expired) atomicExch(w.status, (unsigned)PP_ERR_TIMEOUT);
        if (expired || (dt > 1000000ull && *reinterpret_cast<volatile unsigned*>(w.status) == PP_ERR_TIMEOUT)) {
            *w.lost = 1u;
            return false;
        }
    }
    return true;
}
PP_DEVINL bool attn_wait(uint64_t* bar, uint32_t parity, const Waits& w) {
    return mbar_try_wait(bar, parity) || attn_wait_slow(bar, parity, w);
}

// Barrier over n threads of whole warps; true for all where any brings true.
PP_DEVINL bool named_bar_or(int id, int n, bool any) {
    unsigned r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %1, 0;\n\t"
        "bar.red.or.pred p, %2, %3, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(any ? 1u : 0u), "r"(id), "r"(n)
        : "memory");
    return r != 0u;
}

// 2^x, flushing subnormals (softmax weights below 2^-126 count as zero).
PP_DEVINL float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 operations an instruction.
PP_DEVINL unsigned long long pair2(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
PP_DEVINL void unpair2(unsigned long long v, float& a, float& b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
PP_DEVINL unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
PP_DEVINL unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
PP_DEVINL float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

}  // namespace pp
