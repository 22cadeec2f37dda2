// Attention of few rows over the 8-bit cache on the tensor cores (bf16 queries,
// e4m3 keys and values): the codes go into the products as they lie in the
// cache, so that a step is bound by reading half the bytes of a bf16 cache.
//
// The other operand of each product is wider and is split into e4m3 numbers.  A
// code has 4 significant bits.  Queries, x = p0 + p1 / 2^4: p0 the nearest code,
// p1 that of 16 times the rest, which holds a query element (8 significant bits)
// exactly down to 2^-14 of its head's largest and to 2^-21 of the largest below.
// Weights, x = p0 + p1 / 2^4 + p2 / 2^22 + p3 / 2^26: p2 and p3 are the same for
// what p0 and p1 leave of small numbers, at a second base.  (That is at most
// 2^-14, half of p1's last place, so 2^22 times it stays below 448.  What is left
// of a larger number may pass that; p2 then holds part of it.)  So a weight is
// held to 2^-8 of itself, as in bf16, or 2^-36: 2^-41 of its row's largest (times
// their value scales, below).  With p0 and p1 alone, to 2^-19 of the largest, the
// result is lost where one key takes most of a row and has small values, or lies
// in a block of large scale whose other elements are small.
//
// The 128 rows of a product are filled with the pieces: lane 8 p + i of each
// quarter holds piece p of row i's weights (i < 8), and piece p % 2 of its query;
// the quarters hold copies, each with its own 32 keys of the tile (as for few
// rows in attn_tc.cuh).  So a tile of 128 keys costs two products of 256 cycles,
// where reading it takes 1400.  The four lanes of a row share its 32 keys: lane
// 8 p + i weighs the p-th eight (of one scale's block).  They hand one another
// the parts of the scores, S = p0.k + p1.k / 16, and the codes of the weights.
//
// Scales: a key's score is S times its row's and its block's scale.  A weight is
// multiplied by its block's value scale before it is split; the running base of
// these products (b, per row and quarter) is apart from the scores' running
// maximum (m, per lane), since scales may differ widely between blocks:
// w = 2^(z - x) vs 2^(x - b) with x the tile's largest z, and the sum of weights
// is that of 2^(z - m).
//
// Warps: four softmax, four that finish parts (O has two buffers for that, up to
// 128 elements), two that issue products, one that splits the rows of q, four
// producers of the ring (TMA, a box a page; else cp.async), one that walks the
// stretch.  A quarter's weights of a tile take 8 of the 32 columns that its scores
// had, and zeros the same columns of the other quarters' keys.
//
// Measured (GB300): one token for each of 64 ragged sequences of 64 to 8191
// entries, 32 heads on 8 key heads of 128: 99 us, 5.4 TB/s (0.80 of the copy rate;
// the same call over a bf16 cache 166), 32 key heads 333 us.  Two things are close
// to one another: HBM's rows of 128 bytes, fetched without what lies beside them,
// and the softmax of a tile, which one warp a quarter does in a chain (four pieces
// of the query as well, three times as many exchanged scores: 109 and 386 us).
#include "attn_tc.cuh"
#include "pp_tc_f8.cuh"

namespace pp {
namespace {

constexpr int kFewRows = 8;         // rows of an item
// Tiles that an item counts more than it has: 0 / 2 / 4 / 8, 64 ragged single tokens 100.2 / 99.0 / 99.1 / 102.6 us.
constexpr int kPad = 2;
// Growth of the base (log2) that O absorbs unscaled: 1 / 2 / 3, 100.5 / 99.0 / 98.2 us; 3 costs small weights a bit.
constexpr float kLazy8 = 2.0f;
// The largest weight at its base, in codes: 2^kLazy8 times that, times the fraction of a scale (below 2), stays below 448.
constexpr float kTopWeight = 32.f;
constexpr int kFacTiles = 8;        // tiles whose scales are held
constexpr int kFac = 24;            // floats of a tile: 8 blocks of 16 keys each: score factor, value scale's fraction, its exponent

template <int DP>
struct Few {
    static constexpr int BN = DP == 256 ? 64 : 128, NG = DP / 128;
    static constexpr int kSlots = DP == 256 ? 6 : 8, kSlot = BN * DP;  // even: keys and values keep to slots of their own
    static constexpr int kQBufs = 2, kQTile = 128 * DP;
    static constexpr int kParts = BN / 32;      // quarters with keys of their own
    static constexpr int kOuts = DP == 256 ? 1 : 2;  // O buffers in TMEM, behind two slots of scores and weights
    static constexpr int kPitch = 128 + 4;      // floats of a staged row
    static constexpr int kStage = 4 * kFewRows * kPitch * 4;
    static constexpr int kSmem = kSlots * kSlot + kQBufs * kQTile + kStage + 1024;
    static constexpr int kWarpOut = 4, kWarpMma = 8, kWarpQ = 10, kWarpLoad = 11, kLoads = 4, kWarps = kWarpLoad + kLoads + 1;
    static constexpr int kReaders = kWarps - 1;
    static constexpr uint32_t kTmemO = 2 * BN;
    static_assert(kTmemO + kOuts * DP <= 512, "TMEM columns");
    static_assert(kFacTiles >= kSlots, "a tile's scales outlive its softmax");
};

// 32 rows of DP codes into a swizzled tile, by 16-byte cp.async (as copy_rows32).
template <int DP, int BN>
PP_DEVINL void copy_codes32(unsigned char* tile, int r0, const char* base, long long off, int D, int lane) {
    constexpr int kLanes = DP / 16, kPer = 32 / kLanes;
    const int sub = lane / kLanes, c = lane % kLanes;
#pragma unroll 2
    for (int i = 0; i < kLanes; i++) {
        const long long o = __shfl_sync(kFull, off, kPer * i + sub);
        const int r = r0 + kPer * i + sub;
        const bool in = o >= 0 && c * 16 < D;
        cp_async_16(tile + (c >> 3) * BN * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4), in ? base + o + c * 16 : base, in ? 16u : 0u);
    }
}

template <int DP, int BN>
PP_DEVINL void zero_codes(unsigned char* tile, int r0, int r1, int lane) {
#pragma unroll 1
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32)
#pragma unroll
        for (int g = 0; g < DP / 128; g++) *reinterpret_cast<uint4*>(tile + g * BN * 128 + e * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// NaN codes of rows [r0, r1) of a value tile set to zero, and the entries that
// held any noted (as finite_rows).  A byte's low 7 bits are all ones exactly if
// adding one carries into the eighth.
template <int DP, int BN>
PP_DEVINL void finite_codes(unsigned char* tile, int r0, int r1, int lane, int k0, int* odd0, int* odd1) {
    auto nan_bytes = [](uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };
    uint32_t any = 0;
#pragma unroll 2
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32)
#pragma unroll
        for (int g = 0; g < DP / 128; g++) {
            const uint4 v = *reinterpret_cast<const uint4*>(tile + g * BN * 128 + e * 16);
            any |= nan_bytes(v.x) | nan_bytes(v.y) | nan_bytes(v.z) | nan_bytes(v.w);
        }
    if (any == 0) return;
#pragma unroll 1
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32) {
        bool odd = false;
#pragma unroll 1
        for (int i = 0; i < 4 * (DP / 128); i++) {
            uint32_t* w = reinterpret_cast<uint32_t*>(tile + (i >> 2) * BN * 128 + e * 16) + (i & 3);
            const uint32_t bad = nan_bytes(*w);
            if (!bad) continue;
            *w &= ~((bad >> 7) * 255u);
            odd = true;
        }
        if (!odd) continue;
        atomicMin(odd0, k0 + (e >> 3));
        atomicMax(odd1, k0 + (e >> 3) + 1);
    }
}

// Two values in N pieces of two codes each.
template <int N>
PP_DEVINL void split2(unsigned long long x, uint32_t (&p)[N]) {
    constexpr float kUp[4] = {1.f, 0x1p4f, 0x1p22f, 0x1p26f};
    float a, b;
    unpair2(x, a, b);
    p[0] = to_codes(a, b);
#pragma unroll
    for (int i = 1; i < N; i++) {
        const float2 v = from_codes(p[i - 1]);
        x = fma2(pair2(v.x, v.y), pair2(-1.f / kUp[i - 1], -1.f / kUp[i - 1]), x);
        unpair2(mul2(x, pair2(kUp[i], kUp[i])), a, b);
        p[i] = to_codes(a, b);
    }
}
// Four values, a word a piece.
template <int N>
PP_DEVINL void split4(unsigned long long x, unsigned long long y, uint32_t (&w)[N]) {
    uint32_t a[N], b[N];
    split2(x, a);
    split2(y, b);
#pragma unroll
    for (int i = 0; i < N; i++) w[i] = a[i] | b[i] << 16;
}
// A piece's weight.
PP_DEVINL float piece_weight(int p) { return p == 0 ? 1.f : p == 1 ? 0x1p-4f : p == 2 ? 0x1p-22f : 0x1p-26f; }

template <int DP>
__global__ void __launch_bounds__(Few<DP>::kWarps * 32, 1)
    attn8_few_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using C = Few<DP>;
    constexpr int BN = C::BN, NG = C::NG, ROWS = kFewRows, NS = C::kSlots;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* ring = smem;
    unsigned char* qs = smem + NS * C::kSlot;
    float* stage = reinterpret_cast<float*>(qs + C::kQBufs * C::kQTile);
    __shared__ uint64_t full[NS], empty[NS], landed[C::kLoads], qfull[2], qempty[2], sfull[2], pfull[2], odone[2];
    __shared__ uint64_t opart[2], ofull[2], ofree[2];
    __shared__ uint32_t taddr_s;
    __shared__ float stat_m[2][4][32], stat_b[2][4][32], stat_l[2][4][32], q_scale[kItems][ROWS];
    __shared__ __align__(16) float fac[kFacTiles][kFac];
    __shared__ unsigned last_s;
    __shared__ Item<ROWS, BN> items[kItems];
    __shared__ uint64_t ifull[kItems], isplit[kItems], iempty[kItems];
    __shared__ unsigned lost_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Waits w{a.status, a.timeout_ns, &lost_s};
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < NS; i++) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < C::kLoads; i++) mbar_init(&landed[i], 1);
        for (int i = 0; i < 2; i++) {
            mbar_init(&qfull[i], 1);
            mbar_init(&qempty[i], 1);
            mbar_init(&sfull[i], 1);
            mbar_init(&pfull[i], C::kParts);
            mbar_init(&odone[i], 1);
            mbar_init(&opart[i], 1);
            mbar_init(&ofull[i], C::kParts);
            mbar_init(&ofree[i], 4);
        }
        for (int i = 0; i < kItems; i++) {
            mbar_init(&ifull[i], 1);
            mbar_init(&isplit[i], 1);
            mbar_init(&iempty[i], C::kReaders);
        }
        lost_s = 0u;
        fence_mbar_init();
    }
    if (warp == C::kWarpMma) {
        tmem_alloc(&taddr_s, 512);
        tmem_relinquish();
    }
    // rows that an item does not fill: finite
    for (int i = tid; i < C::kQBufs * C::kQTile / 16; i += C::kWarps * 32) reinterpret_cast<uint4*>(qs)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < kItems * ROWS) q_scale[tid / ROWS][tid % ROWS] = 1.f;
    fence_proxy_async_smem();
    if (tid == C::kWarpLoad * 32 && a.box) {
        prefetch_map(&map_k);
        prefetch_map(&map_v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = taddr_s;
    pdl_wait();
    // a wait that gives up ends the CTA's work in order, as in attn_tc_kernel
    ItemAt<ROWS, BN, true> at{items, ifull, iempty, w, 0, 0, 0, 0, false};
    // order of the loads: K0 K1 V0 K2 V1 K3 ... (scores run two tiles ahead)
    auto k_pos = [](int g) { return g == 0 ? 0 : 2 * g - 1; };
    auto v_pos = [](int g) { return 2 * g + 2; };

    if (warp == C::kWarps - 1) {
        // ---------------------------------------------------------- schedule
        Walk<ROWS, BN, true> walk = start_walk<ROWS, BN, true>(&a, lane, blockIdx.x == 0, 1, kPad, a.head_shift);
        if (lane == 0) {
            Part p;
            for (int n = 0;; n++) {
                const bool some = walk.next(p);
                Item<ROWS, BN>& it = items[n % kItems];
                if (n >= kItems && !attn_wait(&iempty[n % kItems], (uint32_t)(n / kItems - 1) & 1u, w)) break;
                if (!some) {  // the stretch's end: a part of no rows
                    it.rows = 0;
                    mbar_arrive(&ifull[n % kItems]);
                    break;
                }
                static_cast<Part&>(it) = p;
                it.rows = min(ROWS, p.seq.n * a.group - p.j * ROWS);
                it.open = all_see<ROWS>(a, p);
                it.odd0 = 0x7fffffff;
                it.odd1 = 0;
                mbar_arrive(&ifull[n % kItems]);
                if (!p.whole()) it.split = Split<ROWS, BN>(walk.sched, p);
                mbar_arrive(&isplit[n % kItems]);
            }
        }
        __syncwarp();
    } else if (warp >= C::kWarpLoad) {
        // ----------------------------------- producer of every fourth load
        const int me = warp - C::kWarpLoad;
        at.enter(0);
        int g_at = 0, fixes = 0, page = 0;
        // tile of load pos; page of the lane's 16 keys of it (lanes 8 apart hold the same)
        auto tile_of = [](int pos) { return pos == 0 ? 0 : pos & 1 ? (pos + 1) / 2 : (pos - 2) / 2; };
        auto go_to = [&](int pos) {
            const int g = tile_of(pos);
            at.step(g - g_at, lane, true);
            if (at.lost) return false;
            g_at = g;
            const int k = at.t * BN + (lane & 7) * 16;
            page = (lane & 7) * 16 < BN && k < at.item().key_end ? entry_page(a.batch, at.item().b, k) : 0;
            return true;
        };
        auto put_scales = [&](int g, float f) {
            float* to = fac[g % kFacTiles];
            if (lane < 8) to[lane] = f * a.scale_log2;
            if (lane >= 8 && lane < 16) {  // a positive normal number: fraction and exponent
                const int bits = __float_as_int(f);
                to[lane] = __int_as_float((bits & 0x7fffff) | 0x3f800000);
                to[lane + 8] = (float)((bits >> 23) - 127);
            }
            __syncwarp();
        };
        bool more = go_to(me);
        for (int pos = me; more; pos += C::kLoads) {
            const int slot = pos % NS, g = g_at;
            unsigned char* dst = ring + slot * C::kSlot;
            const bool key = pos == 0 || (pos & 1);
            const Item<ROWS, BN>& p = at.item();
            const int k0 = at.t * BN, h = p.h;
            const int end = min(p.key_end - k0, BN);  // rows of the tile that exist
            const int open = max(p.open - k0, 0);     // values from here on: not every row of the item sees them
            // the tile's scales, keys' (lanes 0 to 7) and values' (8 to 15), on their way while the slot is waited for
            float f = 1.f;
            const int x = (lane & 7) * 16;
            if (key && lane < 16 && x < end && page >= 0)
                f = (lane < 8 ? a.scales.k : a.scales.v)[scale_index(a.batch, a.scales, a.n_kv_heads, page, h, k0 + x)];
            if (page < 0) record_status(a.status, PP_ERR_INVALID_ARG);
            if (__any_sync(kFull, pos >= NS && !attn_wait(&empty[slot], (uint32_t)(pos / NS - 1) & 1u, w))) break;
            // rows past the end: zeros (a weight of zero does not outweigh NaN); hidden ones: finite
            const bool fix = !key && (end < BN || open < end);
            if (a.box > 0) {
                // boxes of 128 elements x min(page, BN) tokens
                const int boxes = (end + a.box - 1) / a.box * NG;
                uint64_t* bar = fix ? &landed[me] : &full[slot];
                const int row = lane / NG * a.box, grp = lane % NG;
                const int in_page = (int)((unsigned)(k0 + row) % (unsigned)a.batch.page_size);
                const int of = __shfl_sync(kFull, page, (row >> 4) & 7);
                if (lane < boxes)  // a page that does not exist lies past the last one: zeros
                    tma_load_4d(dst + grp * BN * 128 + row * 128, key ? &map_k : &map_v, grp * 128, h, in_page,
                                of < 0 ? a.batch.n_pages : of, bar);
                if (key) put_scales(g, f);
                // (bytes may have landed before they are expected: the phase waits for this arrival)
                if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(boxes * a.box * 128));
            } else {
#pragma unroll 1
                for (int r0 = 0; r0 < BN; r0 += 32) {
                    const int of = __shfl_sync(kFull, page, (r0 + lane) >> 4 & 7);
                    const long long off = r0 + lane < end && of >= 0
                        ? entry_offset(a.batch, a.cache, of, k0 + r0 + lane) + (long long)h * a.cache.head_stride : -1;
                    copy_codes32<DP, BN>(dst, r0, key ? a.cache.k : a.cache.v, off, a.head_dim, lane);
                }
                cp_async_commit();
                if (key) put_scales(g, f);
            }
            if (!key || a.box == 0) {
                // landed, and mended where it has to be
                bool gone = false;
                if (a.box == 0) {
                    cp_async_wait<0>();
                    __syncwarp();
                } else if (fix) {
                    gone = __any_sync(kFull, !attn_wait(&landed[me], (uint32_t)fixes++ & 1u, w));
                }
                if (gone) break;
                if (fix) {
                    Item<ROWS, BN>& it = items[at.n % kItems];
                    finite_codes<DP, BN>(dst, open, end, lane, k0, &it.odd0, &it.odd1);
                    zero_codes<DP, BN>(dst, end, BN, lane);
                }
                if (a.box == 0 || fix) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&full[slot]);
                }
            }
            more = go_to(pos + C::kLoads);
        }
    } else if (warp == C::kWarpQ) {
        // ------------------------------------- rows of q: two pieces, eight copies
        at.enter(0);
        bool lost = at.lost;
        constexpr int kE = DP / 32, kAhead = 4;  // elements of a lane, rows on their way
        const int d = lane * kE;
        auto fetch = [&](const Item<ROWS, BN>& p, int r, uint2 (&v)[kE / 4]) {
#pragma unroll
            for (int i = 0; i < kE / 4; i++) v[i] = make_uint2(0u, 0u);
            if (r >= p.rows || d >= a.head_dim) return;
            const uint2* src = reinterpret_cast<const uint2*>(a.q + row_offset(a, p, p.j * ROWS + r, a.q_stride, 2) + d * 2);
#pragma unroll
            for (int i = 0; i < kE / 4; i++) v[i] = src[i];
        };
        while (!lost) {
            const Item<ROWS, BN>& p = at.item();
            const int n = at.n, buf = n & 1;
            uint2 v[kAhead][kE / 4];
#pragma unroll
            for (int k = 0; k < kAhead; k++) fetch(p, k, v[k]);  // while the buffer is waited for
            lost = __any_sync(kFull, n > 1 && !attn_wait(&qempty[buf], (uint32_t)(n / 2 - 1) & 1u, w));
            if (lost) break;
#pragma unroll 1
            for (int r0 = 0; r0 < p.rows; r0 += kAhead) {
#pragma unroll
                for (int k = 0; k < kAhead; k++) {
                    const int r = r0 + k;
                    if (r >= p.rows) break;
                    float x[kE], amax = 0.f;
#pragma unroll
                    for (int i = 0; i < kE / 4; i++) {
                        x[4 * i] = bf16lo(v[k][i].x);
                        x[4 * i + 1] = bf16hi(v[k][i].x);
                        x[4 * i + 2] = bf16lo(v[k][i].y);
                        x[4 * i + 3] = bf16hi(v[k][i].y);
                    }
#pragma unroll
                    for (int i = 0; i < kE; i++) amax = fmaxf(amax, magnitude(x[i]));
                    const float sc = scale_for(warp_max(amax)), inv = 1.f / sc;
                    if (lane == 0) q_scale[n % kItems][r] = sc;
#pragma unroll
                    for (int i = 0; i < kE; i += 4) {
                        float y[4];
#pragma unroll
                        for (int u = 0; u < 4; u++) y[u] = to_hold(x[i + u]) * inv;
                        uint32_t piece[2];
                        split4(pair2(y[0], y[1]), pair2(y[2], y[3]), piece);
                        const int e = d + i;  // element: 16-byte chunk e / 16 of group e / 128
                        unsigned char* base = qs + buf * C::kQTile + (e >> 7) * 128 * 128 + (e & 15) + r * 128 +
                                              ((((e & 127) >> 4) ^ (r & 7)) << 4);
#pragma unroll
                        for (int c = 0; c < 4; c++)
#pragma unroll
                            for (int u = 0; u < 4; u++) *reinterpret_cast<uint32_t*>(base + (32 * c + 8 * u) * 128) = piece[u & 1];
                    }
                }
#pragma unroll
                for (int k = 0; k < kAhead; k++) fetch(p, r0 + kAhead + k, v[k]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&qfull[buf]);
            at.next(lane, true);
            lost = at.lost;
        }
    } else if (warp >= C::kWarpMma) {
        // ---------------------------------------------------------- products
        const uint32_t id_s = idesc_f8_m128(BN, false), id_o = idesc_f8_m128(a.head_dim, true);
        const int who = __shfl_sync(kFull, warp - C::kWarpMma, 0);
        const bool one = lane == 0;
        const uint32_t tm = __shfl_sync(kFull, tmem, 0);
        const int steps = (a.head_dim + 31) / 32;  // of K = 32
        at.enter(0);
        auto wait_full = [&](int pos) { attn_wait(&full[pos % NS], (uint32_t)(pos / NS) & 1u, w); };
        if (who == 0) {
#pragma unroll 1
            for (int g = 0; !at.lost; g++) {
                const int buf = at.n & 1;
                if (at.t == at.t0) attn_wait(&qfull[buf], (uint32_t)(at.n / 2) & 1u, w);
                wait_full(k_pos(g));
                const int sl = g & 1;
                if (g >= 2)  // the slot's last weights have been multiplied
                    attn_wait(&odone[g & 1], (uint32_t)((g - 2) >> 1) & 1u, w);
                tc_fence_after();
                if (one) {
                    const uint64_t ad = sdesc_sw128(qs + buf * C::kQTile), bd = sdesc_sw128(ring + (k_pos(g) % NS) * C::kSlot);
#pragma unroll
                    for (int d = 0; d < DP / 32; d++)  // 32 bytes a step, in descriptors' units of 16
                        if (d < steps)
                            umma_f8(tm + (uint32_t)(sl * BN), ad + (uint64_t)((d >> 2) * 1024 + 2 * (d & 3)),
                                    bd + (uint64_t)((d >> 2) * BN * 8 + 2 * (d & 3)), id_s, d > 0 ? 1u : 0u);
                    umma_commit(&sfull[sl]);
                    umma_commit(&empty[k_pos(g) % NS]);
                    if (at.t + 1 == at.t1) umma_commit(&qempty[buf]);
                }
                __syncwarp();
                at.step(1, lane, true);
            }
        } else {
#pragma unroll 1
            for (int g = 0; !at.lost; g++) {
                wait_full(v_pos(g));
                attn_wait(&pfull[g & 1], (uint32_t)(g >> 1) & 1u, w);
                tc_fence_after();
                if (one) {
                    const uint64_t vd = sdesc_sw128_n(ring + (v_pos(g) % NS) * C::kSlot, BN * 128);
#pragma unroll
                    for (int k = 0; k < BN / 32; k++)
                        umma_f8_ta(tm + C::kTmemO + (uint32_t)(at.n % C::kOuts * DP), tm + (uint32_t)((g & 1) * BN + 32 * k), vd + (uint64_t)(k * 256),
                                   id_o, (at.t > at.t0 || k > 0) ? 1u : 0u);
                    umma_commit(&odone[g & 1]);
                    if (at.t + 1 == at.t1) umma_commit(&opart[at.n % C::kOuts]);
                    umma_commit(&empty[v_pos(g) % NS]);
                }
                __syncwarp();
                at.step(1, lane, true);
            }
        }
    } else if (warp < C::kWarpOut) {
        // ----------------------------------------------------------- softmax
        const int wq = warp, row = lane & 7, piece = lane >> 3;
        const bool b1 = lane & 16, b0 = lane & 8;  // the piece's (and the eight keys') bits
        const uint32_t lanes = (uint32_t)(32 * wq) << 16;
        const float c_own = b0 ? 0x1p-4f : 1.f, c_other = b0 ? 1.f : 0x1p-4f;  // of the queries' pieces
        int g = 0;  // tile of the stretch
        auto products_done = [&](int x) {
            attn_wait(&odone[x & 1], (uint32_t)(x >> 1) & 1u, w);
            tc_fence_after();
        };
        if (wq < C::kParts) at.enter(0);
        while (wq < C::kParts && !at.lost) {
            const Item<ROWS, BN>& p = at.item();
            const int tok = min((p.j * ROWS + row) / a.group, p.seq.n - 1);
            const int open = p.open, t0 = at.t0, t1 = at.t1, ob = at.n % C::kOuts;
            const uint32_t t_o = tmem + C::kTmemO + (uint32_t)(ob * DP) + lanes;
            float m = -INFINITY, b = -INFINITY, sum = 0.f, qsc = 0.f;
            // the buffer's last part has been read
            if (at.n >= C::kOuts) attn_wait(&ofree[ob], (uint32_t)(at.n / C::kOuts - 1) & 1u, w);
            for (int t = t0; t < t1; t++, g++) {
                const uint32_t t_s = tmem + (uint32_t)((g & 1) * BN) + lanes;
                attn_wait(&sfull[g & 1], (uint32_t)(g >> 1) & 1u, w);
                tc_fence_after();
                uint32_t u[32];
                tmem_ld32(t_s + 32 * wq, u);
                tmem_ld_wait();
                // scales of the row and the tile: written ahead of the products
                if (t == t0) qsc = q_scale[at.n % kItems][row];
                const float* fc = fac[g % kFacTiles] + 2 * wq + (b1 ? 1 : 0);
                const float f = fminf(fmaxf(fc[0] * qsc, 0x1p-126f), 0x1p127f);  // positive and finite: -inf stays, and 0
                const float vs = fc[8], lv = fc[16];
                // the row's scores of this lane's eight keys, from its piece of the query and that of the lane 8 further
                float s[8];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    float own[2], got[2];
#pragma unroll
                    for (int v = 0; v < 2; v++) {
                        const uint32_t first = b1 ? u[16 + i + v] : u[i + v], second = b1 ? u[24 + i + v] : u[8 + i + v];
                        got[v] = __shfl_xor_sync(kFull, __uint_as_float(b0 ? first : second), 8);
                        own[v] = __uint_as_float(b0 ? second : first);
                    }
                    unpair2(fma2(pair2(got[0], got[1]), pair2(c_other, c_other), mul2(pair2(own[0], own[1]), pair2(c_own, c_own))), s[i], s[i + 1]);
                }
                const int k0 = t * BN + 32 * wq;
                if (k0 + 32 > open) {
                    const uint32_t see = seen_bits(a, p, tok, k0) >> 8 * piece;
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (!(see >> i & 1u)) s[i] = -INFINITY;
                }
                const float x = max3(max3(s[0], s[1], s[2]), max3(s[3], s[4], s[5]), fmaxf(s[6], s[7])) * f;
                const float xb = x == -INFINITY ? 0.f : x;
                // the scores' maximum moves with every tile (a register), O's base when it has to
                const float m_new = fmaxf(x, m), mb = m_new == -INFINITY ? 0.f : m_new;
                const float own_top = x + lv;
                if (__any_sync(kFull, own_top > b + kLazy8)) {  // (also the first keys that are seen: b is -inf ahead of them)
                    float top = fmaxf(own_top, __shfl_xor_sync(kFull, own_top, 16));
                    top = fmaxf(top, __shfl_xor_sync(kFull, top, 8));
                    const bool grow = top > b + kLazy8;
                    const float fo = grow ? ex2(b - top) : 1.f;  // 0 from -inf
                    b = grow ? top : b;
                    if (t > t0) {
                        products_done(g - 1);
#pragma unroll 1
                        for (int c = 0; c < a.head_dim; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(t_o + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; i++) o[i] = __float_as_uint(__uint_as_float(o[i]) * fo);
                            tmem_st16(t_o + c, o);
                        }
                    }
                }
                // (x + lv is at most b + kLazy8, unless nothing is seen and the weights are zero whatever this is)
                const float weight = ex2(fminf(xb - (b == -INFINITY ? 0.f : b) + lv, kLazy8 + 1.f)) * kTopWeight * vs;
                const unsigned long long f2 = pair2(f, f), w2 = pair2(weight, weight), nb = pair2(-xb, -xb);
                unsigned long long part = 0ull;
                uint32_t w_own[4][2];  // of a piece: the codes of the eight keys
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    unsigned long long y[2];
#pragma unroll
                    for (int v = 0; v < 2; v++) {
                        float e0, e1;
                        unpair2(fma2(pair2(s[4 * i + 2 * v], s[4 * i + 2 * v + 1]), f2, nb), e0, e1);
                        const unsigned long long e = pair2(ex2(e0), ex2(e1));
                        part = add2(part, e);
                        y[v] = mul2(e, w2);
                    }
                    uint32_t word[4];
                    split4(y[0], y[1], word);
#pragma unroll
                    for (int u2 = 0; u2 < 4; u2++) w_own[u2][i] = word[u2];
                }
                float e0, e1;
                unpair2(part, e0, e1);
                sum = fmaf(e0 + e1, ex2(x - mb), sum * ex2(m - mb));
                m = m_new;
                // lane 8 p + i stores piece p of all 32 keys of row i: first pieces 2 b1 and 2 b1 + 1 of this lane's eight
                // keys and of those of the lane 16 further, then its own piece of all four
                uint32_t two[2][2][2];  // [keys' upper bit][piece's lower bit][word]
#pragma unroll
                for (int v = 0; v < 2; v++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint32_t own = b1 ? w_own[2 + v][i] : w_own[v][i];
                        const uint32_t got = __shfl_xor_sync(kFull, b1 ? w_own[v][i] : w_own[2 + v][i], 16);
                        two[0][v][i] = b1 ? got : own;
                        two[1][v][i] = b1 ? own : got;
                    }
                uint32_t out[8];
#pragma unroll
                for (int v = 0; v < 2; v++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint32_t own = b0 ? two[v][1][i] : two[v][0][i];
                        const uint32_t got = __shfl_xor_sync(kFull, b0 ? two[v][0][i] : two[v][1][i], 8);
                        out[4 * v + i] = b0 ? got : own;
                        out[4 * v + 2 + i] = b0 ? own : got;
                    }
                const uint32_t zero[8] = {};
#pragma unroll
                for (int c = 1; c < C::kParts; c++) tmem_st8(t_s + 32 * ((wq + c) % C::kParts), zero);
                tmem_st8(t_s + 32 * wq, out);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&pfull[g & 1]);
            }
            stat_m[ob][wq][lane] = m;
            stat_b[ob][wq][lane] = b;
            stat_l[ob][wq][lane] = sum;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ofull[ob]);
            at.next(lane, true);
        }
        // (quarters without keys free the parts all the same)
        if (wq >= C::kParts) {
            at.enter(0);
            while (!at.lost) at.next(lane, true);
        }
    } else {
        // ------------------------------------------------------- ends of parts
        const int wq = warp - C::kWarpOut, row = lane & 7, piece = lane >> 3, otid = tid - 32 * C::kWarpOut;
        const bool b1 = lane & 16, b0 = lane & 8, active = wq < C::kParts;
        const uint32_t lanes = (uint32_t)(32 * wq) << 16;
        const float c_own = piece_weight(piece);
        const int D = a.head_dim;
        at.enter(0);
        while (!named_bar_or(2, 128, at.lost)) {
            const Item<ROWS, BN>& p = at.item();
            const int rows = p.rows, ob = at.n % C::kOuts;
            const uint32_t t_o = tmem + C::kTmemO + (uint32_t)(ob * DP) + lanes, par = (uint32_t)(at.n / C::kOuts) & 1u;
            attn_wait(&ofull[ob], par, w);
            attn_wait(&opart[ob], par, w);
            tc_fence_after();
            const bool whole = p.whole();
            // written by the producers ahead of the products
            const int odd0 = *const_cast<const volatile int*>(&p.odd0), odd1 = *const_cast<const volatile int*>(&p.odd1);
            const Split<ROWS, BN>& sp = p.split;
            float* place = nullptr;
            if (!whole) {
                attn_wait(&isplit[at.n % kItems], (uint32_t)(at.n / kItems) & 1u, w);
                place = sp.place(a, (int)blockIdx.x / sp.step);
            }
            float top = -INFINITY, l = 0.f;
#pragma unroll
            for (int i = 0; i < C::kParts; i++)
#pragma unroll
                for (int n = row; n < 32; n += 16) top = max3(top, stat_m[ob][i][n], stat_m[ob][i][n + 8]);
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int i = 0; i < C::kParts; i++)
#pragma unroll
                for (int n = row; n < 32; n += 8) l = fmaf(stat_l[ob][i][n], ex2(stat_m[ob][i][n] - base), l);
            const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
            // from this copy's base (a power of two that may be far from the row's maximum: in two steps) to the row's
            // (nothing seen: zeros; scores that are all NaN: O, which is NaN)
            const float b = stat_b[ob][wq][lane], all = stat_l[ob][wq][row] + stat_l[ob][wq][row + 8] + stat_l[ob][wq][row + 16] +
                        stat_l[ob][wq][row + 24];
            const bool none = !active || (b == -INFINITY && all == all);
            const float e = b == -INFINITY ? 0.f : b - base, half = 0.5f * e;
            const float f1 = ex2(half) * c_own * inv / kTopWeight, f2 = ex2(e - half);
#pragma unroll 1
            for (int c = 0; c < D; c += 128) {
                if (active) {
#pragma unroll 1
                    for (int x = 0; x < 128 && c + x < D; x += 32) {
                        uint32_t o[32];
                        tmem_ld32(t_o + c + x, o);
                        tmem_ld_wait();
                        // a row's four pieces added up, eight elements a lane
                        float h[16], y[8];
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            const float u = none ? 0.f : __uint_as_float(o[i]) * f1 * f2;
                            const float v = none ? 0.f : __uint_as_float(o[16 + i]) * f1 * f2;
                            const float got = __shfl_xor_sync(kFull, b1 ? u : v, 16);
                            h[i] = (b1 ? v : u) + got;
                        }
#pragma unroll
                        for (int i = 0; i < 8; i++) {
                            const float got = __shfl_xor_sync(kFull, b0 ? h[i] : h[8 + i], 8);
                            y[i] = (b0 ? h[8 + i] : h[i]) + got;
                        }
                        float* dst = stage + (wq * ROWS + row) * C::kPitch + x + 8 * piece;
                        reinterpret_cast<float4*>(dst)[0] = make_float4(y[0], y[1], y[2], y[3]);
                        reinterpret_cast<float4*>(dst)[1] = make_float4(y[4], y[5], y[6], y[7]);
                    }
                }
                if (c + 128 >= D) {  // O and the statistics have been read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ofree[ob]);
                }
                named_bar_sync(2, 128);
#pragma unroll 1
                for (int i = otid; i < rows * 16; i += 128) {
                    const int er = i >> 4, ed = (i & 15) * 8;
                    if (c + ed >= D) continue;
                    float o[8] = {};
#pragma unroll
                    for (int x = 0; x < C::kParts; x++)
#pragma unroll
                        for (int k = 0; k < 8; k += 4) {
                            const float4 v = *reinterpret_cast<const float4*>(stage + (x * ROWS + er) * C::kPitch + ed + k);
                            o[k] += v.x;
                            o[k + 1] += v.y;
                            o[k + 2] += v.z;
                            o[k + 3] += v.w;
                        }
                    if (odd0 < odd1) {
                        float t[8];
                        odd_values<true, 8>(a, p, odd0, odd1, p.j * ROWS + er, c + ed, t);
                        for (int k = 0; k < 8; k++) o[k] += t[k];
                    }
                    if (whole) {
                        *reinterpret_cast<uint4*>(a.out + row_offset(a, p, p.j * ROWS + er, a.out_stride, 2) + (c + ed) * 2) =
                            Elem<__nv_bfloat16>::pack(o);
                    } else {
                        float4* dst = reinterpret_cast<float4*>(place + (size_t)er * D + c + ed);
                        dst[0] = make_float4(o[0], o[1], o[2], o[3]);
                        dst[1] = make_float4(o[4], o[5], o[6], o[7]);
                    }
                }
                if (c + 128 < D) named_bar_sync(2, 128);  // (the next part's barrier otherwise)
            }
            if (!whole && otid < ROWS) {
                place[(size_t)ROWS * D + otid] = top;
                place[(size_t)ROWS * (D + 1) + otid] = l;
            }
            if (!whole) {
                named_bar_sync(2, 128);
                // (a part whose split did not come has set lost_s before the barrier)
                if (otid == 0) last_s = !*w.lost && arrive_last(a.counters + sp.cta(sp.c0), (unsigned)(sp.c1 - sp.c0 + 1));
                named_bar_sync(2, 128);
                if (last_s) merge_few<__nv_bfloat16, ROWS, BN, 4>(a, p, sp, rows, otid, 128);
            }
            at.next(lane, true);
        }
    }
    if (*w.lost)  // copies and products that may still be on their way: 1 ms is a hundred times what they take
        for (const uint64_t t0 = globaltimer_ns(); globaltimer_ns() - t0 < 1000000ull;) __nanosleep(10000);
    tc_fence_before();
    __syncthreads();
    if (warp == C::kWarpMma) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Codes as a 4-D tensor (element, head, offset in the page, page), boxes of 128
// elements x `box` tokens of one head and page.
bool code_map(CUtensorMap* map, const AttnArgs& a, const char* base) {
    auto enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.batch.page_size,
                                (cuuint64_t)a.batch.n_pages};
    const long long steps[3] = {a.cache.head_stride, a.cache.token_stride, a.cache.page_stride};
    cuuint64_t strides[3];
    for (int i = 0; i < 3; i++) strides[i] = dims[i + 1] == 1 && steps[i] < 16 ? 16 : (cuuint64_t)steps[i];
    const cuuint32_t box[4] = {128, 1, (cuuint32_t)a.box, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    // no more than a head's row from HBM where what lies beside it is another head's that is read at another time
    const bool alone = a.head_dim <= 128 && a.head_shift == 0 && a.cache.head_stride < a.cache.token_stride;
    const CUtensorMapL2promotion promote = alone ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<char*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, promote, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP>
cudaError_t few_go(AttnArgs a, int sms, cudaStream_t st) {
    using C = Few<DP>;
    auto* kern = attn8_few_kernel<DP>;
    static std::atomic<bool> allowed[64];
    cudaError_t e = allow_smem(kern, C::kSmem, allowed);
    if (e != cudaSuccess) return e;
    // TMA boxes where pages and key tiles divide one another; else 16-byte cp.async
    const int ps = a.batch.page_size;
    a.box = C::BN % ps == 0 || ps % C::BN == 0 ? (ps < C::BN ? ps : C::BN) : 0;
    // Heads side by side at the same time where a token's lie together: HBM gives rows of 128 bytes a kilobyte apart slower
    // than their neighbours' with them (1 / 2 / 4 / 8 heads, 64 single tokens 105.1 / 100.1 / 99.1 / 99.7 us).
    a.head_shift = 0;
    if (a.cache.head_stride < a.cache.token_stride)
        while (a.head_shift < 2 && a.n_kv_heads % (2 << a.head_shift) == 0) a.head_shift++;
    CUtensorMap mk{}, mv{};
    if (a.box && (!code_map(&mk, a, a.cache.k) || !code_map(&mv, a, a.cache.v))) a.box = 0;
    const unsigned grid = (unsigned)(sms < kAttnTcGrid ? sms : kAttnTcGrid) >> a.head_shift << a.head_shift;
    return launch_overlapped(kern, dim3(grid), dim3(C::kWarps * 32), C::kSmem, st, a, mk, mv);
}

}  // namespace

cudaError_t attn8_few_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    return a.head_dim <= 128 ? few_go<128>(a, sms, st) : few_go<256>(a, sms, st);
}

}  // namespace pp
