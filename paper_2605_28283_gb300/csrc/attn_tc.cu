// Attention over the paged cache on the tensor cores (bf16).
//
// One persistent CTA per SM walks its stretch of the key line
// (pp_attn_sched.cuh).  For a tile of BN keys: S = Q K^T (tcgen05, 128 rows x
// BN, accumulator in TMEM), softmax weights by one thread a row with a running
// maximum, P (bf16) written back over S in TMEM, O += P V (P from TMEM, V from
// shared memory as it lies in the cache, O in TMEM).  The maximum is lazy: O
// and the weight sum are rescaled only when a row's maximum has grown by more
// than 2^8, so the rescaling round trip through registers almost never runs.
//
// Warps: 4 per row tile for the softmax, two that issue the products, one that
// loads the rows of q, one producer for each slot of the key/value ring, and
// one that walks the stretch and hands its parts to the others.  A producer
// fills its slot by TMA, a box a page, where pages divide the key tile (or the
// reverse), else with 16-byte cp.async into the same swizzled layout (any page
// size, stride and head dimension); rows past the sequence are zeros.
//
// Few rows (a single token has as many as heads share a key head): 128-row
// products cost the tensor cores less than the keys cost HBM (8 of 23 cycles a
// key at D = 128), but one warp would hold all rows.  For up to 32 rows the
// rows are therefore repeated in every warp's lanes, each warp weighs its own
// 32 keys of the tile (P is zero elsewhere) with its own maximum and sum, and
// the copies are added up at the end of the part.
//
// More than 128 rows on average (MT = 2): two row tiles share each key tile.
//
// Measured (GB300): one token for each of 64 ragged sequences of 64 to 8191
// entries, 32 heads on 8 key heads of 128: 168 us, 6.4 TB/s (0.94 of the copy
// rate), bound by HBM.  One token over 1024 entries: 11.8 us, a chain of
// latencies.  8 drafted trees of 17 to 48 tokens over 500 to 6000 entries: 43
// us, bound by the softmax warps and the ends of parts.  4 prompts of 2048
// tokens, 40 heads of 128: 196 us, 877 TFLOP/s (0.46 of the bf16 rate), the
// row tiles' softmaxes and products in turns.  The code is long for its cache:
// loops stay rolled unless straight-line code was measured to be faster.
#include "pp_attn_sched.cuh"
#include "pp_kernels.h"
#include "pp_launch.cuh"
#include "pp_tc_attn.cuh"

namespace pp {
namespace {

constexpr float kLazy = 8.0f;  // growth of a row's maximum (log2) that O and the sum absorb unscaled

constexpr int kTurn = 5;  // 16-byte words a row of 32 bf16 takes in the turning area (one of padding)

template <int DP, int MT>
struct Tc {
    static constexpr int BN = DP == 256 ? 64 : 128;  // keys of a tile
    static constexpr int NG = DP / 64;               // 64-element groups of the head dimension
    static constexpr int kRows = 128 * MT;
    static constexpr int kSlot = BN * DP * 2;
    static constexpr int kSlots = DP == 64 && MT == 1 ? 6 : 4;  // even: a producer sees keys only or values only
    static constexpr int kQTile = 128 * DP * 2;
    static constexpr int kQBufs = MT == 2 ? 2 : DP == 256 ? 1 : 2;  // MT 2: one for each row tile
    static constexpr int kParts = BN / 32;           // copies of the rows when there are few
    // few rows: 4 warps x 32 rows x 32 elements, or 8 x 128 (fp32); else 32 rows x 32 elements (bf16) a warp
    static constexpr int kStage = MT == 1 ? 4 * 32 * 36 * 4 : 8 * 32 * kTurn * 16;
    static constexpr int kSmem = kSlots * kSlot + kQBufs * kQTile + kStage + 1024;
    static constexpr int kSoftWarps = 4 * MT;
    // warps after the softmax ones: two that issue products, the rows of q, the slots' producers, the schedule
    static constexpr int kWarpMma = kSoftWarps, kWarpQ = kSoftWarps + 2, kWarpSlot = kSoftWarps + 3;
    static constexpr int kWarps = kWarpSlot + kSlots + 1;
    static constexpr int kReaders = kWarps - 1;  // that free a part
    static constexpr uint32_t kTmemO = 2 * BN;       // S / P slots first
    static constexpr uint32_t kTmemCols = 512;
    static_assert(kTmemO + MT * DP <= 512, "TMEM columns");
};

// First entry that some row of the tile does not see (entries below it need
// no mask, and their values no check).
template <int ROWS>
PP_DEVINL int all_see(const AttnArgs& a, const Part& p) {
    return a.mask ? p.seq.ctx : p.seq.ctx + (int)((unsigned)p.j * ROWS / (unsigned)a.group) + 1;
}

// Key tiles [p.t0, tile_end) of the part are of use to row tile m (MT 2: the
// first one's rows end earlier in a prompt; a short item leaves the second
// one empty).
template <int BN, int MT>
PP_DEVINL int tile_end(const AttnArgs& a, const Part& p, int m) {
    if (MT == 1) return p.t1;
    const int rows = p.seq.n * a.group - p.j * 128 * MT;
    if (128 * m >= rows) return p.t0;
    if (a.mask) return p.t1;
    const unsigned last = ((unsigned)p.j * (128 * MT) + 128u * (unsigned)(m + 1) - 1u) / (unsigned)a.group;
    const int end = p.seq.ctx + min(p.seq.n, (int)last + 1);
    return max(p.t0, min(p.t1, (end + BN - 1) / BN));
}

// Bits of the 32 entries from k0 on that new token `tok` sees.
PP_DEVINL uint32_t seen_bits(const AttnArgs& a, const Part& p, int tok, int k0) {
    const int j = k0 - p.seq.ctx;  // new token's number of bit 0
    int end;
    uint32_t bits = 0xffffffffu;
    if (a.mask) {
        end = p.seq.n - j;
        if (j > -32) {
            const uint32_t* w = a.mask + (size_t)(p.seq.q0 + tok) * a.mask_words;
            if (j < 0) {  // the first -j bits are cached tokens
                bits = (w[0] << -j) | (0xffffffffu >> (32 + j));
            } else {
                const int i = j >> 5;
                const uint32_t lo = i < a.mask_words ? w[i] : 0u, hi = i + 1 < a.mask_words ? w[i + 1] : 0u;
                bits = __funnelshift_r(lo, hi, j & 31);
            }
        }
    } else {
        end = tok + 1 - j;
    }
    return end >= 32 ? bits : end <= 0 ? 0u : bits & ((1u << end) - 1u);
}

PP_DEVINL bool sees(const AttnArgs& a, const Part& p, int tok, int j) {  // new token j
    if (!a.mask) return j <= tok;
    return j < 32 * a.mask_words && (a.mask[(size_t)(p.seq.q0 + tok) * a.mask_words + (j >> 5)] >> (j & 31) & 1u);
}

// A part as the warps of the CTA get it from the scheduling warp, in a ring in
// shared memory: walking the stretch takes divisions and dependent loads that
// the others' loops are spared.
template <int ROWS, int TOK>
struct Item : Part {
    int rows;    // query rows of the item
    int open;    // all_see
    int end[2];  // tile_end of the row tiles
    Split<ROWS, TOK> split;  // of a part that is not the whole item
    int odd0, odd1;  // entries from `open` on whose values are not all finite lie in [odd0, odd1)
};
constexpr int kItems = 8;

// A reader of the ring (a whole warp), at tile t of part n.
template <int ROWS, int TOK>
struct ItemAt {
    const Item<ROWS, TOK>* ring;
    uint64_t *full, *empty;
    Waits w;
    int n, t, t0, t1;
    bool lost;  // the part did not come: nothing of item() may be used, and the part has no end
    PP_DEVINL const Item<ROWS, TOK>& item() const { return ring[n % kItems]; }
    PP_DEVINL void enter(int n_) {
        n = n_;
        lost = __any_sync(kFull, !attn_wait(&full[n % kItems], (uint32_t)(n / kItems) & 1u, w));
        t = t0 = lost ? 0 : item().t0;
        t1 = lost ? 0x7fffffff : item().t1;
    }
    // The next part.  `release`: this reader counts among those that free an entry.
    PP_DEVINL void next(int lane, bool release) {
        __syncwarp();
        if (release && lane == 0) mbar_arrive(&empty[n % kItems]);
        enter(n + 1);
    }
    // k tiles further (the caller stays inside the stretch); true in another part
    PP_DEVINL bool step(int k, int lane, bool release) {
        t += k;
        if (t < t1) return false;
        do {
            const int over = t - t1;
            next(lane, release);
            t += over;
        } while (t >= t1);
        return true;
    }
};

// One warp copies 32 rows of DP elements with 16-byte cp.async into a
// swizzled tile of 64-element groups, `group` bytes each; dst is the first
// row's place.  off is the byte offset from base of row `lane`, negative:
// zeros.  Rolled up: the code is run a few times a tile by one warp, and
// fetching it straight-line cost more than running it.
template <int DP>
PP_DEVINL void copy_rows32(unsigned char* dst, int group, const char* base, long long off, int D, int lane) {
    const int sub = lane >> 3, c = lane & 7;
#pragma unroll 1
    for (int i = 0; i < 8; i += 2) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int r = 4 * (i + k) + sub;
            const long long o = __shfl_sync(kFull, off, r);
#pragma unroll
            for (int g = 0; g < DP / 64; g++) {
                const bool in = o >= 0 && (g * 8 + c) * 8 < D;
                cp_async_16(dst + g * group + r * 128 + ((c ^ (r & 7)) << 4), in ? base + o + (g * 8 + c) * 16 : base,
                            in ? 16u : 0u);
            }
        }
    }
}

// Rows [r0, r1) of a value tile set to zero.
template <int DP, int BN>
PP_DEVINL void zero_rows(unsigned char* tile, int r0, int r1, int lane) {
#pragma unroll 1
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32)
#pragma unroll
        for (int g = 0; g < DP / 64; g++)
            *reinterpret_cast<uint4*>(tile + g * BN * 128 + e * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// Elements of rows [r0, r1) of a value tile that are not finite set to zero,
// and the entries that held any noted in [*odd0, *odd1) (k0: entry of row 0).
// For the entries that some row of the item does not see: its weight of zero
// does not outweigh NaN (or infinity) in the product.  0 * v summed is zero
// for finite values alone; one branch for the whole tile, since a branch a row
// kept the loads apart (4 prompts of 2048 tokens 194 -> 210 us, 8 trees 42.4 -> 43.9).
template <int DP, int BN>
PP_DEVINL void finite_rows(unsigned char* tile, int r0, int r1, int lane, int k0, int* odd0, int* odd1) {
    constexpr int NG = DP / 64;
    const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
    __nv_bfloat162 x[4] = {zero, zero, zero, zero};
#pragma unroll 4
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32) {
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const uint4 v = *reinterpret_cast<const uint4*>(tile + g * BN * 128 + e * 16);
            x[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&v.x), zero, x[0]);
            x[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&v.y), zero, x[1]);
            x[2] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&v.z), zero, x[2]);
            x[3] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&v.w), zero, x[3]);
        }
    }
    x[0] = __hadd2(__hadd2(x[0], x[1]), __hadd2(x[2], x[3]));
    if (__hbeq2(x[0], zero)) return;
#pragma unroll 1
    for (int e = r0 * 8 + lane; e < r1 * 8; e += 32) {
        bool odd = false;
#pragma unroll 1
        for (int i = 0; i < 8 * NG; i++) {
            uint16_t* v = reinterpret_cast<uint16_t*>(tile + (i >> 3) * BN * 128 + e * 16) + (i & 7);
            if ((*v & 0x7f80u) != 0x7f80u) continue;
            *v = 0;
            odd = true;
        }
        if (!odd) continue;
        atomicMin(odd0, k0 + (e >> 3));
        atomicMax(odd1, k0 + (e >> 3) + 1);
    }
}

// t[0..N) = sum of the non-finite values (elements d..) of the entries in
// [odd0, odd1) that the row sees: what finite_rows took out of its sum.  With
// a positive weight such a value counts as itself.
template <int N>
__device__ __noinline__ void odd_values(const AttnArgs& a, const Part& p, int odd0, int odd1, int row, int d, float* t) {
    const int tok = row / a.group;
#pragma unroll
    for (int i = 0; i < N; i++) t[i] = 0.f;
    for (int k = odd0; k < odd1; k++) {
        if (!sees(a, p, tok, k - p.seq.ctx)) continue;
        const int page = entry_page(a.batch, p.b, k);
        if (page < 0) continue;
        const char* v = a.cache.v + entry_offset(a.batch, a.cache, page, k) + (long long)p.h * a.cache.head_stride + d * 2;
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            if (d + i >= a.head_dim) break;
            float x[8];
            Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(v + i * 2), x);
#pragma unroll
            for (int u = 0; u < 8; u++)
                if (!isfinite(x[u])) t[i + u] += x[u];
        }
    }
}

// Scores of 32 N keys of one row, from t_s in TMEM (this warp's lanes).
template <int N>
struct Scores {
    uint32_t s[32 * N];
    PP_DEVINL void load(uint32_t t_s) {
#pragma unroll
        for (int c = 0; c < N; c++) tmem_ld32(t_s + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(s + 32 * c));
        tmem_ld_wait();
    }
    PP_DEVINL void hide(const AttnArgs& a, const Part& p, int tok, int k0) {
#pragma unroll
        for (int c = 0; c < N; c++) {
            const uint32_t see = seen_bits(a, p, tok, k0 + 32 * c);
            if (__all_sync(kFull, see == 0xffffffffu)) continue;
#pragma unroll
            for (int i = 0; i < 32; i++)
                if (!(see >> i & 1u)) s[32 * c + i] = __float_as_uint(-INFINITY);
        }
    }
    PP_DEVINL float max() const {
        float t[4] = {__uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2]), __uint_as_float(s[3])};
#pragma unroll
        for (int i = 4; i < 32 * N - 4; i += 8)
#pragma unroll
            for (int k = 0; k < 4; k++)
                t[k] = max3(t[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
        float u = max3(t[0], t[1], __uint_as_float(s[32 * N - 4])), v = max3(t[2], t[3], __uint_as_float(s[32 * N - 3]));
        return max3(max3(u, v, __uint_as_float(s[32 * N - 2])), __uint_as_float(s[32 * N - 1]), u);
    }
    // Weights 2^(s scale - base) to t_p as bf16 pairs; returns their sum.
    PP_DEVINL float weigh(uint32_t t_p, float scale, float base) {
        const unsigned long long sc = pair2(scale, scale), nb = pair2(-base, -base);
        unsigned long long sum0 = 0ull, sum1 = 0ull;
#pragma unroll
        for (int c = 0; c < N; c++) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int e = 32 * c + 2 * i;
                const unsigned long long x2 = fma2(pair2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), sc, nb);
                float x, y;
                unpair2(x2, x, y);
                x = ex2(x);
                y = ex2(y);
                w[i] = pack_bf16x2(x, y);
                if (i & 1)
                    sum1 = add2(sum1, pair2(x, y));
                else
                    sum0 = add2(sum0, pair2(x, y));
            }
            tmem_st16(t_p + 16 * c, w);
        }
        float x, y;
        unpair2(add2(sum0, sum1), x, y);
        return x + y;
    }
};

template <int DP, int MT>
__global__ void __launch_bounds__(Tc<DP, MT>::kWarps * 32, 1)
    attn_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q) {
    using C = Tc<DP, MT>;
    constexpr int BN = C::BN, NG = C::NG, ROWS = C::kRows, NS = C::kSlots;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* ring = smem;
    unsigned char* qs = smem + NS * C::kSlot;
    float* stage = reinterpret_cast<float*>(qs + C::kQBufs * C::kQTile);
    __shared__ uint64_t full[NS], empty[NS], landed[NS], qfull[2], qempty[2], sfull[2], pfull[2], odone[4], turn[2];
    __shared__ uint32_t taddr_s;
    __shared__ float stat_m[4][32], stat_l[4][32];
    __shared__ unsigned last_s;
    __shared__ Item<ROWS, BN> items[kItems];
    __shared__ uint64_t ifull[kItems], isplit[kItems], iempty[kItems], stretch;
    __shared__ int tiles_s;
    __shared__ unsigned lost_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Waits w{a.status, a.timeout_ns, &lost_s};
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < NS; i++) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], MT);
            mbar_init(&landed[i], 1);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(&qfull[i], 1);
            mbar_init(&qempty[i], 1);
            mbar_init(&sfull[i], 1);
            mbar_init(&pfull[i], 4);
            mbar_init(&odone[i], 1);
            mbar_init(&odone[2 + i], 1);
            mbar_init(&turn[i], 1);
        }
        for (int i = 0; i < kItems; i++) {
            mbar_init(&ifull[i], 1);
            mbar_init(&isplit[i], 1);
            mbar_init(&iempty[i], C::kReaders);
        }
        mbar_init(&stretch, 1);
        lost_s = 0u;
        fence_mbar_init();
    }
    if (warp == C::kWarpMma) {
        tmem_alloc(&taddr_s, C::kTmemCols);
        tmem_relinquish();
    }
    if (tid == C::kWarpSlot * 32 && a.box) {
        prefetch_map(&map_k);
        prefetch_map(&map_v);
    }
    if (tid == C::kWarpQ * 32 && a.q_box) prefetch_map(&map_q);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = taddr_s;
    pdl_wait();
    // A wait that gives up ends the CTA's work, its results lost: the scheduling
    // warp hands out no further part (nor overwrites one that others read), the
    // warps that load stop, those that issue products run through their tiles on
    // what lies there, and the softmax warps of a row tile, which meet in
    // barriers, agree before each part whether to go on.
    ItemAt<ROWS, BN> at{items, ifull, iempty, w, 0, 0, 0, 0, false};
    int tiles = 0;  // of this CTA
    if (warp < C::kWarps - 1) {
        bool lost = !attn_wait(&stretch, 0, w);
        lost = warp < C::kSoftWarps ? named_bar_or(2 + (warp >> 2), 128, lost) : __any_sync(kFull, lost);
        if (!lost) tiles = tiles_s;
    }

    if (warp == C::kWarps - 1) {
        // ---------------------------------------------------------- schedule
        Walk<ROWS, BN> walk = start_walk<ROWS, BN>(&a, lane, blockIdx.x == 0, 1);
        if (lane == 0) {
            tiles_s = (int)(walk.end - walk.at);
            mbar_arrive(&stretch);
            // the record that the second kernel joins by: no rows until an item is split here
            Item<ROWS, BN>* tail = reinterpret_cast<Item<ROWS, BN>*>(a.tails) + blockIdx.x;
            if (a.join_later) tail->rows = 0;
            Part p;
            for (int n = 0; walk.next(p); n++) {
                Item<ROWS, BN>& it = items[n % kItems];
                if (n >= kItems && !attn_wait(&iempty[n % kItems], (uint32_t)(n / kItems - 1) & 1u, w)) break;
                static_cast<Part&>(it) = p;
                it.rows = min(ROWS, p.seq.n * a.group - p.j * ROWS);
                it.open = all_see<ROWS>(a, p);
                it.odd0 = 0x7fffffff;
                it.odd1 = 0;
#pragma unroll 1
                for (int m = 0; m < MT; m++) it.end[m] = tile_end<BN, MT>(a, p, m);
                mbar_arrive(&ifull[n % kItems]);
                // the rest is for the end of the part
                if (!p.whole()) {
                    it.split = Split<ROWS, BN>(walk.sched, p);
                    mbar_arrive(&isplit[n % kItems]);
                    // an item that begins here and goes on in other stretches
                    if (a.join_later && p.t0 == 0) *tail = it;
                } else {
                    mbar_arrive(&isplit[n % kItems]);
                }
            }
        }
        __syncwarp();
    } else if (tiles <= 0) {
        // nothing for this CTA
    } else if (warp >= C::kWarpSlot) {
        // ------------------------------------------------- producer of one slot
        const int slot = warp - C::kWarpSlot;
        unsigned char* dst = ring + slot * C::kSlot;
        at.enter(0);
        int g_at = 0, uses = 0, fixes = 0;
        for (int pos = slot;; pos += NS, uses++) {
            // order of the loads: K0 K1 V0 K2 V1 K3 ... (MT 1: scores run two
            // tiles ahead), K0 V0 K1 V1 ... (MT 2)
            const bool key = MT == 1 ? pos == 0 || (pos & 1) : !(pos & 1);
            const int g = MT == 1 ? (pos == 0 ? 0 : key ? (pos + 1) / 2 : (pos - 2) / 2) : pos / 2;
            if (g >= tiles) break;
            at.step(g - g_at, lane, true);
            if (at.lost) break;
            g_at = g;
            const Item<ROWS, BN>& p = at.item();
            const int k0 = at.t * BN;
            const int end = min(p.key_end - k0, BN);  // rows of the tile that exist
            const int open = max(p.open - k0, 0);     // values from here on: not every row of the item sees them
            Item<ROWS, BN>& it = items[at.n % kItems];
            if (a.box > 0) {
                // boxes of 64 elements x min(page, BN) tokens, one for each of up to 32 lanes
                static_assert(BN / 8 * NG <= 32, "a lane for each box");
                const int boxes = (end + a.box - 1) / a.box * NG;
                // rows past the end: zeros (a weight of zero does not outweigh NaN); hidden ones: finite
                const bool fix = !key && (end < BN || open < end);
                uint64_t* bar = fix ? &landed[slot] : &full[slot];
                const int row = lane / NG * a.box, grp = lane % NG;
                const int in_page = (int)((unsigned)(k0 + row) % (unsigned)a.batch.page_size);
                int page = 0;
                if (lane < boxes) {
                    page = entry_page(a.batch, p.b, k0 + row);
                    if (page < 0) {  // lies past the last page: zeros
                        record_status(a.status, PP_ERR_INVALID_ARG);
                        page = a.batch.n_pages;
                    }
                }
                if (__any_sync(kFull, uses > 0 && !attn_wait(&empty[slot], (uint32_t)(uses - 1) & 1u, w))) break;
                if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(boxes * a.box * 128));
                __syncwarp();
                if (lane < boxes)
                    tma_load_4d(dst + grp * BN * 128 + row * 128, key ? &map_k : &map_v, grp * 64, p.h, in_page, page, bar);
                if (fix) {
                    if (__any_sync(kFull, !attn_wait(bar, (uint32_t)fixes++ & 1u, w))) break;
                    finite_rows<DP, BN>(dst, open, end, lane, k0, &it.odd0, &it.odd1);
                    zero_rows<DP, BN>(dst, end, BN, lane);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&full[slot]);
                }
            } else {
                if (__any_sync(kFull, uses > 0 && !attn_wait(&empty[slot], (uint32_t)(uses - 1) & 1u, w))) break;
#pragma unroll 1
                for (int x = 0; x < BN; x += 32) {
                    const int j = k0 + x + lane;
                    long long off = -1;
                    if (x + lane < end) {
                        const int page = entry_page(a.batch, p.b, j);
                        if (page >= 0)
                            off = entry_offset(a.batch, a.cache, page, j) + (long long)p.h * a.cache.head_stride;
                        else
                            record_status(a.status, PP_ERR_INVALID_ARG);
                    }
                    copy_rows32<DP>(dst + x * 128, BN * 128, key ? a.cache.k : a.cache.v, off, a.head_dim, lane);
                }
                cp_async_commit();
                cp_async_wait<0>();
                __syncwarp();
                if (!key) finite_rows<DP, BN>(dst, open, end, lane, k0, &it.odd0, &it.odd1);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&full[slot]);
            }
        }
    } else if (warp == C::kWarpQ) {
        // --------------------------------------------------------- rows of q
        at.enter(0);
        bool lost = at.lost;
        for (int left = tiles; !lost;) {
            const Item<ROWS, BN>& p = at.item();
            const int rows = p.rows, n = at.n;
#pragma unroll 1
            for (int m = 0; m < MT; m++) {
                const int buf = MT == 2 ? m : n % C::kQBufs, use = MT == 2 ? n : n / C::kQBufs;
                const bool few = MT == 1 && rows <= 32;
                lost = __any_sync(kFull, use > 0 && !attn_wait(&qempty[buf], (uint32_t)(use - 1) & 1u, w));
                if (lost) break;
                if (a.q_box) {
                    // boxes of 32 rows; past the item's rows they hold other tokens' (rows that nobody reads)
                    if (lane == 0) mbar_arrive_expect_tx(&qfull[buf], C::kQTile);
                    __syncwarp();
                    if (lane < 4 * NG) {
                        const int x = lane / NG, grp = lane % NG;
                        const int row = p.j * ROWS + 128 * m + (few ? 0 : 32 * x);
                        tma_load_3d(qs + buf * C::kQTile + grp * 128 * 128 + x * 32 * 128, &map_q, grp * 64,
                                    p.h * a.group, p.seq.q0 + row / a.group, &qfull[buf]);
                    }
                    __syncwarp();
                    continue;
                }
                __syncwarp();
#pragma unroll 1
                for (int x = 0; x < 4; x++) {
                    const int r = few ? (x < C::kParts ? lane : ROWS) : 128 * m + 32 * x + lane;
                    const long long off = r < rows ? row_offset(a, p, p.j * ROWS + r, a.q_stride, 2) : -1;
                    copy_rows32<DP>(qs + buf * C::kQTile + x * 32 * 128, 128 * 128, a.q, off, a.head_dim, lane);
                }
                cp_async_commit();
                cp_async_wait<0>();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&qfull[buf]);
            }
            left -= at.t1 - at.t0;
            if (lost || left <= 0) break;
            at.next(lane, true);
            lost = at.lost;
        }
    } else if (warp >= C::kWarpMma) {
        // ---------------------------------------------------------- products
        // Two warps, so that one's waits and address arithmetic (every wake-up
        // fetches its code anew) run under the other's products.  MT 2: one
        // for each row tile, scores one tile ahead of the values; MT 1: one
        // for the scores (two S slots), one for the values.
        constexpr uint32_t id_s = idesc_bf16_m128(BN), id_o = idesc_bf16_m128_bn(DP);
        const int who = __shfl_sync(kFull, warp - C::kWarpMma, 0);
        const int m = MT == 2 ? who : 0;
        const bool one = lane == 0;
        const uint32_t tm = __shfl_sync(kFull, tmem, 0);
        ItemAt<ROWS, BN> cs = at, co = at;  // scores, values
        cs.enter(0);
        co.enter(0);
        int end_s = cs.item().end[m], end_o = co.item().end[m];
        auto k_pos = [&](int g) { return MT == 1 ? (g == 0 ? 0 : 2 * g - 1) : 2 * g; };
        auto v_pos = [&](int g) { return MT == 1 ? 2 * g + 2 : 2 * g + 1; };
        auto s_slot = [&](int g) { return MT == 1 ? g & 1 : m; };
        auto wait_full = [&](int pos) { attn_wait(&full[pos % NS], (uint32_t)(pos / NS) & 1u, w); };
        auto q_buf = [&]() { return MT == 2 ? m : cs.n % C::kQBufs; };
        auto wait_q = [&]() { attn_wait(&qfull[q_buf()], (uint32_t)(MT == 2 ? cs.n : cs.n / C::kQBufs) & 1u, w); };
        auto issue_scores = [&](int g) {
            const unsigned char* kt = ring + (k_pos(g) % NS) * C::kSlot;
            const unsigned char* qt = qs + q_buf() * C::kQTile;
#pragma unroll
            for (int d = 0; d < NG; d++)
                umma_k64(tm + (uint32_t)(s_slot(g) * BN), qt + d * 128 * 128, kt + d * BN * 128, id_s, d > 0);
            umma_commit(&sfull[s_slot(g)]);
        };
        // n: the tile's number among those of use to the row tile
        auto release_values = [&](int g, int n, bool live) {
            if (live) umma_commit(&odone[2 * m + (n & 1)]);
            umma_commit(&empty[v_pos(g) % NS]);
        };
        auto release_scores = [&](int g) {  // the key slot and, behind the part's last tile, the rows of q
            umma_commit(&empty[k_pos(g) % NS]);
            if (cs.t + 1 == cs.t1) umma_commit(&qempty[q_buf()]);
        };
        auto issue_values = [&](int g) {
            const uint64_t vd = sdesc_sw128_n(ring + (v_pos(g) % NS) * C::kSlot, BN * 128);
#pragma unroll
            for (int k = 0; k < BN / 16; k++)
                umma_bf16_ta(tm + C::kTmemO + (uint32_t)(m * DP), tm + (uint32_t)(s_slot(g) * BN + 8 * k),
                             vd + (uint64_t)(k * 128), id_o, (co.t > co.t0 || k > 0) ? 1u : 0u);
        };
        if (MT == 2) {
            uint32_t n_o = 0;  // value products issued
#pragma unroll 1
            for (int g = -1; g < tiles; g++) {  // values of tile g, scores of the next: every wait but the weights' first
                const bool v = g >= 0 && co.t < end_o, more = g + 1 < tiles, sc = more && cs.t < end_s;
                const bool fresh = more && cs.t == cs.t0;  // its queries may still be on their way: values do not wait for them
                if (v) wait_full(v_pos(g));
                if (sc && !fresh) wait_full(k_pos(g + 1));
                if (v) attn_wait(&pfull[m], n_o++ & 1u, w);
                // the row tiles take turns: products of both at once would end at once, and then both softmaxes
                // run at once with the tensor cores idle
                // (the first after the second's last burst, the second after the first's of the same tile)
                if (g + m >= 0) attn_wait(&turn[m], (uint32_t)(g + m) & 1u, w);
                tc_fence_after();
                if (one && v) issue_values(g);
                if (fresh) {
                    if (one && g >= 0) release_values(g, (int)n_o - 1, v);
                    if (one) mbar_arrive(&turn[1 - m]);
                    wait_q();
                    if (sc) wait_full(k_pos(g + 1));
                    tc_fence_after();
                }
                if (one && sc) issue_scores(g + 1);
                if (one && !fresh) mbar_arrive(&turn[1 - m]);
                if (one && !fresh && g >= 0) release_values(g, (int)n_o - 1, v);  // behind the scores: commits cost issue time
                if (one && more) release_scores(g + 1);
                __syncwarp();
                if (g >= 0 && more && co.step(1, lane, true)) end_o = co.item().end[m];
                if (g + 2 < tiles && cs.step(1, lane, false)) end_s = cs.item().end[m];
            }
        } else if (who == 0) {
#pragma unroll 1
            for (int g = 0; g < tiles; g++) {
                if (cs.t == cs.t0) wait_q();
                wait_full(k_pos(g));
                // the slot's last weights have been multiplied
                if (g >= 2) attn_wait(&odone[g & 1], (uint32_t)((g - 2) >> 1) & 1u, w);
                tc_fence_after();
                if (one) {
                    issue_scores(g);
                    release_scores(g);
                }
                __syncwarp();
                if (g + 1 < tiles) cs.step(1, lane, true);
            }
        } else {
#pragma unroll 1
            for (int g = 0; g < tiles; g++) {
                wait_full(v_pos(g));
                attn_wait(&pfull[g & 1], (uint32_t)(g >> 1) & 1u, w);
                tc_fence_after();
                if (one) {
                    issue_values(g);
                    release_values(g, g, true);
                }
                __syncwarp();
                if (g + 1 < tiles) co.step(1, lane, true);
            }
        }
    } else {
        // ----------------------------------------------------------- softmax
        const int m = warp >> 2, wq = warp & 3;  // row tile, quarter of its lanes
        const uint32_t lanes = (uint32_t)(32 * wq) << 16;
        const uint32_t t_o = tmem + C::kTmemO + (uint32_t)(m * DP) + lanes;
        int g = 0;  // tile of the stretch
        // O holds the products up to tile x of this row tile (barriers take turns, so that a parity cannot stand
        // for the last phase but one)
        auto products_done = [&](int x) {
            attn_wait(&odone[2 * m + (x & 1)], (uint32_t)(x >> 1) & 1u, w);
            tc_fence_after();
        };
        at.enter(0);
        for (int left = tiles; !named_bar_or(2 + m, 128, at.lost);) {
            const Item<ROWS, BN>& p = at.item();
            const int rows = p.rows;
            const bool few = MT == 1 && rows <= 32;
            const int r = few ? lane : tid;  // row of the item
            const bool active = few ? wq < C::kParts : 32 * warp < rows;
            const int tok = min((p.j * ROWS + r) / a.group, p.seq.n - 1);
            const int open = p.open, t0 = at.t0;
            float mx = -INFINITY, sum = 0.f;
            const int t_end = p.end[m];
            // the running maximum after tile t, whose largest score is tm
            auto raise = [&](float tm, int t) {
                tm *= a.scale_log2;
                const bool grow = tm > mx + kLazy || (mx == -INFINITY && tm > mx);
                if (t == t0) {
                    mx = tm;
                } else if (__any_sync(kFull, grow)) {
                    // every product before this tile's is done; this tile's waits for us
                    products_done(g - 1);
                    const float top = grow ? tm : mx;
                    const float f = grow ? ex2(mx - top) : 1.f;  // 0 from -inf
                    mx = top;
                    sum *= f;
#pragma unroll 1
                    for (int c = 0; c < DP; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(t_o + c, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; i++) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st16(t_o + c, o);
                    }
                }
                return mx == -INFINITY ? 0.f : mx;
            };
            for (int t = t0; t < t_end; t++, g++) {
                const int sl = MT == 1 ? g & 1 : m;
                const uint32_t par = (uint32_t)(MT == 1 ? g >> 1 : g) & 1u;
                const uint32_t t_s = tmem + (uint32_t)(sl * BN) + lanes;
                attn_wait(&sfull[sl], par, w);
                tc_fence_after();
                if (active) {
                    const int k0 = t * BN;
                    const bool masked = k0 + BN > open;
                    if (few) {
                        Scores<1> s;
                        s.load(t_s + 32 * wq);
                        if (masked) s.hide(a, p, tok, k0 + 32 * wq);
                        sum += s.weigh(t_s + 16 * wq, a.scale_log2, raise(s.max(), t));
                        const uint32_t z[16] = {};  // the other warps' keys
#pragma unroll 1
                        for (int c = 0; c < BN / 32; c++)
                            if (c != wq) tmem_st16(t_s + 16 * c, z);
                    } else {
                        // 64 scores in registers at a time: the upper half's maximum, the lower half's (which
                        // stay), then their weights, which leave the upper half's scores in place, then the upper's
                        Scores<2> s;
                        float tm = -INFINITY, part = 0.f;
#pragma unroll 1
                        for (int c = BN - 64; c >= 0; c -= 64) {
                            s.load(t_s + c);
                            if (masked) s.hide(a, p, tok, k0 + c);
                            tm = fmaxf(tm, s.max());
                        }
                        const float base = raise(tm, t);
#pragma unroll 1
                        for (int c = 0; c < BN; c += 64) {
                            if (c > 0) {
                                s.load(t_s + c);
                                if (masked) s.hide(a, p, tok, k0 + c);
                            }
                            part += s.weigh(t_s + c / 2, a.scale_log2, base);
                        }
                        sum += part;
                    }
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&pfull[sl]);
            }
            const bool none = t_end == t0;  // no tile of use to this row tile
            // ------------------------------------------------ end of the part
            if (!none) products_done(g - 1);
            const bool whole = p.whole();
            // written by the producers ahead of the products
            const int odd0 = *const_cast<const volatile int*>(&p.odd0), odd1 = *const_cast<const volatile int*>(&p.odd1);
            const Split<ROWS, BN>& sp = p.split;
            float* place = nullptr;
            if (!whole) {
                attn_wait(&isplit[at.n % kItems], (uint32_t)(at.n / kItems) & 1u, w);
                place = sp.place(a, blockIdx.x);
            }
            const int D = a.head_dim;
            if (few) {
                // add up the warps' copies through shared memory: 128 elements
                // of up to 8 rows at a time, or 32 of 32
                stat_m[wq][lane] = active ? mx : -INFINITY;
                stat_l[wq][lane] = active ? sum : 0.f;
                named_bar_sync(1, 128);
                float top = -INFINITY, l = 0.f;
#pragma unroll
                for (int i = 0; i < C::kParts; i++) top = fmaxf(top, stat_m[i][lane]);
                const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int i = 0; i < C::kParts; i++) l += stat_l[i][lane] * ex2(stat_m[i][lane] - base);
                const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
                const float f = ex2(mx - base) * inv;
                const int wide = rows <= 8 ? 128 : 32, pitch = wide + 4, per = rows <= 8 ? 8 : 32;
#pragma unroll 1
                for (int c = 0; c < D; c += wide) {
                    if (active) {
#pragma unroll 1
                        for (int x = 0; x < wide && c + x < D; x += 32) {
                            uint32_t o[32];
                            tmem_ld32(t_o + c + x, o);
                            tmem_ld_wait();
                            float4* dst = reinterpret_cast<float4*>(stage + (wq * per + lane) * pitch + x);
                            if (lane < rows) {
#pragma unroll
                                for (int i = 0; i < 8; i++)
                                    dst[i] = make_float4(__uint_as_float(o[4 * i]) * f, __uint_as_float(o[4 * i + 1]) * f,
                                                         __uint_as_float(o[4 * i + 2]) * f, __uint_as_float(o[4 * i + 3]) * f);
                            }
                        }
                    }
                    named_bar_sync(1, 128);
#pragma unroll 1
                    for (int e = tid; e < rows * (wide / 8); e += 128) {
                        const int er = e / (wide / 8), ed = (e - er * (wide / 8)) * 8;
                        if (c + ed >= D) continue;
                        float o[8] = {};
#pragma unroll
                        for (int x = 0; x < C::kParts; x++)
#pragma unroll
                            for (int i = 0; i < 8; i += 4) {
                                const float4 v = *reinterpret_cast<const float4*>(stage + (x * per + er) * pitch + ed + i);
                                o[i] += v.x;
                                o[i + 1] += v.y;
                                o[i + 2] += v.z;
                                o[i + 3] += v.w;
                            }
                        if (odd0 < odd1) {
                            float t[8];
                            odd_values<8>(a, p, odd0, odd1, p.j * ROWS + er, c + ed, t);
                            for (int i = 0; i < 8; i++) o[i] += t[i];
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
                    named_bar_sync(1, 128);
                }
                if (!whole && wq == 0) {
                    place[(size_t)ROWS * D + lane] = top;
                    place[(size_t)ROWS * (D + 1) + lane] = l;
                }
            } else if (active) {
                // 32 elements of the warp's 32 rows at a time, turned through shared memory so that four lanes write
                // 64 bytes of a row (a lane a row: 5.3 us an item of 256 rows)
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                uint4* turn = reinterpret_cast<uint4*>(stage) + warp * 32 * kTurn;
                const char* mine = a.out + row_offset(a, p, p.j * ROWS + min(r, rows - 1), a.out_stride, 2);
                char* dst[4];
#pragma unroll
                for (int k = 0; k < 4; k++)
                    dst[k] = reinterpret_cast<char*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(mine), 8 * k + (lane >> 2)));
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t u[32];
                    tmem_ld32(t_o + c, u);
                    tmem_ld_wait();
                    float o[32];
#pragma unroll
                    for (int i = 0; i < 32; i++) o[i] = none ? 0.f : __uint_as_float(u[i]);
                    if (odd0 < odd1 && r < rows) {
                        float t[32];
                        odd_values<32>(a, p, odd0, odd1, p.j * ROWS + r, c, t);
#pragma unroll
                        for (int i = 0; i < 32; i++) o[i] += t[i];
                    }
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; i++) o[i] *= inv;
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; i++) turn[lane * kTurn + i] = Elem<__nv_bfloat16>::pack(o + 8 * i);
                        __syncwarp();
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            const int row = 8 * k + (lane >> 2), d = c + (lane & 3) * 8;
                            if (r - lane + row < rows && d < D)
                                *reinterpret_cast<uint4*>(dst[k] + d * 2) = turn[row * kTurn + (lane & 3)];
                        }
                    } else if (r < rows) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            if (c + i < D)
                                *reinterpret_cast<float4*>(place + part_at<ROWS>(true, D, r, (c + i) / 4)) =
                                    make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                }
                if (!whole && r < rows) {
                    place[(size_t)ROWS * D + r] = mx;
                    place[(size_t)ROWS * (D + 1) + r] = sum;
                }
            }
            tc_fence_before();
            if (!whole && !a.join_later) {
                named_bar_sync(1, 32 * C::kSoftWarps);
                // (a part whose split did not come has set lost_s before the barrier)
                if (tid == 0) last_s = !*w.lost && arrive_last(a.counters + sp.c0, (unsigned)(sp.c1 - sp.c0 + 1));
                named_bar_sync(1, 32 * C::kSoftWarps);
                if (last_s) {
                    if (few)
                        merge_few<__nv_bfloat16, ROWS, BN, 4>(a, p, sp, rows, tid, 32 * C::kSoftWarps);
                    else if (r < rows)
#pragma unroll 1
                        for (int d = 0; d < D / 4; d += 4) merge_row<__nv_bfloat16, ROWS, BN, 4, 2, true>(a, p, sp, r, d);
                }
            }
            left -= at.t1 - at.t0;
            if (left <= 0) break;
            at.next(lane, true);
        }
    }
    if (*w.lost)  // copies and products that may still be on their way: 1 ms is a hundred times what they take
        for (const uint64_t t0 = globaltimer_ns(); globaltimer_ns() - t0 < 1000000ull;) __nanosleep(10000);
    tc_fence_before();
    __syncthreads();
    if (warp == C::kWarpMma) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
}

// Joins the split items of a launch whose items mostly have many rows: block
// (c, y) the one that begins in stretch c (if any), 16 elements of 128 rows
// each.  In the attention kernel the last CTA to arrive would do it alone: 7 to
// 11 us for 128 rows of 128, against 2 to 3 us here, all SMs at once.
template <int DP, int MT>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ AttnArgs a) {
    using C = Tc<DP, MT>;
    pdl_launch_dependents();
    pdl_wait();
    const Item<C::kRows, C::BN> it = reinterpret_cast<const Item<C::kRows, C::BN>*>(a.tails)[blockIdx.x];  // a copy, in registers
    // no split item begins in this stretch: the rest of the record is of an earlier launch on the workspace
    if (it.rows == 0) return;
    const int r = 128 * (int)(blockIdx.y % MT) + (int)threadIdx.x;
    const bool few = MT == 1 && it.rows <= 32;
    if (few) {  // laid out row by row
        if (blockIdx.y == 0) merge_few<__nv_bfloat16, C::kRows, C::BN, 4>(a, it, it.split, it.rows, threadIdx.x, 128);
    } else if (r < it.rows) {
        merge_row<__nv_bfloat16, C::kRows, C::BN, 4, 4, true>(a, it, it.split, r, (int)(blockIdx.y / MT) * 4);
    }
}

// Keys or values as a 4-D tensor (element, head, offset in the page, page),
// boxes of 64 elements x `box` tokens of one head and page.
bool cache_map(CUtensorMap* map, const AttnArgs& a, const char* base) {
    auto enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.batch.page_size,
                                (cuuint64_t)a.batch.n_pages};
    // a dimension of one entry may carry any stride, 0 too; it is never stepped over
    const long long steps[3] = {a.cache.head_stride, a.cache.token_stride, a.cache.page_stride};
    cuuint64_t strides[3];
    for (int i = 0; i < 3; i++) strides[i] = dims[i + 1] == 1 && steps[i] < 16 ? 16 : (cuuint64_t)steps[i];
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)a.box, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<char*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// q as a 3-D tensor (element, head, token), boxes of 64 elements x 32 rows of
// one key head's group, token-major.
bool query_map(CUtensorMap* map, const AttnArgs& a) {
    auto enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.n_kv_heads * a.group, (cuuint64_t)a.batch.n_tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)a.head_dim * 2, (cuuint64_t)a.q_stride};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)(32 / a.group)};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<char*>(a.q), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP, int MT>
cudaError_t go(AttnArgs a, bool join_later, int sms, cudaStream_t st) {
    using C = Tc<DP, MT>;
    auto* kern = attn_tc_kernel<DP, MT>;
    static std::atomic<bool> allowed[64];
    cudaError_t e = allow_smem(kern, C::kSmem, allowed);
    if (e != cudaSuccess) return e;
    // TMA boxes where pages and key tiles divide one another and a box fills
    // whole 8-row swizzle atoms; else 16-byte cp.async, for any page
    const int ps = a.batch.page_size;
    a.box = ps >= 8 && (C::BN % ps == 0 || ps % C::BN == 0) ? (ps < C::BN ? ps : C::BN) : 0;
    CUtensorMap mk{}, mv{}, mq{};
    if (a.box && (!cache_map(&mk, a, a.cache.k) || !cache_map(&mv, a, a.cache.v))) a.box = 0;
    // rows of q: 32 of one key head are whole tokens where the group divides 32
    a.q_box = 32 % a.group == 0 && query_map(&mq, a);
    a.join_later = join_later;
    static_assert(sizeof(Item<C::kRows, C::BN>) <= kAttnTail, "a stretch's last item in the workspace");
    const unsigned grid = (unsigned)(sms < kAttnTcGrid ? sms : kAttnTcGrid);
    e = launch_overlapped(kern, dim3(grid), dim3(C::kWarps * 32), C::kSmem, st, a, mk, mv, mq);
    if (e != cudaSuccess || !join_later) return e;
    return launch_overlapped(join_kernel<DP, MT>, dim3(grid, (unsigned)(MT * ((a.head_dim + 15) / 16))), dim3(128), 0, st, a);
}

}  // namespace

cudaError_t attn_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // Rows a sequence brings to a key head on average (the host knows no
    // lengths; padding tokens and empty sequences count): two row tiles share
    // each key tile where one does not hold them.  One / two, 32 heads on 8 of
    // 128: 8 trees of 32 tokens (128 rows) 35 / 40 us, of 36 (144 rows) 53 / 44,
    // of 64 58 / 49; 4 prompts of 160 tokens, 40 heads, 31 / 26.  An average
    // says little of mixed lengths: a prompt of 2048 tokens beside 7 single
    // tokens over 64 to 8191 entries (1027) 111 / 98, beside 31 (259) 176 / 190,
    // beside 63 (131) 252 / 301, beside 127 (67) 415 / 518: from 129 to about 300
    // such a batch is up to a fifth slower than it could be.
    const long long rows = ((long long)a.batch.n_tokens * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
    const bool two = rows > 128;
    // Split items of a few rows are joined by the CTA that finishes last, those of many by a second kernel (8 trees of
    // 8 tokens, 32 rows: 40 us against 41; of 9, 36 rows: 48 against 32; one of 12 over 4000 entries: 56 against 16).
    const bool later = rows > 32;
    if (a.head_dim <= 64) return two ? go<64, 2>(a, later, sms, st) : go<64, 1>(a, later, sms, st);
    if (a.head_dim <= 128) return two ? go<128, 2>(a, later, sms, st) : go<128, 1>(a, later, sms, st);
    return go<256, 1>(a, later, sms, st);
}

}  // namespace pp
