// Attention over the paged cache on the CUDA cores: the fp32 path, fp32
// throughout.  One CTA streams its stretch of the key line (pp_attn_sched.cuh)
// tile by tile: TOK keys and values into shared memory (cp.async, entries past
// the sequence as zeros), scores, the running maximum and weight sum of each
// row, weighted values into registers.
//
// Register tiles are 4 rows x 1 key (scores, the head dimension split over
// the threads that a small row tile leaves free) and 4 rows x 4 elements
// (values, the keys split likewise); the splits are joined through shared
// memory.  Up to four CTAs per SM overlap the loads of one with the arithmetic
// of the others.  3 drafted trees of 9 to 13 tokens over 100 to 1000 entries,
// 16 heads of 64: 19 us, a chain of latencies (16 MB, 2.4 us of HBM); for
// many rows the score loop's shared-memory loads bound it.
#include "pp_attn_sched.cuh"
#include "pp_launch.cuh"
#include "pp_tc.cuh"

namespace pp {
namespace {

constexpr int kThreads = 256;
// A stretch's key tiles.  A tile takes 2 to 4 us and every further part of an
// item a join, and stretches that do not divide the items' tiles cut more of
// them, so no number is best everywhere.  1 / 2 / 3 tiles, 16 heads of 64: one
// token over 400 entries 10.0 / 12.4 / 14.3 us, 3 tokens over 400 16.2 / 13.6 /
// 15.5, 3 over 1000 21.7 / 21.6 / 17.5; 13 tokens over 400 12.1 / 16.3 / 18.9, 3
// times 13 over 400 20.5 / 18.2 / 21.0, over 1000 31.2 / 30.8 / 24.1, 3 trees of 9
// to 13 over 100 to 1000 23.3 / 19.2 / 23.6; alike from about 4000 entries on.
constexpr int kLeastTiles = 2;

// Rows of a tile, keys of a tile, padded head dimension.
template <int ROWS, int TOK, int DP>
struct Simt {
    static constexpr int kRG = ROWS / 4;                        // groups of 4 rows
    static constexpr int kScoreCols = TOK * kRG;                 // (row group, key) pairs
    static constexpr int kDSplit = kThreads / kScoreCols;        // head-dimension split of the scores
    static constexpr int kD4 = DP / 4;
    static constexpr int kTSplit = kThreads / (kD4 * kRG);       // key split of the values
    static constexpr int kKStride = DP + 4;
    static_assert(kDSplit >= 1 && kTSplit >= 1 && kRG >= 1, "thread layout");
    static constexpr int kQ = 0;
    static constexpr int kK = kQ + ROWS * DP;
    static constexpr int kV = kK + TOK * kKStride;
    static constexpr int kS = kV + TOK * DP;                     // partial scores [kDSplit][ROWS][TOK]
    static constexpr int kP = kS + kDSplit * ROWS * TOK;         // weights [TOK][ROWS]
    static constexpr int kStat = kP + TOK * ROWS;                // max, sum, factor [ROWS] each
    static constexpr int kFloats = kStat + 3 * ROWS;
    static_assert((kTSplit - 1) * ROWS * DP <= TOK * (kKStride + DP), "joining area");
};

template <int ROWS, int TOK, int DP>
__global__ void __launch_bounds__(kThreads) attn_simt_kernel(const __grid_constant__ AttnArgs a) {
    using L = Simt<ROWS, TOK, DP>;
    extern __shared__ __align__(16) float sm[];
    __shared__ unsigned last_s;
    float *Qs = sm + L::kQ, *Ks = sm + L::kK, *Vs = sm + L::kV, *Ss = sm + L::kS, *Ps = sm + L::kP;
    float *Mx = sm + L::kStat, *Sum = Mx + ROWS, *Fac = Sum + ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    Walk<ROWS, TOK> walk = start_walk<ROWS, TOK>(&a, lane, blockIdx.x == 0 && warp == 0, kLeastTiles);
    const int D = a.head_dim;
    // score threads: key, row group, part of the head dimension
    const int s_key = tid % TOK, s_rg = tid / TOK % L::kRG, s_ds = tid / L::kScoreCols;
    // value threads: 4 elements, row group, part of the keys
    const int v_d = tid % L::kD4 * 4, v_rg = tid / L::kD4 % L::kRG, v_ts = tid / (L::kD4 * L::kRG);
    Part p;
    while (walk.next(p)) {
        const int rows = min(ROWS, p.seq.n * a.group - p.j * ROWS);
        __syncthreads();  // the last part's readers are done
        for (int e = tid; e < ROWS * (DP / 4); e += kThreads) {
            const int r = e / (DP / 4), d = e % (DP / 4) * 4;
            const bool in = r < rows && d < D;
            cp_async_16(Qs + r * DP + d, in ? a.q + row_offset(a, p, p.j * ROWS + r, a.q_stride, 4) + d * 4 : a.q, in ? 16u : 0u);
        }
        if (tid < ROWS) {
            Mx[tid] = -INFINITY;
            Sum[tid] = 0.f;
        }
        float o[4][4] = {};
        for (int t = p.t0; t < p.t1; t++) {
            const int k0 = t * TOK;
            __syncthreads();  // the last tile's readers are done (first tile: rows are in place)
            for (int e = tid; e < TOK * (DP / 4); e += kThreads) {
                const int r = e / (DP / 4), d = e % (DP / 4) * 4, j = k0 + r;
                long long at = 0;
                bool in = j < p.key_end && d < D;
                if (in) {
                    const int page = entry_page(a.batch, p.b, j);
                    if (page >= 0) {
                        at = entry_offset(a.batch, a.cache, page, j) + (long long)p.h * a.cache.head_stride + d * 4;
                    } else {
                        record_status(a.status, PP_ERR_INVALID_ARG);
                        in = false;
                    }
                }
                cp_async_16(Ks + r * L::kKStride + d, a.cache.k + at, in ? 16u : 0u);
                cp_async_16(Vs + r * DP + d, a.cache.v + at, in ? 16u : 0u);
            }
            cp_async_commit();
            cp_async_wait<0>();
            __syncthreads();
            if (s_ds < L::kDSplit) {
                float acc[4] = {};
                constexpr int kPart = DP / L::kDSplit;
                const float* kr = Ks + s_key * L::kKStride + s_ds * kPart;
                const float* qr = Qs + s_rg * 4 * DP + s_ds * kPart;
#pragma unroll 8
                for (int d = 0; d < kPart; d += 4) {
                    const float4 kv = *reinterpret_cast<const float4*>(kr + d);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float4 qv = *reinterpret_cast<const float4*>(qr + i * DP + d);
                        acc[i] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, acc[i]))));
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; i++) Ss[(s_ds * ROWS + s_rg * 4 + i) * TOK + s_key] = acc[i];
            }
            __syncthreads();
            // running maximum and weights, one warp a row
            for (int r = warp; r < ROWS; r += kThreads / 32) {
                const int row = p.j * ROWS + r, tok = row / a.group;
                float s[TOK / 32];
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < TOK / 32; i++) {
                    const int c = i * 32 + lane, j = k0 + c - p.seq.ctx;  // new token's number when >= 0
                    bool see = r < rows && k0 + c < p.key_end;
                    if (see && j >= 0)
                        see = a.mask ? j < 32 * a.mask_words &&
                                           (a.mask[(size_t)(p.seq.q0 + tok) * a.mask_words + (j >> 5)] >> (j & 31) & 1u)
                                     : j <= tok;
                    s[i] = 0.f;
#pragma unroll
                    for (int x = 0; x < L::kDSplit; x++) s[i] += Ss[(x * ROWS + r) * TOK + c];
                    s[i] = see ? s[i] * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, s[i]);
                }
                const float m_old = Mx[r], m_new = fmaxf(m_old, warp_max(mx));
                const float m = m_new == -INFINITY ? 0.f : m_new;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < TOK / 32; i++) {
                    const float w = exp2f(s[i] - m);
                    Ps[(i * 32 + lane) * ROWS + r] = w;
                    sum += w;
                }
                sum = warp_sum(sum);
                if (lane == 0) {
                    const float f = exp2f(m_old - m);
                    Mx[r] = m_new;
                    Fac[r] = f;
                    Sum[r] = Sum[r] * f + sum;
                }
                __syncwarp();
            }
            __syncthreads();
            if (v_ts < L::kTSplit) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float f = Fac[v_rg * 4 + i];
#pragma unroll
                    for (int x = 0; x < 4; x++) o[i][x] *= f;
                }
                // past the cached tokens a weight of zero may stand for an unseen
                // entry, whose values (NaN, say) must not reach the sum
                const bool strict = k0 + TOK > p.seq.ctx;
#pragma unroll 4
                for (int c = v_ts; c < TOK; c += L::kTSplit) {
                    const float4 v = *reinterpret_cast<const float4*>(Vs + c * DP + v_d);
                    const float4 w4 = *reinterpret_cast<const float4*>(Ps + c * ROWS + v_rg * 4);
                    const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        if (strict && w[i] == 0.f) continue;
                        o[i][0] = fmaf(w[i], v.x, o[i][0]);
                        o[i][1] = fmaf(w[i], v.y, o[i][1]);
                        o[i][2] = fmaf(w[i], v.z, o[i][2]);
                        o[i][3] = fmaf(w[i], v.w, o[i][3]);
                    }
                }
            }
        }
        // join the key splits in the key and value area
        if (L::kTSplit > 1) {
            __syncthreads();
            float* J = Ks;
            if (v_ts > 0 && v_ts < L::kTSplit) {
#pragma unroll
                for (int i = 0; i < 4; i++)
                    *reinterpret_cast<float4*>(J + ((v_ts - 1) * ROWS + v_rg * 4 + i) * DP + v_d) =
                        make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
            }
            __syncthreads();
            if (v_ts == 0) {
#pragma unroll
                for (int x = 0; x < L::kTSplit - 1; x++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float4 v = *reinterpret_cast<const float4*>(J + (x * ROWS + v_rg * 4 + i) * DP + v_d);
                        o[i][0] += v.x;
                        o[i][1] += v.y;
                        o[i][2] += v.z;
                        o[i][3] += v.w;
                    }
            }
        }
        if (p.whole()) {
            if (v_ts == 0 && v_d < D) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int r = v_rg * 4 + i;
                    if (r >= rows) break;
                    const float l = Sum[r], inv = l == 0.f ? 0.f : 1.f / l;
                    char* dst = a.out + row_offset(a, p, p.j * ROWS + r, a.out_stride, 4) + v_d * 4;
                    store4<float>(dst, make_float4(o[i][0], o[i][1], o[i][2], o[i][3]), inv);
                }
            }
            continue;
        }
        const Split<ROWS, TOK> sp(walk.sched, p);
        float* pl = sp.place(a, blockIdx.x);
        if (v_ts == 0 && v_d < D) {
#pragma unroll
            for (int i = 0; i < 4; i++)
                *reinterpret_cast<float4*>(pl + (size_t)(v_rg * 4 + i) * D + v_d) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
        }
        if (tid < ROWS) {
            pl[(size_t)ROWS * D + tid] = Mx[tid];
            pl[(size_t)ROWS * (D + 1) + tid] = Sum[tid];
        }
        __syncthreads();
        if (tid == 0) last_s = arrive_last(a.counters + sp.c0, (unsigned)(sp.c1 - sp.c0 + 1));
        __syncthreads();
        if (last_s) merge_few<float, ROWS, TOK, 1>(a, p, sp, rows, tid, kThreads);
    }
}

template <int ROWS, int TOK, int DP>
cudaError_t go(const AttnArgs& a, int sms, cudaStream_t st) {
    using L = Simt<ROWS, TOK, DP>;
    auto* kern = attn_simt_kernel<ROWS, TOK, DP>;
    constexpr int kBytes = L::kFloats * 4;
    static std::atomic<bool> allowed[64];
    cudaError_t e = allow_smem(kern, kBytes, allowed);
    if (e != cudaSuccess) return e;
    const int per_sm = 227 * 1024 / (kBytes + 2048);
    int grid = sms * (per_sm < 1 ? 1 : per_sm > 4 ? 4 : per_sm);
    if (grid > kAttnMaxGrid) grid = kAttnMaxGrid;
    return launch_overlapped(kern, dim3((unsigned)grid), dim3(kThreads), kBytes, st, a);
}

}  // namespace

size_t attn_part_floats(int head_dim) {
    const size_t simt = (size_t)kAttnMaxGrid * kAttnSimtRows, tc = (size_t)kAttnTcGrid * kAttnTcRows;
    return 2 * (simt > tc ? simt : tc) * (head_dim + 2);
}

cudaError_t attn_simt_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // rows a sequence brings to a key head on average: small tiles spread
    // their threads over keys and elements instead of rows that do not exist
    // (tiles of 16 / 4 rows, 3 sequences over 100 to 1000 entries: 4 rows 19.2 /
    // 14.9 us for 16 heads of 64, 44.0 / 36.9 for 32 of 128; 5 rows 19.0 / 23.5,
    // 44.0 / 49.5)
    const long long rows = ((long long)a.batch.n_tokens * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
    const bool few = rows <= 4;
    if (a.head_dim <= 64) return few ? go<4, 64, 64>(a, sms, st) : go<16, 64, 64>(a, sms, st);
    if (a.head_dim <= 128) return few ? go<4, 64, 128>(a, sms, st) : go<16, 64, 128>(a, sms, st);
    return few ? go<4, 64, 256>(a, sms, st) : go<16, 64, 256>(a, sms, st);
}

}  // namespace pp
