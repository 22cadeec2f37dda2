// The paged key/value cache in 8 bits: append, entries read back, and the
// commit of a drafted tree's accepted path.  All move bytes and compute little,
// so HBM bounds them (and launch latency, for a few tokens).
#include <algorithm>

#include <cuda_fp16.h>

#include "pp_cache8.cuh"
#include "pp_head.cuh"
#include "pp_launch.cuh"
#include "pp_tc.cuh"

namespace pp {
namespace {

// ------------------------------------------------------------------- append
// Two kinds of CTAs in one launch.  The first slots * parts take the keys and
// values: a slot is a block of one sequence's entries, dealt without the host
// knowing a length: sequence b's slots start at q_start[b] / block + 2 b, which
// leaves it the (n - 1) / block + 2 blocks that n new entries can touch.  A
// strip of R rows of one head's keys or values is held by one warp, in
// registers: its largest magnitude is known before anything is written, and
// every element is read once.  The strips of a longer block meet in shared
// memory.  The other CTAs take a token's query heads, as in norm_kernel.  8192
// tokens of 40 + 40 + 40 heads of 128, bf16, blocks of 64, normed (399 MB): 108 us,
// 3.7 TB/s (0.55 of the copy rate); the keys and values are most of it, of which 16
// warps an SM keep too little on its way.  Blocks of 16: 100 us, of 128: 176;
// without norms 88; fp32 (719 MB) 256.  64 single tokens: 5.4 us, a chain of
// latencies.
constexpr int kMaxStrips = 16;  // warps of a CTA at most (8 where that does)
constexpr int kAppend8Smem = 216 * 1024;

struct Slot {
    int page, lo;      // the block's page and first entry; page -1: nothing to do
    int e0, e1;        // its new entries
    int token;         // of entry e0
    int ctx;
};

// By one warp.
PP_DEVINL Slot find_slot(const BatchArgs& B, int shift, int slot, int lane, unsigned* status) {
    int lo = 0, hi = B.n_seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int i = at < hi ? at : lo;
        const unsigned le = __ballot_sync(kFull, at < hi && (long long)(B.q_start[i] >> shift) + 2ll * i <= slot);
        const int c = __popc(le);
        if (c == 0) break;
        lo += (c - 1) * step;
        hi = min(hi, lo + step);
    }
    Slot s{-1, 0, 0, 0, 0, 0};
    const Seq q = load_seq(B, lo);
    const long long j = (long long)slot - (q.q0 >> shift) - 2ll * lo;
    if (q.bad || q.n == 0 || j < 0 || j > (q.n >> shift) + 1) return s;
    const long long first = (((long long)q.ctx >> shift) + j) << shift;
    if (first >= (long long)q.ctx + q.n) return s;
    s.lo = (int)first;
    s.ctx = q.ctx;
    s.e0 = max(s.lo, q.ctx);
    s.e1 = (int)min(first + (1 << shift), (long long)q.ctx + q.n);
    s.token = q.q0 + s.e0 - q.ctx;
    s.page = entry_page(B, lo, s.lo);
    if (s.page < 0 && lane == 0) record_status(status, PP_ERR_INVALID_ARG);
    return s;
}

// Finite values (or NaN) times inv as codes.
template <int V>
PP_DEVINL void store_codes(char* p, const F2 (&f)[V / 2], float inv) {
    uint32_t w[V > 4 ? V / 4 : 1] = {};
    const F2 inv2 = pair2(inv, inv);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        float a, b;
        unpair2(mul2(f[i / 2], inv2), a, b);
        w[i / 4] |= to_codes(a, b) << (i % 4 * 8);
    }
    if constexpr (V == 8)
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V == 4)
        *reinterpret_cast<uint32_t*>(p) = w[0];
    else
        *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
}
// V codes at p rounded again at the scale `now`.
template <int V>
PP_DEVINL void again(char* p, float ratio, float now) {
    const float top = top_code(now);
    F2 f[V / 2];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float2 v = from_codes(*reinterpret_cast<const uint16_t*>(p + i));
        f[i / 2] = pair2(within(v.x * ratio, top), within(v.y * ratio, top));
    }
    store_codes<V>(p, f, 1.f);
}

template <typename T, int V, bool HALF, int UPL, int ITER, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, WARPS == 8 ? 2 : 1) append8_kernel(const Append8Args a) {
    using Lane = HeadLane<T, V, HALF, UPL>;
    extern __shared__ __align__(16) float cs[];
    __shared__ Slot slot_s;
    __shared__ int pos_s[kMaxStrips], in_s[kMaxStrips];
    __shared__ float amax_s[2][kMaxStrips];
    pdl_launch_dependents();
    pdl_wait();
    const HeadArgs& h = a.head;
    const int tid = threadIdx.x, warp = tid >> 5, l32 = tid & 31, D = h.head_dim;
    const Lane lane(h, l32 % h.group);
    const int kv_ctas = a.slots * a.parts;
    if ((int)blockIdx.x >= kv_ctas) {
        // ------------------------------------------------------------ queries
        // a team of a.team threads takes a token; with one team a CTA, a.split CTAs share a token
        const int q_cta = (int)blockIdx.x - kv_ctas, team = tid / a.team, teams = (int)blockDim.x / a.team;
        const int t = q_cta / a.split * teams + team, y = q_cta % a.split, in_team = tid - team * a.team;
        const int groups = a.team / h.group, step = groups * a.split;
        const bool exists = t < a.batch.n_tokens;
        const char* q = a.q + t * a.q_stride;
        char* out = a.q_out + t * a.q_out_stride;
        const int pitch = (h.rot_dim / 2 + V - 1) / V;
        float* table = cs + team * (pitch * V * 2);
        if (in_team < 32 && exists) {
            const int b = find_seq(a.batch, t, l32);
            const Seq s = load_seq(a.batch, b);
            const int i = t - s.q0;
            const bool in = !s.bad && i >= 0 && i < s.n;
            if (l32 == 0) {
                pos_s[team] = h.positions ? h.positions[t] : s.ctx + i;
                in_s[team] = in;
            }
        }
        typename Lane::Factors c;
        bool ready = false, in = false;
        for (int r0 = y * groups; r0 < a.n_heads; r0 += 2 * step) {
            Vec<T, V> x[2][UPL][2];
#pragma unroll
            for (int n = 0; n < 2; n++) {
                const int r = r0 + n * step + in_team / h.group;
                if (r < a.n_heads && exists) lane.load(q + (long long)r * D * (int)sizeof(T), x[n]);
            }
            if (!ready) {
                __syncthreads();
                in = exists && in_s[team];  // padding, or a skipped sequence: nothing is written
                if (h.rot_dim > 0) {
                    if (in) fill_pairs(table, h, V, pos_s[team], in_team, a.team);
                    __syncthreads();
                    lane.factors(table, h, c);
                }
                ready = true;
            }
#pragma unroll
            for (int n = 0; n < 2; n++) {
                const int r = r0 + n * step + in_team / h.group;
                F2 f[UPL][2][V / 2], g[UPL][2][V / 2];
                Lane::widen(x[n], f);
                if (h.norm) {
                    const float inv = inverse_rms(Lane::group_sum(r < a.n_heads && exists ? Lane::dot(f, f) : 0.f, h.group), h);
                    lane.weights(a.q_gamma, g);
                    Lane::scale_by(f, inv, g);
                }
                if (r >= a.n_heads || !in) continue;
                if (h.rot_dim > 0) lane.rotate(f, c);
                if (h.norm || h.rot_dim > 0) Lane::narrow(f, x[n]);
                lane.store(out + (long long)r * D * (int)sizeof(T), x[n]);
            }
        }
        return;
    }
    // --------------------------------------------------------- keys and values
    const int slot = (int)blockIdx.x / a.parts, part = (int)blockIdx.x % a.parts, block = 1 << a.scales.shift;
    if (warp == 0) {
        const Slot s = find_slot(a.batch, a.scales.shift, slot, l32, a.status);
        if (l32 == 0) slot_s = s;
    } else if (tid == 32 && part == 0) {
        // every sequence is looked at once, also one that no token belongs to
        for (int b = slot; b < a.batch.n_seqs; b += a.slots)
            if (load_seq(a.batch, b).bad) record_status(a.status, PP_ERR_INVALID_ARG);
    }
    __syncthreads();
    const Slot s = slot_s;
    if (s.page < 0) return;
    const int per = 32 / h.group, R = ITER * per;  // rows of a warp at once, of a strip
    const int strips = max(1, block / R), units = (int)blockDim.x / 32 / strips;
    const int strip = warp % strips;
    const int pitch = (h.rot_dim / 2 + V - 1) / V, row_pairs = pitch * V;  // factors of a row
    // a part takes units side by side, so that most have keys only or values only
    const int u_first = part * a.passes * units, u_end = min(2 * a.n_kv_heads, u_first + a.passes * units);
    const int factors = u_first < a.n_kv_heads ? (s.e1 - s.e0) * (h.rot_dim / 2) : 0;  // values need none
    for (int i = tid; i < factors; i += blockDim.x) {
        const int row = i / (h.rot_dim / 2), p = i - row * (h.rot_dim / 2), t = s.token + row;
        const float2 v = cos_sin(h.positions ? h.positions[t] : s.e0 + row, h.inv_freq[p]);
        put_pair(cs + (s.e0 - s.lo + row) * row_pairs * 2, p, V, pitch, make_float2(v.x * h.scale, v.y * h.scale));
    }
    // A thread's vectors of the next units on their way into shared memory, for itself alone: loads in registers would
    // leave too few of them in flight (8192 tokens, 40 heads of 128: 199 us).
    constexpr int kVecs = ITER * UPL * 2;
    unsigned char* stages = reinterpret_cast<unsigned char*>(cs) + a.table_bytes + tid * Lane::kBytes;
    const int stage_bytes = kVecs * (int)blockDim.x * Lane::kBytes;
    const int first = s.lo + strip * R + l32 / h.group;  // entry of the lane's first row
    uint32_t rows = 0;                                   // which of the lane's rows are new entries
#pragma unroll
    for (int n = 0; n < ITER; n++)
        if (first + n * per >= s.e0 && first + n * per < s.e1) rows |= 1u << n;
    const int vec_step = (int)blockDim.x * Lane::kBytes;
    // the lane's first row of unit u (row 0 may lie ahead of the tensor: only new entries' are read)
    auto row0_of = [&](int u, long long& step) {
        const bool key = u < a.n_kv_heads;
        const long long stride = key ? a.k_stride : a.v_stride;
        step = per * stride;
        return (key ? a.k : a.v) + (long long)(s.token + first - s.e0) * stride + (long long)(key ? u : u - a.n_kv_heads) * D * (int)sizeof(T);
    };
    auto fetch = [&](int u0, int stage) {
        const int u = u0 + warp / strips;
        if (u < u_end) {
            long long step;
            const char* row = row0_of(u, step);
            unsigned char* to = stages + stage * stage_bytes;
#pragma unroll
            for (int n = 0; n < ITER; n++, row += step)
#pragma unroll
                for (int k = 0; k < UPL; k++) {
                    unsigned char* at = to + (n * UPL + k) * 2 * vec_step;
                    if ((rows >> n & 1u) && lane.va[k] >= 0) cp_async_small<Lane::kBytes>(at, row + lane.va[k] * Lane::kBytes);
                    if ((rows >> n & 1u) && lane.vb[k] >= 0) cp_async_small<Lane::kBytes>(at + vec_step, row + lane.vb[k] * Lane::kBytes);
                }
        }
        cp_async_commit();
    };
    int turn = 0, pass = 0;
    const bool cached = s.lo < s.ctx;
    const long long dst0 = entry_offset(a.batch, a.cache, s.page, s.lo) + (first - s.lo) * a.cache.token_stride,
                    scale0 = scale_index(a.batch, a.scales, a.n_kv_heads, s.page, 0, s.lo);
    for (int i = 0; i + 1 < a.stages; i++) fetch(u_first + i * units, i);
    __syncthreads();
    for (int u0 = u_first; u0 < u_end; u0 += units, pass ^= 1) {
        const int u = u0 + warp / strips;
        const bool have = u < u_end, key = u < a.n_kv_heads;
        const int head = key ? u : u - a.n_kv_heads;
        float* scale_p = (key ? a.scales.k : a.scales.v) + scale0 + (long long)head * a.scales.blocks;
        float old = have && cached && l32 == 0 ? *scale_p : 0.f;
        F2 f[ITER][UPL][2][V / 2];
        if (a.stages) {
            fetch(u0 + (a.stages - 1) * units, (turn + a.stages - 1) % a.stages);
            if (a.stages == 1)
                cp_async_wait<0>();
            else  // two at most
                cp_async_wait<1>();
        }
        const unsigned char* from = stages + turn * stage_bytes;
        turn = turn + 1 >= a.stages ? 0 : turn + 1;
        float amax = 0.f;
        if (have) {
            long long step;
            const char* row = row0_of(u, step);
#pragma unroll
            for (int n = 0; n < ITER; n++, row += step) {
                Vec<T, V> x[UPL][2] = {};
                if (a.stages)
                    lane.load_own(from + n * UPL * 2 * vec_step, vec_step, rows >> n & 1u, x);
                else if (rows >> n & 1u)  // no room beside the factors
                    lane.load(row, x);
                Lane::widen(x, f[n]);
            }
            if (key && h.norm) {
                F2 g[UPL][2][V / 2];
                lane.weights(a.k_gamma, g);
#pragma unroll
                for (int n = 0; n < ITER; n++) {
                    const float inv = inverse_rms(Lane::group_sum(Lane::dot(f[n], f[n]), h.group), h);
                    if (rows >> n & 1u) Lane::scale_by(f[n], inv, g);  // (zeros may have no root mean square)
                }
            }
            if (key && h.rot_dim > 0) {
#pragma unroll
                for (int n = 0; n < ITER; n++) {
                    if (!(rows >> n & 1u)) continue;
                    typename Lane::Factors c;
                    lane.factors(cs + (first + n * per - s.lo) * row_pairs * 2, h, c);
                    lane.rotate(f[n], c);
                }
            }
            // 0 x summed is zero for finite values alone
            F2 zero = 0ull;
#pragma unroll
            for (int n = 0; n < ITER; n++)
#pragma unroll
                for (int k = 0; k < UPL; k++)
#pragma unroll
                    for (int v = 0; v < 2; v++)
#pragma unroll
                        for (int i = 0; i < V / 2; i++) {
                            float x, y;
                            unpair2(f[n][k][v][i], x, y);
                            amax = fmaxf(amax, fmaxf(fabsf(x), fabsf(y)));
                            zero = fma2(f[n][k][v][i], 0ull, zero);
                        }
            float zx, zy;
            unpair2(zero, zx, zy);
            if (__any_sync(kFull, zx != 0.f || zy != 0.f)) {
                // what is not finite does not count, and is held as NaN
                amax = 0.f;
#pragma unroll
                for (int n = 0; n < ITER; n++)
#pragma unroll
                    for (int k = 0; k < UPL; k++)
#pragma unroll
                        for (int v = 0; v < 2; v++)
#pragma unroll
                            for (int i = 0; i < V / 2; i++) {
                                float x, y;
                                unpair2(f[n][k][v][i], x, y);
                                amax = fmaxf(amax, fmaxf(magnitude(x), magnitude(y)));
                                f[n][k][v][i] = pair2(to_hold(x), to_hold(y));
                            }
            }
            amax = warp_max(amax);
            old = __shfl_sync(kFull, old, 0);
        }
        if (strips > 1) {  // the block's largest magnitude, from all its strips (in turns: one barrier a pass)
            if (l32 == 0) amax_s[pass][warp] = amax;
            __syncthreads();
            for (int i = 0; i < strips; i++) amax = fmaxf(amax, amax_s[pass][warp - strip + i]);
        }
        if (!have) continue;
        const float now = block_scale(amax, old, cached);
        char* dst = (key ? a.cache.k : a.cache.v) + dst0 + (long long)head * a.cache.head_stride;
        if (cached && now != old) {
            char* row = dst;
#pragma unroll 1
            for (int e = first; e < min(s.ctx, s.lo + strip * R + R); e += per, row += per * a.cache.token_stride) {
#pragma unroll
                for (int k = 0; k < UPL; k++) {
                    if (lane.va[k] >= 0) again<V>(row + lane.va[k] * V, old / now, now);
                    if (lane.vb[k] >= 0) again<V>(row + lane.vb[k] * V, old / now, now);
                }
            }
        }
        const float inv = 1.0f / now;
        if (now >= kLargeScale) {  // what is finite stays so
            const float top = top_code(now) * now;
#pragma unroll
            for (int n = 0; n < ITER; n++)
#pragma unroll
                for (int k = 0; k < UPL; k++)
#pragma unroll
                    for (int v = 0; v < 2; v++)
#pragma unroll
                        for (int i = 0; i < V / 2; i++) {
                            float x, y;
                            unpair2(f[n][k][v][i], x, y);
                            f[n][k][v][i] = pair2(within(x, top), within(y, top));
                        }
        }
#pragma unroll
        for (int n = 0; n < ITER; n++, dst += per * a.cache.token_stride) {
            if (!(rows >> n & 1u)) continue;
#pragma unroll
            for (int k = 0; k < UPL; k++) {
                if (lane.va[k] >= 0) store_codes<V>(dst + lane.va[k] * V, f[n][k][0], inv);
                if (lane.vb[k] >= 0) store_codes<V>(dst + lane.vb[k] * V, f[n][k][1], inv);
            }
        }
        if (l32 == 0 && strip == 0 && now != old) *scale_p = now;
    }
}

template <typename T, int V, bool HALF, int UPL, int ITER, int WARPS>
cudaError_t append8_run(Append8Args& a, int block, cudaStream_t st) {
    constexpr int warps = WARPS;
    const int R = ITER * 32 / a.head.group, strips = std::max(1, block / R);
    if constexpr (WARPS == 8) {
        if (strips > 8) return append8_run<T, V, HALF, UPL, ITER, 16>(a, block, st);
    }
    const int units = warps / strips, passes = (2 * a.n_kv_heads + units - 1) / units;
    const long long T_ = a.batch.n_tokens;
    a.slots = (int)(T_ / block + 2ll * a.batch.n_seqs);
    // a pass of all heads a CTA where there are few blocks; else about two CTAs an SM (8192 tokens: two / four / eight, 107 /
    // 110 / 119 us)
    a.parts = std::min(passes, std::max(1, (304 + a.slots - 1) / a.slots));
    a.passes = (passes + a.parts - 1) / a.parts;
    a.parts = (passes + a.passes - 1) / a.passes;
    const int threads = warps * 32, pairs = (a.head.rot_dim / 2 + V - 1) / V * V;
    // queries: ten rows' lanes a thread where there are many tokens; few tokens: several CTAs each
    const int rows = threads / a.head.group;  // query rows of a CTA at once
    a.split = a.n_heads ? (int)std::min<long long>((a.n_heads + rows - 1) / rows, std::max<long long>(1, 304 / T_)) : 1;
    a.team = threads;
    if (a.split == 1 && T_ > 608)
        while (a.team > 64 && a.team / 2 * 10 >= a.n_heads * a.head.group) a.team /= 2;
    const int teams = threads / a.team;
    const long long ctas = (long long)a.slots * a.parts + (a.n_heads ? (T_ + teams - 1) / teams * a.split : 0);
    if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
    a.table_bytes = std::max(block, teams) * pairs * 8;
    const int stage = ITER * UPL * 2 * threads * V * (int)sizeof(T);
    // two CTAs an SM where that leaves two stages, else as many as fit
    a.stages = (kAppend8Smem / 2 - a.table_bytes) / stage;
    if (a.stages < 2) a.stages = (kAppend8Smem - a.table_bytes) / stage;
    a.stages = std::max(0, std::min({a.stages, 2, a.passes}));
    const int smem = a.table_bytes + a.stages * stage;
    auto* kern = append8_kernel<T, V, HALF, UPL, ITER, WARPS>;
    static std::atomic<bool> allowed[64];
    const cudaError_t e = allow_smem(kern, kAppend8Smem, allowed);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kern, dim3((unsigned)ctas), dim3((unsigned)threads), (size_t)smem, st, a);
}

template <typename T, int V, bool HALF>
cudaError_t append8_go(Append8Args a, int block, cudaStream_t st) {
    const int units = head_units<V>(a.head);
    int group = 4;
    while (group < 32 && group < units) group *= 2;
    a.head.group = group;
    // strips of up to 64 fp32 values a lane
    if constexpr (V == 2) {
        if (units > 32) return append8_run<T, V, HALF, 2, 8, 8>(a, block, st);
        return append8_run<T, V, HALF, 1, 8, 8>(a, block, st);
    } else if constexpr (V == 4) {
        return group <= 8 ? append8_run<T, V, HALF, 1, 4, 8>(a, block, st) : append8_run<T, V, HALF, 1, 8, 8>(a, block, st);
    } else {
        return append8_run<T, V, HALF, 1, 4, 8>(a, block, st);
    }
}

template <typename T>
cudaError_t append8_typed(const Append8Args& a, int layout, int block, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool half = layout == PP_ROPE_HALF;
    const bool whole = half ? a.head.rot_dim % (2 * V) == 0 : a.head.rot_dim % V == 0;
    if (whole) return half ? append8_go<T, V, true>(a, block, st) : append8_go<T, V, false>(a, block, st);
    return half ? append8_go<T, 2, true>(a, block, st) : append8_go<T, 2, false>(a, block, st);
}

// --------------------------------------------------------------------- read
// 8 * share tokens a CTA (gridDim.y of them share the tokens' rows, where there
// are few): a warp looks the entries of its share up, then all threads go over
// the rows, V codes (a 16-byte store) at a time.  128 thousand tokens of 8 heads of
// 128 to bf16 (765 MB): 126 us, 6.1 TB/s (0.89 of the copy rate).
constexpr int kReadTokens = 32, kReadUnits = 4;

template <typename T>
__global__ void __launch_bounds__(256) read8_kernel(const Read8Args a, const int share) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ long long code_s[kReadTokens], scale_s[kReadTokens];  // -1: zeros, -2: left alone
    pdl_launch_dependents();
    pdl_wait();
    const int t0 = (int)blockIdx.x * 8 * share, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (t0 + warp * share < a.batch.n_tokens) {
        // the sequence of the share's first token; from there a lane for each token
        int b = find_seq(a.batch, t0 + warp * share, lane);
        const int t = t0 + warp * share + lane;
        if (lane < share && t < a.batch.n_tokens) {
            while (b + 1 < a.batch.n_seqs && a.batch.q_start[b + 1] <= t) b++;
            const Seq s = load_seq(a.batch, b);
            const int i = t - s.q0, e = s.ctx + i;
            long long code = -2, sc = 0;
            if (!s.bad && i >= 0 && i < s.n) {
                const int page = entry_page(a.batch, b, e);
                code = -1;
                if (page >= 0) {
                    code = entry_offset(a.batch, a.cache, page, e);
                    sc = scale_index(a.batch, a.scales, a.n_kv_heads, page, 0, e);
                } else {
                    record_status(a.status, PP_ERR_INVALID_ARG);
                }
            }
            code_s[warp * share + lane] = code;
            scale_s[warp * share + lane] = sc;
        }
    }
    if (tid == 0 && blockIdx.y == 0)
        for (int b = blockIdx.x; b < a.batch.n_seqs; b += gridDim.x)
            if (load_seq(a.batch, b).bad) record_status(a.status, PP_ERR_INVALID_ARG);
    __syncthreads();
    // a thread keeps to one place of a row of keys and values and goes over the tokens; rows shorter than the CTA: as
    // many tokens at once as fit
    const int tokens = min(8 * share, a.batch.n_tokens - t0);
    const int per = a.head_dim / V, row = 2 * a.n_kv_heads * per;
    const int width = min(row, 256), at_once = 256 / width, lines = (tokens + at_once - 1) / at_once;
    const int mine = tid / width, col0 = tid - mine * width;
    if (mine >= at_once) return;
    // (columns, lines) of the CTA in chunks of kReadUnits lines, dealt over gridDim.y
    const int chunks = (lines + kReadUnits - 1) / kReadUnits, cols = (row + width - 1) / width;
    for (int w = blockIdx.y; w < chunks * cols; w += gridDim.y) {
        const int c = w % cols, u = c * width + col0, n0 = w / cols * kReadUnits;
        if (u >= row) continue;
        const bool key = u < row / 2;
        const int x = key ? u : u - row / 2, head = x / per;
        const char* codes = (key ? a.cache.k : a.cache.v) + head * a.cache.head_stride + (x - head * per) * V;
        const float* scales = (key ? a.scales.k : a.scales.v) + (long long)head * a.scales.blocks;
        const long long stride = key ? a.k_stride : a.v_stride;
        char* out = (key ? a.k_out : a.v_out) + t0 * stride + (long long)x * 16;
        typename Raw<V>::type code[kReadUnits];
        float sc[kReadUnits];
        int n[kReadUnits];
#pragma unroll
        for (int k = 0; k < kReadUnits; k++) {
            n[k] = (n0 + k) * at_once + mine;
            code[k] = {};
            sc[k] = 0.f;
            if (n[k] >= tokens || code_s[n[k]] == -2) {
                n[k] = -1;
            } else if (code_s[n[k]] >= 0) {
                code[k] = __ldcs(reinterpret_cast<const typename Raw<V>::type*>(codes + code_s[n[k]]));
                sc[k] = scales[scale_s[n[k]]];
            }
        }
#pragma unroll
        for (int k = 0; k < kReadUnits; k++) {
            if (n[k] < 0) continue;
            Vec<T, V> y;
            const uint32_t* words = reinterpret_cast<const uint32_t*>(&code[k]);
            const F2 sc2 = pair2(sc[k], sc[k]);
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const float2 v = from_codes(words[i / 4] >> (i % 4 * 8) & 0xffffu);
                float p, q;
                unpair2(mul2(pair2(v.x, v.y), sc2), p, q);
                y.set2(i, p, q);
            }
            y.store(out + n[k] * stride);
        }
    }
}

// ------------------------------------------------------------------- commit
// A CTA takes some of a sequence's units, one layer's and head's keys or values
// each: the path is looked up once, then a warp takes a unit at a time, two of
// them side by side, and moves their accepted entries a destination block at a time: first
// their largest magnitude, and with it the block's scale, then the codes.  Rows
// are read once where a warp holds a block's (16 rows of 128), else twice.  In
// place and without a barrier between warps: path[j] >= j, so what is read lies
// at or past what is written, and rows of one batch are read by the whole warp
// before any is written.  32 sequences of 8 accepted tokens in 32 layers (34 MB):
// 20 to 21 us (paths in their place already 18), half of it instructions (codes apart and together again) and the rest
// the chain path - places - codes - stores; one sequence: 4.9 us.
constexpr int kMoveBatch = 4;
constexpr int kMoveChunk = 128;  // entries of a destination block at most

// Largest magnitude among 16 codes times their scale: codes without their sign
// ascend as numbers do, four of them as two pairs of 16 bits an instruction.
PP_DEVINL float largest_of(const uint4& w, float scale) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        top = __vmaxu2(top, x[i] & 0x007f007fu);
        top = __vmaxu2(top, x[i] >> 8 & 0x007f007fu);
    }
    uint32_t m = max(top & 0xffffu, top >> 16);
    if (m == 0x7fu) {  // NaN among them, which does not count
        m = 0;
#pragma unroll 1
        for (int i = 0; i < 16; i++) {
            const uint32_t c = x[i >> 2] >> (i & 3) * 8 & 0x7fu;
            if (c != 0x7fu) m = max(m, c);
        }
    }
    return from_codes(m).x * scale;
}
// 16 codes rounded again at another scale.  The usual ratio, a power of two that
// fp16 holds, goes in fp16: code * ratio is exact there (a code has four bits,
// the least 2^-9; results are at most 448).  Numbers stay finite: at powers of two
// a value stays what it is or becomes less.
PP_DEVINL uint4 recode(const uint4& w, float ratio) {
    if (ratio == 1.f) return w;
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t y[4];
    const bool power = (__float_as_uint(ratio) & 0x7fffffu) == 0 && ratio >= 0x1p-14f && ratio <= 0x1p15f;
    if (power) {
        const __half2 r = __float2half2_rn(ratio);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint32_t out = 0;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                uint32_t h;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(x[i] >> 16 * k)));
                const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&h), r);
                uint16_t c;
                asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(*reinterpret_cast<const uint32_t*>(&v)));
                out |= (uint32_t)c << 16 * k;
            }
            y[i] = out;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 a = from_codes(x[i] & 0xffffu), b = from_codes(x[i] >> 16);
            y[i] = to_codes(a.x * ratio, a.y * ratio) | to_codes(b.x * ratio, b.y * ratio) << 16;
        }
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

__global__ void __launch_bounds__(256, 3) commit8_kernel(const Commit8Args a8) {
    const CommitArgs& a = a8.c;
    // of a window of accepted entries: code (-1: in its place already) and scale of the source, page of the destination
    __shared__ long long src_s[kMoveChunk], scale_s[kMoveChunk];
    __shared__ int page_s[kMoveChunk], bad_s;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x % a.batch.n_seqs, part = blockIdx.x / a.batch.n_seqs;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = (int)blockDim.x >> 5;
    const int32_t* path = a.path + (size_t)b * a.max_path;
    // the first path entries are asked for together with the lengths, not behind them
    const int first = tid < a.max_path ? path[tid] : 0, before = tid > 0 && tid < a.max_path ? path[tid - 1] : -1;
    const Seq s = load_seq(a.batch, b);
    const int acc = a.n_accept[b];
    auto look_up = [&](int j, int p, int w0) {  // accepted entry j, p in the tree; false: no such page
        const int from = entry_page(a.batch, b, s.ctx + p), to = entry_page(a.batch, b, s.ctx + j), i = j - w0;
        if (from < 0 || to < 0) return false;
        if (i < kMoveChunk) {
            src_s[i] = p == j ? -1 : entry_offset(a.batch, a.cache, from, s.ctx + p);
            scale_s[i] = scale_index(a.batch, a8.scales, a.n_kv_heads, from, 0, s.ctx + p);
            page_s[i] = to;
        }
        return true;
    };
    if (tid == 0) bad_s = s.bad || acc < 0 || acc > a.max_path || acc > s.n;
    __syncthreads();
    if (!bad_s) {
        bool bad = false;
        for (int j = tid; j < acc && !bad; j += blockDim.x) {
            const int p = j == tid ? first : path[j], prev = j == tid ? before : path[j - 1];
            bad = p < 0 || p >= s.n || p <= prev || !look_up(j, p, 0);
        }
        if (bad) bad_s = 1;
    }
    __syncthreads();
    const bool bad = bad_s != 0;
    if (part == 0 && tid == 0) {
        if (bad) record_status(a.status, PP_ERR_INVALID_ARG);
        if (a.new_len) a.new_len[b] = bad ? s.ctx : s.ctx + acc;
    }
    if (bad) return;
    const int D = a.head_bytes, shift = a8.scales.shift, block = 1 << shift;
    int group = 1;  // lanes of a row, 16 codes each
    while (group * 16 < D) group *= 2;
    const int per = 32 / group, col = lane % group * 16, row = lane / group;
    const bool on = col < D;
    // one layer's and head's keys or values each
    const int units = a.n_layers * 2 * a.n_kv_heads, u_end = min(units, (part + 1) * a8.units);
    for (int w0 = 0, w1; w0 < acc; w0 = w1) {
        w1 = min(acc, w0 + kMoveChunk);
        if (w1 < acc) w1 = ((s.ctx + w1) >> shift << shift) - s.ctx;  // whole blocks
        if (w0 > 0) {
            __syncthreads();  // the last window's readers are done
            for (int j = w0 + tid; j < w1; j += blockDim.x) look_up(j, path[j], w0);
            __syncthreads();
        }
        for (int u0 = part * a8.units + warp; u0 < u_end; u0 += 2 * warps) {
            char* codes[2];
            float* scales[2];
            bool have[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int u = u0 + k * warps, layer = u / (2 * a.n_kv_heads), v = u - layer * 2 * a.n_kv_heads;
                have[k] = u < u_end;
                const bool key = v < a.n_kv_heads;
                const int head = key ? v : v - a.n_kv_heads;
                codes[k] = (key ? a.cache.k : a.cache.v) + (long long)layer * a.layer_stride + (long long)head * a.cache.head_stride + col;
                scales[k] = (key ? a8.scales.k : a8.scales.v) + (long long)layer * a8.scale_layer_stride + (long long)head * a8.scales.blocks;
            }
            for (int j0 = w0, j1; j0 < w1; j0 = j1) {
                const int lo = (s.ctx + j0) >> shift << shift, n = min(w1, lo + block - s.ctx) - j0;
                j1 = j0 + n;
                const long long* src = src_s + (j0 - w0);
                const long long* from = scale_s + (j0 - w0);
                const int page = page_s[j0 - w0];
                const long long dst0 = entry_offset(a.batch, a.cache, page, lo),
                                to = scale_index(a.batch, a8.scales, a.n_kv_heads, page, 0, lo);
                bool stays = lo < s.ctx;
                for (int i = lane; i < n; i += 32) stays |= src[i] < 0;
                stays = __any_sync(kFull, stays);
                const bool once = n <= kMoveBatch * per;
                float old[2], amax[2] = {0.f, 0.f};
                uint4 w[2][kMoveBatch];
                float sc[2][kMoveBatch];
                auto fetch = [&](int k, int i0) {
#pragma unroll
                    for (int x = 0; x < kMoveBatch; x++) {
                        const int i = i0 + x * per;
                        w[k][x] = make_uint4(0u, 0u, 0u, 0u);
                        sc[k][x] = 0.f;
                        if (!have[k] || i >= n || src[i] < 0 || !on) continue;
                        w[k][x] = *reinterpret_cast<const uint4*>(codes[k] + src[i]);
                        sc[k][x] = scales[k][from[i]];
                    }
                };
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    old[k] = have[k] && stays ? scales[k][to] : 0.f;
                    if (once) fetch(k, row);
                }
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    if (!have[k]) continue;
                    for (int i0 = row; i0 - row < n; i0 += kMoveBatch * per) {
                        if (!once) fetch(k, i0);
#pragma unroll
                        for (int x = 0; x < kMoveBatch; x++)
                            if (i0 - row + x * per < n) amax[k] = fmaxf(amax[k], largest_of(w[k][x], sc[k][x]));
                    }
                    amax[k] = warp_max(amax[k]);
                    const float now = block_scale(amax[k], old[k], stays), inv = 1.f / now;
                    if (stays && now != old[k] && on) {
                        // entries that stay: cached ones, and accepted ones in their place
                        for (int e = lo + row; e < s.ctx + j1; e += per) {
                            if (e >= s.ctx && (e < s.ctx + j0 || src[e - s.ctx - j0] >= 0)) continue;
                            uint4* p = reinterpret_cast<uint4*>(codes[k] + dst0 + (e - lo) * a.cache.token_stride);
                            *p = recode(*p, old[k] * inv);
                        }
                    }
                    for (int i0 = row; i0 - row < n; i0 += kMoveBatch * per) {
                        if (!once) fetch(k, i0);
                        __syncwarp();
#pragma unroll
                        for (int x = 0; x < kMoveBatch; x++) {
                            const int i = i0 + x * per;
                            if (i >= n || src[i] < 0 || !on) continue;
                            *reinterpret_cast<uint4*>(codes[k] + dst0 + (s.ctx + j0 + i - lo) * a.cache.token_stride) =
                                recode(w[k][x], sc[k][x] * inv);
                        }
                        __syncwarp();
                    }
                    if (lane == 0 && now != old[k]) scales[k][to] = now;
                    __syncwarp();
                }
            }
        }
    }
}

}  // namespace

cudaError_t append8_launch(const Append8Args& a, int dtype, int layout, int block, cudaStream_t st) {
    return dtype == PP_BF16 ? append8_typed<__nv_bfloat16>(a, layout, block, st) : append8_typed<float>(a, layout, block, st);
}

cudaError_t read8_launch(const Read8Args& a, int dtype, cudaStream_t st) {
    // four CTAs an SM at least, where there is that much to do
    int share = kReadTokens / 8;
    while (share > 1 && (a.batch.n_tokens + 8 * share - 1) / (8 * share) < 608) share /= 2;
    const long long ctas = (a.batch.n_tokens + 8ll * share - 1) / (8 * share);
    const int row = 2 * a.n_kv_heads * (a.head_dim / (dtype == PP_BF16 ? 8 : 4)), at_once = std::max(1, 256 / row);
    const int chunks = ((8 * share + at_once - 1) / at_once + kReadUnits - 1) / kReadUnits * ((row + 255) / 256);
    const long long split = std::min<long long>(chunks, (608 + ctas - 1) / ctas);
    auto* kern = dtype == PP_BF16 ? read8_kernel<__nv_bfloat16> : read8_kernel<float>;
    return launch_overlapped(kern, dim3((unsigned)ctas, (unsigned)split), dim3(256), 0, st, a, share);
}

cudaError_t commit8_launch(Commit8Args a, cudaStream_t st) {
    // a unit a warp where that makes few CTAs, else about three CTAs an SM in all
    const long long units = (long long)a.c.n_layers * 2 * a.c.n_kv_heads;
    const int warps = (int)std::min<long long>(8, units);
    const long long most = (units + warps - 1) / warps, parts = std::max<long long>(1, std::min<long long>(most, 456 / a.c.batch.n_seqs));
    a.units = (int)((units + parts - 1) / parts);
    const long long ctas = (long long)a.c.batch.n_seqs * ((units + a.units - 1) / a.units);
    return launch_overlapped(commit8_kernel, dim3((unsigned)ctas), dim3((unsigned)(warps * 32)), 0, st, a);
}

}  // namespace pp
