// Norms of query and key heads with the position rotation in the same pass,
// and their backward pass.  With r = 1 / sqrt(mean(x^2) + eps) and R the
// rotation by the token's position (times its attention factor m):
//   y = m R (r x * gamma)
//   g = m R^T dy,  u = g * gamma,  dx = r (u - x r^2 mean(u x)),
//   dgamma = sum over tokens and heads of g * x r.
// Every element is read and written once, so HBM bounds both (and launch
// latency, for a few tokens); r is formed again in the backward pass, which
// costs less than reading it.
#include <algorithm>

#include "pp_head.cuh"
#include "pp_launch.cuh"
#include "pp_tc.cuh"

namespace pp {
namespace {

constexpr int kRowsInFlight = 2;  // rows a group has in flight

// One token for each blockIdx.x, its rows (q heads, then k heads) dealt over
// the groups of gridDim.y CTAs.  8 tokens of 32 + 8 heads of 128 in bf16: 2.5 us;
// 4416 tokens (90 MB): 17 us, 5.3 TB/s, which L2 helps; 8192 (168 MB): 31 us, 5.5
// TB/s (0.81 of the copy rate); in fp32 (336 MB): 54 us, 6.2 TB/s (0.91).
template <typename T, int V, bool HALF, int UPL>
__global__ void __launch_bounds__(256) norm_kernel(const NormArgs a) {
    using Lane = HeadLane<T, V, HALF, UPL>;
    __shared__ __align__(16) float cs[256];
    pdl_launch_dependents();
    pdl_wait();
    const HeadArgs& h = a.head;
    const int t = blockIdx.x, tid = threadIdx.x, groups = (int)blockDim.x / h.group;
    const Lane lane(h, tid % h.group);
    const int rows = a.n_heads + a.n_kv_heads, step = groups * (int)gridDim.y;
    typename Lane::Factors c;
    bool ready = false;
    for (int r0 = (int)blockIdx.y * groups; r0 < rows; r0 += step * kRowsInFlight) {
        Vec<T, V> x[kRowsInFlight][UPL][2];
#pragma unroll
        for (int n = 0; n < kRowsInFlight; n++) {
            const int r = r0 + n * step + tid / h.group;
            if (r >= rows) continue;  // (its values are not used)
            const bool key = r >= a.n_heads;
            const long long head = (long long)(key ? r - a.n_heads : r) * h.head_dim * (int)sizeof(T);
            lane.load((key ? a.k + t * a.k_stride : a.q + t * a.q_stride) + head, x[n]);
        }
        if (!ready && h.rot_dim > 0) {
            fill_pairs(cs, h, V, h.positions[t], tid, blockDim.x);
            __syncthreads();
            lane.factors(cs, h, c);
        }
        ready = true;
#pragma unroll
        for (int n = 0; n < kRowsInFlight; n++) {
            const int r = r0 + n * step + tid / h.group;
            const bool in = r < rows, key = r >= a.n_heads;
            F2 f[UPL][2][V / 2], g[UPL][2][V / 2];
            Lane::widen(x[n], f);
            const float inv = inverse_rms(Lane::group_sum(in ? Lane::dot(f, f) : 0.f, h.group), h);
            if (!in) continue;
            lane.weights(key ? a.k_gamma : a.q_gamma, g);
            Lane::scale_by(f, inv, g);
            if (h.rot_dim > 0) lane.rotate(f, c);
            Lane::narrow(f, x[n]);
            const long long head = (long long)(key ? r - a.n_heads : r) * h.head_dim * (int)sizeof(T);
            lane.store((key ? a.k_out + t * a.k_out_stride : a.q_out + t * a.q_out_stride) + head, x[n]);
        }
    }
}

// Backward: the first ctas_q CTAs take the rows of q, the others those of k, in
// steps of as many rows as the CTA has groups (a few tokens' rows, or part of
// one's), every ctas-th step.  A thread copies what it will use of the next
// kStages - 1 steps into shared memory by cp.async, for itself alone, so that
// enough is on its way without registers.  The factors of the next few steps'
// tokens, one a thread where that many fit, are computed behind the present
// ones, with one barrier for all (a step at a time left six of eight warps
// waiting for two: 81 us).  It adds its columns' part of dgamma up
// over all its rows, and the CTA leaves one row of sums, so that the result does
// not depend on the order in which CTAs run.  8192 tokens of 32 + 8 heads of 128
// in bf16 (252 MB): 70 us, 3.6 TB/s (0.53 of the copy rate); a step is a chain of
// copies, two sums across lanes and the stores, with 16 warps an SM.  In fp32 (503
// MB): 94 us, 5.4 TB/s.
constexpr int kStages = 4;
constexpr int kGradSmem = 200 * 1024;  // 64 KB of stages, and up to 64 tokens' factors twice

// Steps whose factors are computed together, from those of a step.
__host__ __device__ inline int factor_batch(int per_step) {
    return per_step == 0 || per_step >= 256 ? 1 : 256 / per_step < 4 ? 256 / per_step : 4;
}

template <typename T, int V, bool HALF, int UPL>
__global__ void __launch_bounds__(256) norm_grad_kernel(const NormArgs a) {
    using Lane = HeadLane<T, V, HALF, UPL>;
    constexpr int kBytes = Lane::kBytes, kVecs = 4 * UPL;  // vectors of x and dy a thread and step
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float sums[256 * UPL * 2 * V];
    pdl_launch_dependents();
    pdl_wait();
    const HeadArgs& h = a.head;
    const int tid = threadIdx.x, groups = (int)blockDim.x / h.group, D = h.head_dim, pairs = h.rot_dim / 2;
    const bool key = (int)blockIdx.x >= a.ctas_q;
    const int first = key ? (int)blockIdx.x - a.ctas_q : (int)blockIdx.x, ctas = key ? a.ctas_k : a.ctas_q;
    const int rows = key ? a.n_kv_heads : a.n_heads;
    const char* xs = key ? a.k : a.q;
    const char* gs = key ? a.k_grad : a.q_grad;
    char* os = key ? a.k_out : a.q_out;
    const long long xstr = key ? a.k_stride : a.q_stride, gstr = key ? a.k_grad_stride : a.q_grad_stride,
                    ostr = key ? a.k_out_stride : a.q_out_stride;
    const Lane lane(h, tid % h.group);
    const int gi = tid / h.group, chunks = (rows + groups - 1) / groups, tokens = max(1, groups / rows);
    const int my_token = chunks == 1 ? gi / rows : 0, my_row = gi - my_token * rows;
    const int steps = (a.n_tokens + tokens - 1) / tokens * chunks;
    const int pitch = (pairs + V - 1) / V, table = V * pitch;  // factors of a token
    unsigned char* mine = smem + tid * kBytes;                 // vector v of stage s at ((s * kVecs + v) * 256 + tid): x's, then dy's
    const int batch = factor_batch(tokens * pairs);            // steps between barriers
    float* cs = reinterpret_cast<float*>(smem + kStages * kVecs * 256 * kBytes);  // two batches' tables
    // token and row of this thread in step s; false: none
    auto place = [&](int s, int& t, int& r) {
        const int c = chunks == 1 ? 0 : s % chunks;
        t = (chunks == 1 ? s : s / chunks) * tokens + my_token;
        r = c * groups + my_row;
        return s < steps && my_token < tokens && t < a.n_tokens && r < rows;
    };
    auto fetch = [&](int s, int stage) {
        int t, r;
        if (place(s, t, r)) {
            const char* x = xs + t * xstr + (long long)r * D * (int)sizeof(T);
            const char* g = gs + t * gstr + (long long)r * D * (int)sizeof(T);
            unsigned char* to = mine + stage * kVecs * 256 * kBytes;
#pragma unroll
            for (int k = 0; k < UPL; k++) {
                unsigned char *tx = to + 2 * k * 256 * kBytes, *tg = tx + 2 * UPL * 256 * kBytes;
                if (lane.va[k] >= 0) {
                    cp_async_small<kBytes>(tx, x + lane.va[k] * kBytes);
                    cp_async_small<kBytes>(tg, g + lane.va[k] * kBytes);
                }
                if (lane.vb[k] >= 0) {
                    cp_async_small<kBytes>(tx + 256 * kBytes, x + lane.vb[k] * kBytes);
                    cp_async_small<kBytes>(tg + 256 * kBytes, g + lane.vb[k] * kBytes);
                }
            }
        }
        cp_async_commit();
    };
    // factor i of the batch that begins with step s: its position, and its place in the tables
    const int per_step = tokens * pairs, entries = batch * per_step;
    auto position = [&](int s, int i) {
        const int j = s + i / per_step * ctas, t = (chunks == 1 ? j : j / chunks) * tokens + i % per_step / pairs;
        return j < steps && t < a.n_tokens ? h.positions[t] : 0;
    };
    auto fill = [&](int buf, int i, int pos) {
        const int n = i / pairs, p = i - n * pairs;  // token of the batch
        const float2 v = cos_sin(pos, h.inv_freq[p]);
        put_pair(cs + (buf * batch * tokens + n) * table * 2, p, V, pitch, make_float2(v.x * h.scale, v.y * h.scale));
    };
    F2 gamma[UPL][2][V / 2], acc[UPL][2][V / 2] = {};
    lane.weights(key ? a.k_gamma : a.q_gamma, gamma);
#pragma unroll
    for (int i = 0; i < kStages - 1; i++) fetch(first + i * ctas, i);
    if (pairs)
        for (int i = tid; i < entries; i += 256) fill(0, i, position(first, i));
    int n = 0, in_batch = 0, buf = 0, pos = 0;
    for (int s = first; s < steps; s += ctas, n++) {
        fetch(s + (kStages - 1) * ctas, (n + kStages - 1) % kStages);
        const int next = s + ctas;
        if (in_batch == batch - 1 && pairs && tid < entries) pos = position(next, tid);
        cp_async_wait<kStages - 1>();
        if (in_batch == 0) __syncthreads();  // this batch's factors are there, the last one's have been read
        int t, r;
        const bool in = place(s, t, r);
        F2 f[UPL][2][V / 2] = {}, g[UPL][2][V / 2] = {};
        Vec<T, V> x[UPL][2], dy[UPL][2];
        if (in) {
            const unsigned char* from = mine + n % kStages * kVecs * 256 * kBytes;
            lane.load_own(from, 256 * kBytes, true, x);
            lane.load_own(from + 2 * UPL * 256 * kBytes, 256 * kBytes, true, dy);
            Lane::widen(x, f);
            Lane::widen(dy, g);
            if (pairs) {
                typename Lane::Factors c;
                lane.factors(cs + ((buf * batch + in_batch) * tokens + my_token) * table * 2, h, c);
                lane.template rotate<true>(g, c);
            }
        }
        F2 u[UPL][2][V / 2];
#pragma unroll
        for (int k = 0; k < UPL; k++)
#pragma unroll
            for (int v = 0; v < 2; v++)
#pragma unroll
                for (int i = 0; i < V / 2; i++) u[k][v][i] = mul2(g[k][v][i], gamma[k][v][i]);
        const float ss = Lane::group_sum(Lane::dot(f, f), h.group), ux = Lane::group_sum(Lane::dot(u, f), h.group);
        if (in) {
            // with x r in place of x: dx = r (u - x r (r ux / D))
            const float inv = inverse_rms(ss, h), along = -inv * ux * h.inv_dim;
            const F2 inv2 = pair2(inv, inv), along2 = pair2(along, along);
#pragma unroll
            for (int k = 0; k < UPL; k++)
#pragma unroll
                for (int v = 0; v < 2; v++)
#pragma unroll
                    for (int i = 0; i < V / 2; i++) {
                        const F2 xr = mul2(f[k][v][i], inv2);
                        acc[k][v][i] = fma2(g[k][v][i], xr, acc[k][v][i]);
                        f[k][v][i] = mul2(fma2(xr, along2, u[k][v][i]), inv2);
                    }
            Lane::narrow(f, x);
            lane.store(os + t * ostr + (long long)r * D * (int)sizeof(T), x);
        }
        if (++in_batch == batch) {
            in_batch = 0;
            buf ^= 1;
            if (pairs && next < steps) {
                if (tid < entries) fill(buf, tid, pos);
                for (int i = tid + 256; i < entries; i += 256) fill(buf, i, position(next, i));
            }
        }
    }
    cp_async_wait<0>();
    if (!a.part) return;
#pragma unroll
    for (int k = 0; k < UPL; k++)
#pragma unroll
        for (int v = 0; v < 2; v++) {
            const int at = v ? lane.vb[k] : lane.va[k];
            if (at < 0) continue;
#pragma unroll
            for (int i = 0; i < V / 2; i++)
                unpair2(acc[k][v][i], sums[gi * D + at * V + 2 * i], sums[gi * D + at * V + 2 * i + 1]);
        }
    __syncthreads();
    for (int d = tid; d < D; d += blockDim.x) {
        float sum = 0.f;
        for (int g = 0; g < groups; g++) sum += sums[g * D + d];
        a.part[(size_t)blockIdx.x * D + d] = sum;
    }
}

// dgamma: the CTAs' sums added up, 8 columns a CTA, 32 threads a column (q for
// blockIdx.y 0, k for 1).
__global__ void __launch_bounds__(256) norm_gamma_kernel(const float* part, int D, int ctas_q, int ctas_k, float* q_gamma,
                                                         float* k_gamma) {
    __shared__ float s[32][9];
    pdl_launch_dependents();
    pdl_wait();
    const bool key = blockIdx.y != 0;
    const int n = key ? ctas_k : ctas_q, c = threadIdx.x & 7, w = threadIdx.x >> 3, d = (int)blockIdx.x * 8 + c;
    float* out = key ? k_gamma : q_gamma;
    if (!out) return;
    const float* p = part + (key ? (size_t)ctas_q * D : 0) + d;
    float sum = 0.f;
    if (d < D)
        for (int i = w; i < n; i += 32) sum += p[(size_t)i * D];
    s[w][c] = sum;
    __syncthreads();
    if (threadIdx.x >= 8 || d >= D) return;
    sum = 0.f;
    for (int i = 0; i < 32; i++) sum += s[i][c];
    out[d] = sum;
}

template <typename T, int V, bool HALF>
cudaError_t norm_go(NormArgs a, bool grad, cudaStream_t st) {
    const int units = head_units<V>(a.head);
    int group = 4;
    while (group < 32 && group < units) group *= 2;
    a.head.group = group;
    constexpr int kMost = V == 2 ? 2 : 1;  // two units a lane: more than 128 elements in vectors of 2
    const bool two = units > group;
    if (grad) {
        // tables of two batches' tokens, for the rows of q and of k
        const int groups = 256 / group, table = (a.head.rot_dim / 2 + V - 1) / V * V;
        auto tables = [&](int rows) {
            const int tokens = std::max(1, groups / std::max(1, rows));
            return 2 * factor_batch(tokens * (a.head.rot_dim / 2)) * tokens * table * 8;
        };
        const int smem = kStages * 4 * (two ? 2 : 1) * 256 * V * (int)sizeof(T) +
                         std::max(tables(a.n_heads), a.n_kv_heads ? tables(a.n_kv_heads) : 0);
        auto* kern = two ? norm_grad_kernel<T, V, HALF, kMost> : norm_grad_kernel<T, V, HALF, 1>;
        static std::atomic<bool> allowed[2][64];
        const cudaError_t e = allow_smem(kern, kGradSmem, allowed[two]);
        if (e != cudaSuccess) return e;
        return launch_overlapped(kern, dim3((unsigned)(a.ctas_q + a.ctas_k)), dim3(256), (size_t)smem, st, a);
    }
    const int rows = a.n_heads + a.n_kv_heads;
    int threads = (rows * group / 10 + 31) / 32 * 32;
    threads = threads < 64 ? 64 : threads > 256 ? 256 : threads;
    // about two CTAs an SM where there are few tokens
    int split = (304 + a.n_tokens - 1) / a.n_tokens;
    const int most = (rows * group + threads - 1) / threads;
    split = split < most ? split : most;
    auto* kern = two ? norm_kernel<T, V, HALF, kMost> : norm_kernel<T, V, HALF, 1>;
    return launch_overlapped(kern, dim3((unsigned)a.n_tokens, (unsigned)split), dim3((unsigned)threads), 0, st, a);
}

template <typename T>
cudaError_t norm_typed(const NormArgs& a, int layout, bool grad, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool half = layout == PP_ROPE_HALF;
    const bool whole = half ? a.head.rot_dim % (2 * V) == 0 : a.head.rot_dim % V == 0;
    if (whole) return half ? norm_go<T, V, true>(a, grad, st) : norm_go<T, V, false>(a, grad, st);
    return half ? norm_go<T, 2, true>(a, grad, st) : norm_go<T, 2, false>(a, grad, st);
}

}  // namespace

cudaError_t norm_launch(const NormArgs& a, int dtype, int layout, cudaStream_t st) {
    return dtype == PP_BF16 ? norm_typed<__nv_bfloat16>(a, layout, false, st) : norm_typed<float>(a, layout, false, st);
}

cudaError_t norm_grad_launch(NormArgs a, int dtype, int layout, float* q_gamma, float* k_gamma, int sms, cudaStream_t st) {
    // CTAs for q and for k in proportion to their rows, two an SM
    const int grid = 2 * sms < kNormGrid ? 2 * sms : kNormGrid, rows = a.n_heads + a.n_kv_heads;
    a.ctas_k = a.n_kv_heads ? std::max(1, (int)((long long)grid * a.n_kv_heads / rows)) : 0;
    a.ctas_q = grid - a.ctas_k;
    a.ctas_q = std::min(a.ctas_q, a.n_tokens);
    a.ctas_k = std::min(a.ctas_k, a.n_tokens);
    if (!q_gamma && !k_gamma) a.part = nullptr;
    if (a.n_tokens > 0) {
        const cudaError_t e = dtype == PP_BF16 ? norm_typed<__nv_bfloat16>(a, layout, true, st)
                                               : norm_typed<float>(a, layout, true, st);
        if (e != cudaSuccess) return e;
    }
    if (!q_gamma && !k_gamma) return cudaSuccess;
    return launch_overlapped(norm_gamma_kernel, dim3((unsigned)((a.head.head_dim + 7) / 8), 2), dim3(256), 0, st,
                             (const float*)a.part, a.head.head_dim, a.ctas_q, a.ctas_k, q_gamma, k_gamma);
}

}  // namespace pp
