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

namespace pp {
namespace {

constexpr int kRowsInFlight = 2;  // rows a group has in flight

// One token for each blockIdx.x, its rows (q heads, then k heads) dealt over
// the groups of gridDim.y CTAs.
template <typename T, int V, bool HALF, int UPL>
__global__ void __launch_bounds__(256) norm_kernel(const NormArgs a) {
    using Lane = HeadLane<T, V, HALF, UPL>;
    __shared__ __align__(16) float2 cs[128];
    pdl_launch_dependents();
    pdl_wait();
    const HeadArgs& h = a.head;
    const int t = blockIdx.x, tid = threadIdx.x, groups = (int)blockDim.x / h.group;
    const Lane lane(h, tid % h.group);
    const int rows = a.n_heads + a.n_kv_heads, step = groups * (int)gridDim.y;
    float2 c[UPL][V];
    bool ready = false;
    for (int r0 = (int)blockIdx.y * groups; r0 < rows; r0 += step * kRowsInFlight) {
        Vec<T, V> x[kRowsInFlight][UPL][2];
#pragma unroll
        for (int n = 0; n < kRowsInFlight; n++) {
            const int r = r0 + n * step + tid / h.group;
            if (r >= rows) continue;
            const bool key = r >= a.n_heads;
            const long long head = (long long)(key ? r - a.n_heads : r) * h.head_dim * (int)sizeof(T);
            lane.load((key ? a.k + t * a.k_stride : a.q + t * a.q_stride) + head, x[n]);
        }
        if (!ready && h.rot_dim > 0) {
            fill_pairs(cs, h, V, h.positions[t], false, tid, blockDim.x);
            __syncthreads();
            lane.factors(cs, h, c);
        }
        ready = true;
#pragma unroll
        for (int n = 0; n < kRowsInFlight; n++) {
            const int r = r0 + n * step + tid / h.group;
            const bool in = r < rows, key = r >= a.n_heads;
            float f[UPL][2][V], g[UPL][2][V];
            lane.widen(x[n], f);
            const float inv = inverse_rms(Lane::group_sum(in ? Lane::dot(f, f) : 0.f, h.group), h);
            if (!in) continue;
            lane.weights(key ? a.k_gamma : a.q_gamma, g);
            Lane::scale_by(f, inv, g);
            if (h.rot_dim > 0) lane.rotate(f, c);
            lane.narrow(f, x[n]);
            const long long head = (long long)(key ? r - a.n_heads : r) * h.head_dim * (int)sizeof(T);
            lane.store((key ? a.k_out + t * a.k_out_stride : a.q_out + t * a.q_out_stride) + head, x[n]);
        }
    }
}

// Backward: the first ctas_q CTAs take the rows of q, the others those of k,
// each every ctas-th token; a thread adds its columns' part of dgamma up over
// all its rows, and the CTA leaves one row of sums, so that the result does
// not depend on the order in which CTAs run.
template <typename T, int V, bool HALF, int UPL>
__global__ void __launch_bounds__(256) norm_grad_kernel(const NormArgs a) {
    using Lane = HeadLane<T, V, HALF, UPL>;
    __shared__ __align__(16) float2 cs[128];
    __shared__ float sums[256 * UPL * 2 * V];
    pdl_launch_dependents();
    pdl_wait();
    const HeadArgs& h = a.head;
    const int tid = threadIdx.x, groups = (int)blockDim.x / h.group, D = h.head_dim;
    const bool key = (int)blockIdx.x >= a.ctas_q;
    const int first = key ? (int)blockIdx.x - a.ctas_q : (int)blockIdx.x, ctas = key ? a.ctas_k : a.ctas_q;
    const int rows = key ? a.n_kv_heads : a.n_heads;
    const char* xs = key ? a.k : a.q;
    const char* gs = key ? a.k_grad : a.q_grad;
    char* os = key ? a.k_out : a.q_out;
    const long long xstr = key ? a.k_stride : a.q_stride, gstr = key ? a.k_grad_stride : a.q_grad_stride,
                    ostr = key ? a.k_out_stride : a.q_out_stride;
    const Lane lane(h, tid % h.group);
    float gamma[UPL][2][V], acc[UPL][2][V] = {};
    lane.weights(key ? a.k_gamma : a.q_gamma, gamma);
    float2 c[UPL][V];
    for (int t = first; t < a.n_tokens; t += ctas) {
        if (h.rot_dim > 0) {
            __syncthreads();  // the last token's factors have been read
            fill_pairs(cs, h, V, h.positions[t], true, tid, blockDim.x);
            __syncthreads();
            lane.factors(cs, h, c);
        }
        for (int r0 = 0; r0 < rows; r0 += groups) {
            const int r = r0 + tid / h.group;
            const bool in = r < rows;
            const long long head = (long long)r * D * (int)sizeof(T);
            Vec<T, V> x[UPL][2], dy[UPL][2];
            float f[UPL][2][V] = {}, g[UPL][2][V] = {}, u[UPL][2][V];
            if (in) {
                lane.load(xs + t * xstr + head, x);
                lane.load(gs + t * gstr + head, dy);
                lane.widen(x, f);
                lane.widen(dy, g);
                if (h.rot_dim > 0) lane.rotate(g, c);
            }
#pragma unroll
            for (int k = 0; k < UPL; k++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    u[k][0][i] = g[k][0][i] * gamma[k][0][i];
                    u[k][1][i] = g[k][1][i] * gamma[k][1][i];
                }
            const float ss = Lane::group_sum(Lane::dot(f, f), h.group), ux = Lane::group_sum(Lane::dot(u, f), h.group);
            if (!in) continue;
            const float inv = inverse_rms(ss, h), along = inv * inv * ux / (float)D;
#pragma unroll
            for (int k = 0; k < UPL; k++)
#pragma unroll
                for (int s = 0; s < 2; s++)
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        acc[k][s][i] = fmaf(g[k][s][i], f[k][s][i] * inv, acc[k][s][i]);
                        f[k][s][i] = inv * (u[k][s][i] - f[k][s][i] * along);
                    }
            lane.narrow(f, x);
            lane.store(os + t * ostr + head, x);
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int k = 0; k < UPL; k++)
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int v = s ? lane.vb[k] : lane.va[k];
            if (v < 0) continue;
#pragma unroll
            for (int i = 0; i < V; i++) sums[tid / h.group * D + v * V + i] = acc[k][s][i];
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
        auto* kern = two ? norm_grad_kernel<T, V, HALF, kMost> : norm_grad_kernel<T, V, HALF, 1>;
        return launch_overlapped(kern, dim3((unsigned)(a.ctas_q + a.ctas_k)), dim3(256), 0, st, a);
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
