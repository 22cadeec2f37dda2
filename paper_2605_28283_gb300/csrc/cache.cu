// Rotary positions and the paged key/value cache: rotation, append, and the
// commit of a drafted tree's accepted path.  All three move bytes and compute
// next to nothing, so HBM bounds them (and launch latency, for a few tokens).
#include "pp_batch.cuh"
#include "pp_launch.cuh"

namespace pp {
namespace {

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

// ------------------------------------------------------------------- append
// One token for each blockIdx.x; its heads' accesses ("units": a pair of
// vectors for half-split pairs, else one vector) are dealt over the threads
// of gridDim.y CTAs.  The token's cosines and sines are computed once, into
// shared memory, while the first loads are in flight.  V elements a vector:
// 16 bytes, or 2 elements where rot_dim does not split into whole vectors.
//
// Bound by HBM for many tokens and by latency for few.  8192 tokens of 40
// query, 40 key and 40 value heads of 128 in bf16 (477 MB): 78 us, 6.1 TB/s
// (0.90 of the copy rate); the queries alone (168 MB): 31 us, 5.5 TB/s (0.81).
// What counts for many tokens is few threads a CTA, so that many tokens are in
// flight (10 units a thread; 5 took 97 us), and for few tokens many CTAs a
// token.
constexpr int kAppendUnits = 2;     // units in flight per thread
constexpr int kUnitsAThread = 10;

template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
    constexpr int kBytes = V * (int)sizeof(T);
    __shared__ float2 cs[128];
    __shared__ long long dst_s;  // byte offset of the token's cache entry, -1: none
    __shared__ int pos_s;
    pdl_launch_dependents();
    pdl_wait();
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const int rv = HALF ? a.rot_dim / 2 / V : 0;          // vectors of the second half, done with the first
    const int per_v = a.head_dim / V, per_q = per_v - rv;  // units of a copied and of a rotated head
    const int nq = a.q ? a.n_heads * per_q : 0, nk = a.n_kv_heads * per_q;
    const int total = nq + nk + a.n_kv_heads * per_v;
    const unsigned magic = (unsigned)((0x100000000ull + per_q - 1) / per_q);    // u / per_q = umulhi(u, magic)
    const unsigned magic_v = (unsigned)((0x100000000ull + per_v - 1) / per_v);  // (u * per < 2^32)
    const int stride = (int)(gridDim.y * blockDim.x);
    const int rot2 = a.rot_dim / 2;

    // the token's entry and position; needs no data, so it runs first in warp 0
    if (tid < 32) {
        int pos = a.positions ? a.positions[t] : 0;
        long long dst = -1;
        if (a.n_kv_heads) {
            const int b = find_seq(a.batch, t, lane);
            const Seq s = load_seq(a.batch, b);
            const int i = t - s.q0;
            if (!s.bad && i >= 0 && i < s.n) {
                const int page = entry_page(a.batch, b, s.ctx + i);
                if (page >= 0)
                    dst = entry_offset(a.batch, a.cache, page, s.ctx + i);
                else if (lane == 0)
                    record_status(a.status, PP_ERR_INVALID_ARG);
                if (!a.positions) pos = s.ctx + i;
            }
            // padding, or a skipped sequence: nothing is written, q_out included
            if (s.bad || i < 0 || i >= s.n) dst = -2;
        }
        if (lane == 0) {
            pos_s = pos;
            dst_s = dst;
        }
    } else if (tid == 32 && blockIdx.y == 0 && a.n_kv_heads) {
        // every sequence is looked at once, also one that no token belongs to
        for (int b = t; b < a.batch.n_seqs; b += gridDim.x)
            if (load_seq(a.batch, b).bad) record_status(a.status, PP_ERR_INVALID_ARG);
    }
    bool ready = false;
    for (int u0 = blockIdx.y * blockDim.x + tid; u0 - tid < total; u0 += kAppendUnits * stride) {
        Vec<T, V> x0[kAppendUnits], x1[kAppendUnits];
        int what[kAppendUnits], head[kAppendUnits], c[kAppendUnits];
#pragma unroll
        for (int k = 0; k < kAppendUnits; k++) {
            int u = u0 + k * stride;
            what[k] = -1;
            if (u >= total) continue;
            const char* src;
            unsigned m = magic, per = per_q;
            long long row;
            if (u < nq) {
                what[k] = 0;
                src = a.q;
                row = a.q_stride;
            } else if (u < nq + nk) {
                what[k] = 1;
                u -= nq;
                src = a.k;
                row = a.k_stride;
            } else {
                what[k] = 2;
                u -= nq + nk;
                src = a.v;
                row = a.v_stride;
                m = magic_v;
                per = per_v;
            }
            head[k] = per == 1 ? u : (int)__umulhi((unsigned)u, m);
            c[k] = u - head[k] * (int)per;
            src += (long long)t * row + (long long)head[k] * a.head_dim * (int)sizeof(T);
            // past the rotated pairs, a unit is one vector behind the second half
            if (HALF && what[k] < 2 && c[k] >= rv) c[k] += rv;
            x0[k].load(src + c[k] * kBytes);
            if (HALF && what[k] < 2 && c[k] < rv) x1[k].load(src + (c[k] + rv) * kBytes);
        }
        if (!ready) {
            __syncthreads();
            for (int i = tid; i < rot2; i += blockDim.x) {
                float2 v = cos_sin(pos_s, a.inv_freq[i]);
                cs[i] = make_float2(v.x * a.scale, (a.inverse ? -v.y : v.y) * a.scale);
            }
            __syncthreads();
            ready = true;
        }
        const long long dst = dst_s;
#pragma unroll
        for (int k = 0; k < kAppendUnits; k++) {
            if (what[k] < 0) continue;
            const bool pair = HALF && what[k] < 2 && c[k] < rv;
            if (pair) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 w0 = cs[c[k] * V + i], w1 = cs[c[k] * V + i + 1];
                    const float a0 = x0[k].get(i), a1 = x0[k].get(i + 1), b0 = x1[k].get(i), b1 = x1[k].get(i + 1);
                    x0[k].set2(i, a0 * w0.x - b0 * w0.y, a1 * w1.x - b1 * w1.y);
                    x1[k].set2(i, b0 * w0.x + a0 * w0.y, b1 * w1.x + a1 * w1.y);
                }
            } else if (!HALF && what[k] < 2 && c[k] * V < a.rot_dim) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 w = cs[(c[k] * V + i) / 2];
                    const float p = x0[k].get(i), q = x0[k].get(i + 1);
                    x0[k].set2(i, p * w.x - q * w.y, q * w.x + p * w.y);
                }
            }
            char* out;
            if (what[k] == 0) {
                if (dst == -2) continue;
                out = a.q_out + (long long)t * a.q_out_stride + (long long)head[k] * a.head_dim * (int)sizeof(T);
            } else {
                if (dst < 0) continue;
                out = (what[k] == 1 ? a.cache.k : a.cache.v) + dst + (long long)head[k] * a.cache.head_stride;
            }
            x0[k].store(out + c[k] * kBytes);
            if (pair) x1[k].store(out + (c[k] + rv) * kBytes);
        }
    }
}

template <typename T, int V, bool HALF>
cudaError_t append_go(const AppendArgs& a, cudaStream_t st) {
    const int per_v = a.head_dim / V, per_q = per_v - (HALF ? a.rot_dim / 2 / V : 0);
    const int total = (a.q ? a.n_heads * per_q : 0) + a.n_kv_heads * (per_q + per_v);
    const int T_ = a.batch.n_tokens;
    int threads = (total / kUnitsAThread + 31) / 32 * 32;
    threads = threads < 64 ? 64 : threads > 256 ? 256 : threads;
    // about two CTAs an SM where there are few tokens
    int split = (304 + T_ - 1) / T_;
    const int most = (total + threads - 1) / threads;
    split = split < most ? split : most;
    return launch_overlapped(append_kernel<T, V, HALF>, dim3((unsigned)T_, (unsigned)split), dim3((unsigned)threads),
                             0, st, a);
}

template <typename T>
cudaError_t append_typed(const AppendArgs& a, int layout, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool half = layout == PP_ROPE_HALF;
    const bool whole = half ? a.rot_dim % (2 * V) == 0 : a.rot_dim % V == 0;
    if (whole) return half ? append_go<T, V, true>(a, st) : append_go<T, V, false>(a, st);
    return half ? append_go<T, 2, true>(a, st) : append_go<T, 2, false>(a, st);
}

// ------------------------------------------------------------------- commit
// One CTA for each (sequence, layer).  A thread owns one 16-byte column of
// the entries (of the keys or of the values) and moves it for the accepted
// tokens in ascending order, kCommitBatch loads before their stores.  In
// place and without a barrier: path[j] >= j, so what a later token reads lies
// past everything that earlier ones wrote, and no other thread touches the
// column.  32 sequences of 8 accepted tokens in 32 layers (67 MB read and
// written): 14.0 us, 4.8 TB/s (0.71 of the copy rate); one sequence: 2.6 us.
constexpr int kCommitBatch = 8;
constexpr int kCommitChunk = 64;  // path entries whose places are held in shared memory

__global__ void __launch_bounds__(256) commit_kernel(const CommitArgs a) {
    __shared__ long long src_s[kCommitChunk], dst_s[kCommitChunk];
    __shared__ int bad_s;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x % a.batch.n_seqs, layer = blockIdx.x / a.batch.n_seqs;
    const int tid = threadIdx.x;
    const int32_t* path = a.path + (size_t)b * a.max_path;
    // the first path entries are asked for together with the lengths, not behind them
    const int first = tid < a.max_path && tid < kCommitChunk ? path[tid] : 0;
    const int before = tid > 0 && tid < a.max_path && tid < kCommitChunk ? path[tid - 1] : -1;
    const Seq s = load_seq(a.batch, b);
    const int acc = a.n_accept[b];
    if (tid == 0) bad_s = s.bad || acc < 0 || acc > a.max_path || acc > s.n;
    __syncthreads();
    if (!bad_s) {
        bool bad = false;
        for (int j = tid; j < acc; j += blockDim.x) {
            const int p = j < kCommitChunk ? first : path[j];
            if (p < 0 || p >= s.n || p <= (j < kCommitChunk ? before : path[j - 1])) {
                bad = true;
                break;
            }
            const int src = entry_page(a.batch, b, s.ctx + p), dst = entry_page(a.batch, b, s.ctx + j);
            if (src < 0 || dst < 0) {
                bad = true;
                break;
            }
            if (j < kCommitChunk) {
                src_s[j] = entry_offset(a.batch, a.cache, src, s.ctx + p);
                dst_s[j] = entry_offset(a.batch, a.cache, dst, s.ctx + j);
            }
        }
        if (bad) bad_s = 1;
    }
    __syncthreads();
    const bool bad = bad_s != 0;
    if (layer == 0 && tid == 0) {
        if (bad) record_status(a.status, PP_ERR_INVALID_ARG);
        if (a.new_len) a.new_len[b] = bad ? s.ctx : s.ctx + acc;
    }
    if (bad) return;
    const int per_head = a.head_bytes / 16, cols = a.n_kv_heads * per_head;
    const long long base = (long long)layer * a.layer_stride;
    for (int j0 = 0; j0 < acc; j0 += kCommitChunk) {
        const int n = min(kCommitChunk, acc - j0);
        if (j0 > 0) __syncthreads();
        if (j0 > 0 && tid < n) {
            const int src = s.ctx + path[j0 + tid], dst = s.ctx + j0 + tid;
            src_s[tid] = entry_offset(a.batch, a.cache, entry_page(a.batch, b, src), src);
            dst_s[tid] = entry_offset(a.batch, a.cache, entry_page(a.batch, b, dst), dst);
        }
        if (j0 > 0) __syncthreads();
        for (int c = tid; c < 2 * cols; c += blockDim.x) {
            const int cc = c < cols ? c : c - cols;
            char* col = (c < cols ? a.cache.k : a.cache.v) + base + (long long)(cc / per_head) * a.cache.head_stride +
                        (cc % per_head) * 16;
            for (int j = 0; j < n; j += kCommitBatch) {
                uint4 v[kCommitBatch];
#pragma unroll
                for (int i = 0; i < kCommitBatch; i++)
                    if (j + i < n) v[i] = *reinterpret_cast<const uint4*>(col + src_s[j + i]);
#pragma unroll
                for (int i = 0; i < kCommitBatch; i++)
                    if (j + i < n && src_s[j + i] != dst_s[j + i]) *reinterpret_cast<uint4*>(col + dst_s[j + i]) = v[i];
            }
        }
    }
}

}  // namespace

cudaError_t append_launch(const AppendArgs& a, int dtype, int layout, cudaStream_t st) {
    return dtype == PP_BF16 ? append_typed<__nv_bfloat16>(a, layout, st) : append_typed<float>(a, layout, st);
}

cudaError_t commit_launch(const CommitArgs& a, cudaStream_t st) {
    const long long ctas = (long long)a.batch.n_seqs * a.n_layers;
    const int cols = 2 * a.n_kv_heads * (a.head_bytes / 16);
    const int threads = cols >= 256 ? 256 : cols <= 64 ? 64 : (cols + 31) / 32 * 32;
    return launch_overlapped(commit_kernel, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, a);
}

}  // namespace pp
