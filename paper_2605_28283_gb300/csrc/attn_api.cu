// C ABI of the attention side: argument checks, workspace layout, dispatch.
// Nothing here allocates, synchronises or lets an exception out.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "pp_attn.h"
#include "pp_common.cuh"

namespace pp {
namespace {

constexpr uint64_t kWaitLimitNs = 2000000000ull;  // bounded waits give up after 2 s

#define PP_TRY(expr)                 \
    do {                             \
        const pp_status s_ = (expr); \
        if (s_ != PP_OK) return s_;  \
    } while (0)

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// SM count of the current device, which must be a GB300.  Asked for once a
// device: what is kept is a property of the device, written as one word.
pp_status device_sms(int* sms) {
    static std::atomic<int> known[64];
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PP_ERR_CUDA;
    const bool keep = dev >= 0 && dev < 64;
    if (keep && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return PP_OK;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return PP_ERR_CUDA;
    if (major != 10 || minor != 3) return PP_ERR_UNSUPPORTED;
    if (keep) known[dev].store(*sms, std::memory_order_relaxed);
    return PP_OK;
}

pp_status cuda_status(cudaError_t e) { return e == cudaSuccess ? PP_OK : PP_ERR_CUDA; }

int elem_size(int dtype) { return dtype == PP_BF16 ? 2 : 4; }

constexpr int kMaxHeads = 1024;
constexpr int kMaxHeadDim = 256;

pp_status check_heads(int dtype, int n_heads, int head_dim) {
    if (dtype != PP_BF16 && dtype != PP_F32) return PP_ERR_DTYPE;
    if (n_heads < 1 || n_heads > kMaxHeads) return PP_ERR_SHAPE;
    if (head_dim < 4 || head_dim > kMaxHeadDim || head_dim * elem_size(dtype) % 16 != 0) return PP_ERR_SHAPE;
    return PP_OK;
}

pp_status check_cache_shape(const pp_cache* c) {
    if (!c) return PP_ERR_INVALID_ARG;
    PP_TRY(check_heads(c->dtype, c->n_heads, c->head_dim));
    if (c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0) return PP_ERR_SHAPE;
    return PP_OK;
}

pp_status check_cache(const pp_cache* c) {
    PP_TRY(check_cache_shape(c));
    if (c->page_size < 1 || c->n_pages < 1) return PP_ERR_SHAPE;
    if (!c->k || !c->v) return PP_ERR_INVALID_ARG;
    const int e = elem_size(c->dtype);
    const int64_t strides[3] = {c->page_stride, c->token_stride, c->head_stride};
    for (int64_t s : strides) {
        if (s < 0 || s > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
        if (s * e % 16 != 0) return PP_ERR_ALIGN;
    }
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return PP_ERR_ALIGN;
    return PP_OK;
}

// Whether no two entries (page, offset, head, layer) of a cache that is to be
// written share memory.  Taken from the smallest stride up, each dimension has
// to step past all that the ones before it span, as in any dense array and its
// parts, whatever the order of its dimensions.
bool entries_apart(const pp_cache& c, int n_layers, int64_t layer_stride) {
    struct Dim {
        int64_t n, stride;
    } dims[4] = {{c.n_pages, c.page_stride}, {c.page_size, c.token_stride}, {c.n_kv_heads, c.head_stride},
                 {n_layers, layer_stride}};
    std::sort(dims, dims + 4, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    __int128 span = c.head_dim;  // 2^31 strides of 2^40
    for (const Dim& d : dims) {
        if (d.n == 1) continue;
        if (d.stride < span) return false;
        span += (__int128)d.stride * (d.n - 1);
    }
    return true;
}

pp_status check_batch_pointers(const pp_batch* b) {
    if (!b->q_start || !b->ctx_len || !b->pages) return PP_ERR_INVALID_ARG;
    if (!aligned(b->q_start, 4) || !aligned(b->ctx_len, 4) || !aligned(b->pages, 4)) return PP_ERR_ALIGN;
    return PP_OK;
}

// The pointers of a batch of no tokens are looked at by the one call that reads it all the same (pp_kv_commit).
pp_status check_batch(const pp_batch* b, const pp_cache* c) {
    if (!b) return PP_ERR_INVALID_ARG;
    if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_pages < 0) return PP_ERR_SHAPE;
    // query rows are numbered in 32 bits
    if ((long long)b->n_tokens * c->n_heads > 0x7fffffffll) return PP_ERR_SHAPE;
    if (b->n_seqs == 0 || b->n_tokens == 0) return PP_OK;
    return check_batch_pointers(b);
}

// A token tensor's rows (of no tokens: not looked at).
pp_status check_rows(const void* p, int64_t stride, int row, int e, int T) {
    if (T == 0) return PP_OK;
    if (!p) return PP_ERR_INVALID_ARG;
    if (stride < row || stride > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
    if (!aligned(p, 16) || stride * e % 16 != 0) return PP_ERR_ALIGN;
    return PP_OK;
}

pp_status check_rotation(const pp_rotation* r, int head_dim) {
    if (!r || !r->inv_freq || !std::isfinite(r->scale)) return PP_ERR_INVALID_ARG;
    if (r->layout != PP_ROPE_HALF && r->layout != PP_ROPE_INTERLEAVED) return PP_ERR_INVALID_ARG;
    if (r->rot_dim < 4 || r->rot_dim % 4 != 0 || r->rot_dim > head_dim) return PP_ERR_SHAPE;
    if (!aligned(r->inv_freq, 4)) return PP_ERR_ALIGN;
    return PP_OK;
}

// Rows [T] of `la` bytes `sa` apart at a against rows of `lb` bytes `sb`
// apart at b: whether any byte is shared.  Rows of one stride may be the
// parts of one buffer.
bool rows_overlap(const void* a, int64_t la, int64_t sa, const void* b, int64_t lb, int64_t sb, int T) {
    if (T < 1) return false;
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    const uint64_t ea = (uint64_t)(T - 1) * sa + la, eb = (uint64_t)(T - 1) * sb + lb;
    if (pa + ea <= pb || pb + eb <= pa) return false;
    if (T == 1 || sa != sb) return true;
    const int64_t d = (int64_t)(pb >= pa ? (pb - pa) % sa : (sa - (pa - pb) % sa) % sa);
    return d < la || d + lb > sa;
}

struct AttnLayout {
    size_t counters, tails, part, total;
};

AttnLayout attn_layout(const pp_cache& c) {
    AttnLayout L;
    L.counters = sizeof(Control);
    L.tails = (L.counters + kAttnMaxGrid * 4 + 255) & ~(size_t)255;
    L.part = (L.tails + kAttnTcGrid * kAttnTail + 255) & ~(size_t)255;
    L.total = (L.part + attn_part_floats(c.head_dim) * 4 + 255) & ~(size_t)255;
    return L;
}

pp_status check_attn_ws(const pp_cache* c, const void* ws, size_t ws_bytes) {
    if (!ws || !aligned(ws, 256) || ws_bytes < attn_layout(*c).total) return PP_ERR_WORKSPACE;
    return PP_OK;
}

BatchArgs batch_args(const pp_batch& b, const pp_cache& c) {
    return BatchArgs{b.q_start, b.ctx_len, b.pages, b.n_seqs, b.n_tokens, b.max_pages, c.page_size, c.n_pages};
}

PageArgs page_args(const pp_cache& c) {
    const long long e = elem_size(c.dtype);
    return PageArgs{static_cast<char*>(c.k), static_cast<char*>(c.v), c.page_stride * e, c.token_stride * e,
                    c.head_stride * e};
}

unsigned* status_of(void* ws) { return &static_cast<Control*>(ws)->status; }

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" {

pp_status pp_rope_frequencies(int scaling, int rot_dim, double base, double factor, double low, double high,
                              int trained_len, float* inv_freq, float* scale) {
    if (!inv_freq || !scale || scaling < PP_ROPE_NONE || scaling > PP_ROPE_YARN) return PP_ERR_INVALID_ARG;
    if (rot_dim < 4 || rot_dim % 4 != 0 || rot_dim > kMaxHeadDim) return PP_ERR_SHAPE;
    if (!std::isfinite(base) || !(base > 0) || !std::isfinite(factor) || !(factor > 0)) return PP_ERR_INVALID_ARG;
    const bool by_length = scaling == PP_ROPE_BANDED || scaling == PP_ROPE_YARN;
    if (by_length && (!std::isfinite(low) || !std::isfinite(high) || !(low > 0) || !(high > low) || trained_len < 1))
        return PP_ERR_INVALID_ARG;
    if (scaling == PP_ROPE_YARN && base == 1.0) return PP_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925286766559, r = rot_dim;
    if (scaling == PP_ROPE_NTK) base *= std::pow(factor, r / (r - 2.0));
    // number of the pair that turns `turns` times over the trained length
    auto pair_of = [&](double turns) { return r * std::log(trained_len / (turns * two_pi)) / (2.0 * std::log(base)); };
    double first = 0, last = 1;
    if (scaling == PP_ROPE_YARN) {
        first = std::fmax(std::floor(pair_of(high)), 0.0);
        last = std::fmin(std::ceil(pair_of(low)), r - 1.0);
        if (last <= first) last = first + 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / r);
        if (scaling == PP_ROPE_LINEAR) f /= factor;
        if (scaling == PP_ROPE_BANDED) {
            const double turns = trained_len * f / two_pi;
            const double w = (turns - low) / (high - low);
            f = w >= 1.0 ? f : w <= 0.0 ? f / factor : (1.0 - w) * f / factor + w * f;
        }
        if (scaling == PP_ROPE_YARN) {
            const double w = std::fmin(std::fmax((i - first) / (last - first), 0.0), 1.0);
            f = f * (1.0 - w) + f / factor * w;
        }
        inv_freq[i] = (float)f;
    }
    *scale = scaling == PP_ROPE_YARN && factor > 1.0 ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return PP_OK;
}

pp_status pp_rope(int dtype, const pp_rotation* rot, const int32_t* positions, int n_tokens, int n_heads,
                  int head_dim, const void* x, int64_t x_stride, void* y, int64_t y_stride, int inverse,
                  void* stream) {
    PP_TRY(check_heads(dtype, n_heads, head_dim));
    PP_TRY(check_rotation(rot, head_dim));
    if (n_tokens < 0) return PP_ERR_SHAPE;
    const int e = elem_size(dtype), row = n_heads * head_dim;
    PP_TRY(check_rows(x, x_stride, row, e, n_tokens));
    PP_TRY(check_rows(y, y_stride, row, e, n_tokens));
    if (!positions && n_tokens > 0) return PP_ERR_INVALID_ARG;
    if (!aligned(positions, 4)) return PP_ERR_ALIGN;
    if (!(x == y && x_stride == y_stride) &&
        rows_overlap(x, (int64_t)row * e, x_stride * e, y, (int64_t)row * e, y_stride * e, n_tokens))
        return PP_ERR_INVALID_ARG;
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (n_tokens == 0) return PP_OK;
    AppendArgs a;
    std::memset(&a, 0, sizeof a);
    a.batch.n_tokens = n_tokens;
    a.positions = positions;
    a.inv_freq = rot->inv_freq;
    a.rot_dim = rot->rot_dim;
    a.scale = rot->scale;
    a.inverse = inverse != 0;
    a.q = static_cast<const char*>(x);
    a.q_stride = x_stride * e;
    a.q_out = static_cast<char*>(y);
    a.q_out_stride = y_stride * e;
    a.n_heads = n_heads;
    a.head_dim = head_dim;
    return cuda_status(append_launch(a, dtype, rot->layout, static_cast<cudaStream_t>(stream)));
}

size_t pp_attn_workspace_size(const pp_cache* cache) {
    return check_cache_shape(cache) == PP_OK ? attn_layout(*cache).total : 0;
}

pp_status pp_kv_append(const pp_cache* cache, const pp_batch* batch, const pp_rotation* rot,
                       const int32_t* positions, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, void* ws,
                       size_t ws_bytes, void* stream) {
    PP_TRY(check_cache(cache));
    if (!entries_apart(*cache, 1, 0)) return PP_ERR_INVALID_ARG;
    PP_TRY(check_batch(batch, cache));
    if (rot) PP_TRY(check_rotation(rot, cache->head_dim));
    const int e = elem_size(cache->dtype), D = cache->head_dim, T = batch->n_tokens;
    const int q_row = cache->n_heads * D, kv_row = cache->n_kv_heads * D;
    if (!q != !q_out && T > 0) return PP_ERR_INVALID_ARG;
    if (positions && !aligned(positions, 4)) return PP_ERR_ALIGN;
    if (q && q_out) {
        PP_TRY(check_rows(q, q_stride, q_row, e, T));
        PP_TRY(check_rows(q_out, q_out_stride, q_row, e, T));
    }
    PP_TRY(check_rows(k, k_stride, kv_row, e, T));
    PP_TRY(check_rows(v, v_stride, kv_row, e, T));
    if (q && q_out) {
        const int64_t lq = (int64_t)q_row * e, lk = (int64_t)kv_row * e, so = q_out_stride * e;
        if (!(q == q_out && q_stride == q_out_stride) && rows_overlap(q, lq, q_stride * e, q_out, lq, so, T))
            return PP_ERR_INVALID_ARG;
        if (rows_overlap(k, lk, k_stride * e, q_out, lq, so, T) || rows_overlap(v, lk, v_stride * e, q_out, lq, so, T))
            return PP_ERR_INVALID_ARG;
    }
    PP_TRY(check_attn_ws(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (batch->n_seqs == 0 || T == 0) return PP_OK;
    AppendArgs a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch_args(*batch, *cache);
    a.cache = page_args(*cache);
    a.positions = positions;
    if (rot) {
        a.inv_freq = rot->inv_freq;
        a.rot_dim = rot->rot_dim;
        a.scale = rot->scale;
    }
    a.q = static_cast<const char*>(q);
    a.k = static_cast<const char*>(k);
    a.v = static_cast<const char*>(v);
    a.q_out = static_cast<char*>(q_out);
    a.q_stride = q_stride * e;
    a.k_stride = k_stride * e;
    a.v_stride = v_stride * e;
    a.q_out_stride = q_out_stride * e;
    a.n_heads = cache->n_heads;
    a.n_kv_heads = cache->n_kv_heads;
    a.head_dim = D;
    a.status = status_of(ws);
    return cuda_status(append_launch(a, cache->dtype, rot ? rot->layout : PP_ROPE_HALF, static_cast<cudaStream_t>(stream)));
}

pp_status pp_tree_attention(const pp_cache* cache, const pp_batch* batch, const void* q, int64_t q_stride,
                            const uint32_t* mask, int mask_words, float scale, void* out, int64_t out_stride,
                            void* ws, size_t ws_bytes, void* stream) {
    PP_TRY(check_cache(cache));
    PP_TRY(check_batch(batch, cache));
    if (!(scale > 0.0f) || !std::isfinite(scale)) return PP_ERR_INVALID_ARG;
    if (mask && mask_words < 1) return PP_ERR_INVALID_ARG;
    if (mask && !aligned(mask, 4)) return PP_ERR_ALIGN;
    if (mask && mask_words > 1 << 20) return PP_ERR_SHAPE;
    const int e = elem_size(cache->dtype), row = cache->n_heads * cache->head_dim;
    PP_TRY(check_rows(q, q_stride, row, e, batch->n_tokens));
    PP_TRY(check_rows(out, out_stride, row, e, batch->n_tokens));
    if (rows_overlap(q, (int64_t)row * e, q_stride * e, out, (int64_t)row * e, out_stride * e, batch->n_tokens))
        return PP_ERR_INVALID_ARG;
    PP_TRY(check_attn_ws(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return PP_OK;
    const AttnLayout L = attn_layout(*cache);
    AttnArgs a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch_args(*batch, *cache);
    a.cache = page_args(*cache);
    a.q = static_cast<const char*>(q);
    a.out = static_cast<char*>(out);
    a.q_stride = q_stride * e;
    a.out_stride = out_stride * e;
    a.mask = mask;
    a.mask_words = mask_words;
    a.n_kv_heads = cache->n_kv_heads;
    a.group = cache->n_heads / cache->n_kv_heads;
    a.head_dim = cache->head_dim;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.part);
    a.tails = static_cast<char*>(ws) + L.tails;
    a.counters = reinterpret_cast<unsigned*>(static_cast<char*>(ws) + L.counters);
    a.status = status_of(ws);
    a.timeout_ns = kWaitLimitNs;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(cache->dtype == PP_BF16 ? attn_tc_launch(a, sms, st) : attn_simt_launch(a, sms, st));
}

pp_status pp_kv_commit(const pp_cache* cache, const pp_batch* batch, int n_layers, int64_t layer_stride,
                       const int32_t* path, int max_path, const int32_t* n_accept, int32_t* new_len, void* ws,
                       size_t ws_bytes, void* stream) {
    PP_TRY(check_cache(cache));
    PP_TRY(check_batch(batch, cache));
    if (n_layers < 1 || max_path < 0) return PP_ERR_SHAPE;
    const int e = elem_size(cache->dtype);
    if (n_layers > 1) {
        if (layer_stride < 0 || layer_stride > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
        if (layer_stride * e % 16 != 0) return PP_ERR_ALIGN;
    }
    if (!entries_apart(*cache, n_layers, layer_stride)) return PP_ERR_INVALID_ARG;
    const int B = batch->n_seqs;
    if (B > 0 && (!n_accept || (!path && max_path > 0))) return PP_ERR_INVALID_ARG;
    if (!aligned(path, 4) || !aligned(n_accept, 4) || !aligned(new_len, 4)) return PP_ERR_ALIGN;
    if (B > 0) PP_TRY(check_batch_pointers(batch));
    if (new_len) {
        auto over = [&](const void* p, int64_t bytes) { return rows_overlap(new_len, 4ll * B, 4ll * B, p, bytes, bytes, B ? 1 : 0); };
        if (over(batch->ctx_len, 4ll * B) || over(n_accept, 4ll * B) || over(path, 4ll * B * max_path) ||
            over(batch->q_start, 4ll * (B + 1)) || over(batch->pages, 4ll * B * batch->max_pages))
            return PP_ERR_INVALID_ARG;
    }
    if ((long long)B * n_layers > 0x7fffffffll) return PP_ERR_SHAPE;
    PP_TRY(check_attn_ws(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (B == 0) return PP_OK;
    CommitArgs a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch_args(*batch, *cache);
    a.cache = page_args(*cache);
    a.path = path;
    a.n_accept = n_accept;
    a.new_len = new_len;
    a.max_path = max_path;
    a.n_layers = n_layers;
    a.layer_stride = layer_stride * e;
    a.n_kv_heads = cache->n_kv_heads;
    a.head_bytes = cache->head_dim * e;
    a.status = status_of(ws);
    return cuda_status(commit_launch(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
