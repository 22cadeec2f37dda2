// Argument checks that the C entry points of the attention side share (host
// code).  Each returns PP_OK or the status to hand back.
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "pp_attn.h"
#include "pp_common.cuh"

namespace pp {
namespace {

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

pp_status check_norm(const pp_head_norm* n) {
    if (!n || !(n->eps >= 0.0f) || !std::isfinite(n->eps)) return PP_ERR_INVALID_ARG;
    if (!aligned(n->q_gamma, 16) || !aligned(n->k_gamma, 16)) return PP_ERR_ALIGN;
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

constexpr uint64_t kWaitLimitNs = 2000000000ull;  // bounded waits give up after 2 s

// Workspace of the calls on a cache.
struct AttnLayout {
    size_t counters, tails, part, total;
};

AttnLayout attn_layout(int head_dim) {
    AttnLayout L;
    L.counters = sizeof(Control);
    L.tails = (L.counters + kAttnMaxGrid * 4 + 255) & ~(size_t)255;
    L.part = (L.tails + kAttnTcGrid * kAttnTail + 255) & ~(size_t)255;
    L.total = (L.part + attn_part_floats(head_dim) * 4 + 255) & ~(size_t)255;
    return L;
}

unsigned* status_of(void* ws) { return &static_cast<Control*>(ws)->status; }

// The tensors and the mask of an attention call; rows of `row` elements.
pp_status check_attention(const pp_batch& batch, int dtype, int row, const void* q, int64_t q_stride, const uint32_t* mask,
                          int mask_words, float scale, const void* out, int64_t out_stride) {
    if (!(scale > 0.0f) || !std::isfinite(scale)) return PP_ERR_INVALID_ARG;
    if (mask && mask_words < 1) return PP_ERR_INVALID_ARG;
    if (mask && !aligned(mask, 4)) return PP_ERR_ALIGN;
    if (mask && mask_words > 1 << 20) return PP_ERR_SHAPE;
    const int e = elem_size(dtype);
    PP_TRY(check_rows(q, q_stride, row, e, batch.n_tokens));
    PP_TRY(check_rows(out, out_stride, row, e, batch.n_tokens));
    if (rows_overlap(q, (int64_t)row * e, q_stride * e, out, (int64_t)row * e, out_stride * e, batch.n_tokens))
        return PP_ERR_INVALID_ARG;
    return PP_OK;
}

AttnArgs attn_args(const pp_cache& c, const BatchArgs& batch, const PageArgs& pages, const void* q, int64_t q_stride,
                   const uint32_t* mask, int mask_words, float scale, void* out, int64_t out_stride, void* ws) {
    const AttnLayout L = attn_layout(c.head_dim);
    const int e = elem_size(c.dtype);
    AttnArgs a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch;
    a.cache = pages;
    a.q = static_cast<const char*>(q);
    a.out = static_cast<char*>(out);
    a.q_stride = q_stride * e;
    a.out_stride = out_stride * e;
    a.mask = mask;
    a.mask_words = mask_words;
    a.n_kv_heads = c.n_kv_heads;
    a.group = c.n_heads / c.n_kv_heads;
    a.head_dim = c.head_dim;
    a.max_rows = 0xffffffffu;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.part);
    a.tails = static_cast<char*>(ws) + L.tails;
    a.counters = reinterpret_cast<unsigned*>(static_cast<char*>(ws) + L.counters);
    a.status = status_of(ws);
    a.timeout_ns = kWaitLimitNs;
    return a;
}

// The accepted paths of a commit.
pp_status check_path(const pp_batch& batch, const int32_t* path, int max_path, const int32_t* n_accept, const int32_t* new_len) {
    const int B = batch.n_seqs;
    if (B > 0 && (!n_accept || (!path && max_path > 0))) return PP_ERR_INVALID_ARG;
    if (!aligned(path, 4) || !aligned(n_accept, 4) || !aligned(new_len, 4)) return PP_ERR_ALIGN;
    if (B > 0) PP_TRY(check_batch_pointers(&batch));
    if (new_len) {
        auto over = [&](const void* p, int64_t bytes) { return rows_overlap(new_len, 4ll * B, 4ll * B, p, bytes, bytes, B ? 1 : 0); };
        if (over(batch.ctx_len, 4ll * B) || over(n_accept, 4ll * B) || over(path, 4ll * B * max_path) ||
            over(batch.q_start, 4ll * (B + 1)) || over(batch.pages, 4ll * B * batch.max_pages))
            return PP_ERR_INVALID_ARG;
    }
    return PP_OK;
}

}  // namespace
}  // namespace pp
