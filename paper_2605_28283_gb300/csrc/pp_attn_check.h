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

unsigned* status_of(void* ws) { return &static_cast<Control*>(ws)->status; }

}  // namespace
}  // namespace pp
