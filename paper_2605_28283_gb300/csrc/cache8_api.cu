// C ABI of the cache in 8 bits: argument checks, dispatch.
#include "pp_attn_check.h"

namespace pp {
namespace {

pp_status check_shape8(const pp_cache8* c) {
    if (!c) return PP_ERR_INVALID_ARG;
    PP_TRY(check_heads(c->dtype, c->n_heads, c->head_dim));
    if (c->head_dim % 16 != 0) return PP_ERR_SHAPE;
    if (c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0) return PP_ERR_SHAPE;
    return PP_OK;
}

// The codes as a pp_cache of one-byte elements.
pp_cache codes_of(const pp_cache8& c) {
    return pp_cache{c.dtype, c.n_heads, c.n_kv_heads, c.head_dim, c.page_size, c.n_pages, c.page_stride, c.token_stride,
                    c.head_stride, c.k, c.v};
}

int64_t scales_of(const pp_cache8& c) { return (int64_t)c.n_pages * c.n_kv_heads * (c.page_size / c.block); }

pp_status check_cache8(const pp_cache8* c) {
    PP_TRY(check_shape8(c));
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return PP_ERR_SHAPE;
    if (c->page_size < 1 || c->page_size % c->block != 0 || c->n_pages < 1) return PP_ERR_SHAPE;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return PP_ERR_INVALID_ARG;
    const int64_t strides[3] = {c->page_stride, c->token_stride, c->head_stride};
    for (int64_t s : strides) {
        if (s < 0 || s > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
        if (s % 16 != 0) return PP_ERR_ALIGN;
    }
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return PP_ERR_ALIGN;
    return PP_OK;
}

// For the calls that write: entries apart, and the two tensors' scales.
pp_status check_written(const pp_cache8& c, int n_layers, int64_t layer_stride, int64_t scale_layer_stride) {
    if (!entries_apart(codes_of(c), n_layers, layer_stride)) return PP_ERR_INVALID_ARG;
    const int64_t n = scales_of(c);
    if (n_layers > 1 && scale_layer_stride < n) return PP_ERR_INVALID_ARG;
    // the keys' and the values' scales may take turns layer by layer, but not share any
    if (rows_overlap(c.k_scale, n * 4, scale_layer_stride * 4, c.v_scale, n * 4, scale_layer_stride * 4, n_layers))
        return PP_ERR_INVALID_ARG;
    return PP_OK;
}

pp_status check_ws8(const pp_cache8* c, const void* ws, size_t ws_bytes) {
    if (!ws || !aligned(ws, 256) || ws_bytes < attn_layout(c->head_dim).total) return PP_ERR_WORKSPACE;
    return PP_OK;
}

BatchArgs batch_args8(const pp_batch& b, const pp_cache8& c) {
    return BatchArgs{b.q_start, b.ctx_len, b.pages, b.n_seqs, b.n_tokens, b.max_pages, c.page_size, c.n_pages};
}

PageArgs page_args8(const pp_cache8& c) {
    return PageArgs{static_cast<char*>(c.k), static_cast<char*>(c.v), c.page_stride, c.token_stride, c.head_stride};
}

ScaleArgs scale_args(const pp_cache8& c) {
    int shift = 4;
    while (1 << shift < c.block) shift++;
    return ScaleArgs{c.k_scale, c.v_scale, shift, c.page_size / c.block};
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" {

size_t pp_kvq_workspace_size(const pp_cache8* cache) {
    return check_shape8(cache) == PP_OK ? attn_layout(cache->head_dim).total : 0;
}

pp_status pp_kvq_append(const pp_cache8* cache, const pp_batch* batch, const pp_head_norm* norm, const pp_rotation* rot,
                        const int32_t* positions, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, void* ws, size_t ws_bytes,
                        void* stream) {
    PP_TRY(check_cache8(cache));
    PP_TRY(check_written(*cache, 1, 0, 0));
    const pp_cache codes = codes_of(*cache);
    PP_TRY(check_batch(batch, &codes));
    if (norm) PP_TRY(check_norm(norm));
    if (rot) PP_TRY(check_rotation(rot, cache->head_dim));
    const int e = elem_size(cache->dtype), D = cache->head_dim, T = batch->n_tokens;
    const int q_row = cache->n_heads * D, kv_row = cache->n_kv_heads * D;
    if (!q != !q_out && T > 0) return PP_ERR_INVALID_ARG;
    if (positions && !aligned(positions, 4)) return PP_ERR_ALIGN;
    const bool queries = q && q_out;
    if (queries) {
        PP_TRY(check_rows(q, q_stride, q_row, e, T));
        PP_TRY(check_rows(q_out, q_out_stride, q_row, e, T));
    }
    PP_TRY(check_rows(k, k_stride, kv_row, e, T));
    PP_TRY(check_rows(v, v_stride, kv_row, e, T));
    if (queries) {
        const int64_t lq = (int64_t)q_row * e, lk = (int64_t)kv_row * e, so = q_out_stride * e;
        if (!(q == q_out && q_stride == q_out_stride) && rows_overlap(q, lq, q_stride * e, q_out, lq, so, T))
            return PP_ERR_INVALID_ARG;
        if (rows_overlap(k, lk, k_stride * e, q_out, lq, so, T) || rows_overlap(v, lk, v_stride * e, q_out, lq, so, T))
            return PP_ERR_INVALID_ARG;
    }
    PP_TRY(check_ws8(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (batch->n_seqs == 0 || T == 0) return PP_OK;
    Append8Args a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch_args8(*batch, *cache);
    a.cache = page_args8(*cache);
    a.scales = scale_args(*cache);
    a.head.positions = positions;
    a.head.head_dim = D;
    a.head.inv_dim = 1.0f / (float)D;
    if (norm) {
        a.head.norm = true;
        a.head.eps = norm->eps;
        a.q_gamma = static_cast<const char*>(norm->q_gamma);
        a.k_gamma = static_cast<const char*>(norm->k_gamma);
    }
    if (rot) {
        a.head.inv_freq = rot->inv_freq;
        a.head.rot_dim = rot->rot_dim;
        a.head.scale = rot->scale;
    }
    a.q = static_cast<const char*>(q);
    a.k = static_cast<const char*>(k);
    a.v = static_cast<const char*>(v);
    a.q_out = static_cast<char*>(q_out);
    a.q_stride = q_stride * e;
    a.k_stride = k_stride * e;
    a.v_stride = v_stride * e;
    a.q_out_stride = q_out_stride * e;
    a.n_heads = queries ? cache->n_heads : 0;
    a.n_kv_heads = cache->n_kv_heads;
    a.status = status_of(ws);
    return cuda_status(append8_launch(a, cache->dtype, rot ? rot->layout : PP_ROPE_HALF, cache->block,
                                      static_cast<cudaStream_t>(stream)));
}

pp_status pp_kvq_read(const pp_cache8* cache, const pp_batch* batch, void* k_out, int64_t k_out_stride, void* v_out,
                      int64_t v_out_stride, void* ws, size_t ws_bytes, void* stream) {
    PP_TRY(check_cache8(cache));
    const pp_cache codes = codes_of(*cache);
    PP_TRY(check_batch(batch, &codes));
    const int e = elem_size(cache->dtype), T = batch->n_tokens, row = cache->n_kv_heads * cache->head_dim;
    PP_TRY(check_rows(k_out, k_out_stride, row, e, T));
    PP_TRY(check_rows(v_out, v_out_stride, row, e, T));
    if (T > 0 && rows_overlap(k_out, (int64_t)row * e, k_out_stride * e, v_out, (int64_t)row * e, v_out_stride * e, T))
        return PP_ERR_INVALID_ARG;
    PP_TRY(check_ws8(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (batch->n_seqs == 0 || T == 0) return PP_OK;
    Read8Args a;
    std::memset(&a, 0, sizeof a);
    a.batch = batch_args8(*batch, *cache);
    a.cache = page_args8(*cache);
    a.scales = scale_args(*cache);
    a.k_out = static_cast<char*>(k_out);
    a.v_out = static_cast<char*>(v_out);
    a.k_stride = k_out_stride * e;
    a.v_stride = v_out_stride * e;
    a.n_kv_heads = cache->n_kv_heads;
    a.head_dim = cache->head_dim;
    a.status = status_of(ws);
    return cuda_status(read8_launch(a, cache->dtype, static_cast<cudaStream_t>(stream)));
}

pp_status pp_kvq_tree_attention(const pp_cache8* cache, const pp_batch* batch, const void* q, int64_t q_stride,
                             const uint32_t* mask, int mask_words, float scale, void* out, int64_t out_stride, void* ws,
                             size_t ws_bytes, void* stream) {
    PP_TRY(check_cache8(cache));
    const pp_cache codes = codes_of(*cache);
    PP_TRY(check_batch(batch, &codes));
    PP_TRY(check_attention(*batch, cache->dtype, cache->n_heads * cache->head_dim, q, q_stride, mask, mask_words, scale, out,
                           out_stride));
    PP_TRY(check_ws8(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return PP_OK;
    AttnArgs a = attn_args(codes, batch_args8(*batch, *cache), page_args8(*cache), q, q_stride, mask, mask_words, scale, out,
                           out_stride, ws);
    a.scales = scale_args(*cache);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(cache->dtype == PP_BF16 ? attn8_tc_launch(a, sms, st) : attn8_simt_launch(a, sms, st));
}

pp_status pp_kvq_commit(const pp_cache8* cache, const pp_batch* batch, int n_layers, int64_t layer_stride,
                        int64_t scale_layer_stride, const int32_t* path, int max_path, const int32_t* n_accept,
                        int32_t* new_len, void* ws, size_t ws_bytes, void* stream) {
    PP_TRY(check_cache8(cache));
    const pp_cache codes = codes_of(*cache);
    PP_TRY(check_batch(batch, &codes));
    if (n_layers < 1 || max_path < 0) return PP_ERR_SHAPE;
    if (n_layers > 1) {
        if (layer_stride < 0 || layer_stride > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
        if (scale_layer_stride < 0 || scale_layer_stride > (int64_t)1 << 40) return PP_ERR_INVALID_ARG;
        if (layer_stride % 16 != 0) return PP_ERR_ALIGN;
    }
    PP_TRY(check_written(*cache, n_layers, layer_stride, scale_layer_stride));
    PP_TRY(check_path(*batch, path, max_path, n_accept, new_len));
    const int B = batch->n_seqs;
    if ((long long)B * n_layers > 0x7fffffffll || (long long)n_layers * 2 * cache->n_kv_heads > 0x7fffffffll) return PP_ERR_SHAPE;
    PP_TRY(check_ws8(cache, ws, ws_bytes));
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (B == 0) return PP_OK;
    Commit8Args a;
    std::memset(&a, 0, sizeof a);
    a.c.batch = batch_args8(*batch, *cache);
    a.c.cache = page_args8(*cache);
    a.c.path = path;
    a.c.n_accept = n_accept;
    a.c.new_len = new_len;
    a.c.max_path = max_path;
    a.c.n_layers = n_layers;
    a.c.layer_stride = layer_stride;
    a.c.n_kv_heads = cache->n_kv_heads;
    a.c.head_bytes = cache->head_dim;
    a.c.status = status_of(ws);
    a.scales = scale_args(*cache);
    a.scale_layer_stride = scale_layer_stride;
    return cuda_status(commit8_launch(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
