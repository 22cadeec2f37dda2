// C ABI of the norms of query and key heads.
#include "pp_attn_check.h"

namespace pp {
namespace {

size_t norm_ws_bytes(int head_dim) { return ((size_t)kNormGrid * head_dim * 4 + 255) & ~(size_t)255; }

// A tensor of the call: rows of `row` bytes, `stride` bytes apart.
struct Rows {
    const void* p;
    int64_t row, stride;
};

// Whether an output shares memory with `x`, other than by being it.
bool clash(const Rows& out, const Rows& x, int T, bool may_be) {
    if (may_be && out.p == x.p && out.stride == x.stride) return false;
    return rows_overlap(out.p, out.row, out.stride, x.p, x.row, x.stride, T);
}

// Whether T rows share memory with `n` bytes at p (NULL: no).
bool touches(const Rows& r, int T, const void* p, int64_t n) {
    if (!p || T < 1) return false;
    const __int128 at = (__int128)(uintptr_t)p - (__int128)(uintptr_t)r.p;
    const __int128 i = at < 0 ? 0 : at / r.stride;  // the row that p lies in or behind, or the first one
    for (__int128 k = i; k < i + 2 && k < T; k++)
        if (at < k * r.stride + r.row && at + n > k * r.stride) return true;
    return false;
}

// Whether an output lies on the weights, the positions or the frequencies.
bool on_parameters(const Rows& out, int T, const pp_head_norm& norm, const pp_rotation* rot, const int32_t* positions,
                   int tokens, int64_t weight_bytes) {
    if (touches(out, T, norm.q_gamma, weight_bytes) || touches(out, T, norm.k_gamma, weight_bytes)) return true;
    return rot && (touches(out, T, positions, 4ll * tokens) || touches(out, T, rot->inv_freq, 2ll * rot->rot_dim));
}

pp_status check_call(int dtype, const pp_head_norm* norm, const pp_rotation* rot, const int32_t* positions, int T, int H,
                     int Hkv, int D) {
    PP_TRY(check_heads(dtype, H, D));
    PP_TRY(check_norm(norm));
    if (rot) PP_TRY(check_rotation(rot, D));
    if (T < 0 || Hkv < 0 || Hkv > kMaxHeads) return PP_ERR_SHAPE;
    if (rot && !positions && T > 0) return PP_ERR_INVALID_ARG;
    if (rot && !aligned(positions, 4)) return PP_ERR_ALIGN;
    return PP_OK;
}

NormArgs norm_args(const pp_head_norm* norm, const pp_rotation* rot, const int32_t* positions, int T, int H, int Hkv, int D) {
    NormArgs a;
    std::memset(&a, 0, sizeof a);
    a.head.norm = true;
    a.head.eps = norm->eps;
    a.head.head_dim = D;
    a.head.inv_dim = 1.0f / (float)D;
    if (rot) {
        a.head.positions = positions;
        a.head.inv_freq = rot->inv_freq;
        a.head.rot_dim = rot->rot_dim;
        a.head.scale = rot->scale;
    }
    a.q_gamma = static_cast<const char*>(norm->q_gamma);
    a.k_gamma = static_cast<const char*>(norm->k_gamma);
    a.n_tokens = T;
    a.n_heads = H;
    a.n_kv_heads = Hkv;
    return a;
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" {

size_t pp_head_norm_workspace_size(int head_dim) {
    return head_dim >= 4 && head_dim <= kMaxHeadDim && head_dim % 4 == 0 ? norm_ws_bytes(head_dim) : 0;
}

pp_status pp_head_norm_rope(int dtype, const pp_head_norm* norm, const pp_rotation* rot, const int32_t* positions,
                            int n_tokens, int n_heads, int n_kv_heads, int head_dim, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out,
                            int64_t k_out_stride, void* stream) {
    const int T = n_tokens;
    PP_TRY(check_call(dtype, norm, rot, positions, T, n_heads, n_kv_heads, head_dim));
    const int e = elem_size(dtype), q_row = n_heads * head_dim, k_row = n_kv_heads * head_dim;
    const bool keys = n_kv_heads > 0;
    PP_TRY(check_rows(q, q_stride, q_row, e, T));
    PP_TRY(check_rows(q_out, q_out_stride, q_row, e, T));
    if (keys) {
        PP_TRY(check_rows(k, k_stride, k_row, e, T));
        PP_TRY(check_rows(k_out, k_out_stride, k_row, e, T));
    }
    const Rows in[2] = {{q, (int64_t)q_row * e, q_stride * e}, {k, (int64_t)k_row * e, k_stride * e}};
    const Rows out[2] = {{q_out, (int64_t)q_row * e, q_out_stride * e}, {k_out, (int64_t)k_row * e, k_out_stride * e}};
    for (int o = 0; o < 1 + keys; o++)
        for (int i = 0; i < 1 + keys; i++)
            if (clash(out[o], in[i], T, o == i) || (i != o && clash(out[o], out[i], T, false))) return PP_ERR_INVALID_ARG;
    for (int o = 0; o < 1 + keys; o++)
        if (on_parameters(out[o], T, *norm, rot, positions, T, (int64_t)head_dim * e)) return PP_ERR_INVALID_ARG;
    int sms = 0;
    PP_TRY(device_sms(&sms));
    if (T == 0) return PP_OK;
    NormArgs a = norm_args(norm, rot, positions, T, n_heads, n_kv_heads, head_dim);
    a.q = static_cast<const char*>(q);
    a.k = static_cast<const char*>(k);
    a.q_out = static_cast<char*>(q_out);
    a.k_out = static_cast<char*>(k_out);
    a.q_stride = q_stride * e;
    a.k_stride = k_stride * e;
    a.q_out_stride = q_out_stride * e;
    a.k_out_stride = k_out_stride * e;
    return cuda_status(norm_launch(a, dtype, rot ? rot->layout : PP_ROPE_HALF, static_cast<cudaStream_t>(stream)));
}

pp_status pp_head_norm_rope_grad(int dtype, const pp_head_norm* norm, const pp_rotation* rot, const int32_t* positions,
                                 int n_tokens, int n_heads, int n_kv_heads, int head_dim, const void* q, int64_t q_stride,
                                 const void* k, int64_t k_stride, const void* q_grad, int64_t q_grad_stride,
                                 const void* k_grad, int64_t k_grad_stride, void* dq, int64_t dq_stride, void* dk,
                                 int64_t dk_stride, float* dq_gamma, float* dk_gamma, void* ws, size_t ws_bytes,
                                 void* stream) {
    const int T = n_tokens;
    PP_TRY(check_call(dtype, norm, rot, positions, T, n_heads, n_kv_heads, head_dim));
    const int e = elem_size(dtype), q_row = n_heads * head_dim, k_row = n_kv_heads * head_dim;
    const bool keys = n_kv_heads > 0;
    PP_TRY(check_rows(q, q_stride, q_row, e, T));
    PP_TRY(check_rows(q_grad, q_grad_stride, q_row, e, T));
    PP_TRY(check_rows(dq, dq_stride, q_row, e, T));
    if (keys) {
        PP_TRY(check_rows(k, k_stride, k_row, e, T));
        PP_TRY(check_rows(k_grad, k_grad_stride, k_row, e, T));
        PP_TRY(check_rows(dk, dk_stride, k_row, e, T));
    }
    if (!aligned(dq_gamma, 4) || !aligned(dk_gamma, 4)) return PP_ERR_ALIGN;
    const int64_t lq = (int64_t)q_row * e, lk = (int64_t)k_row * e, lg = (int64_t)head_dim * 4;
    // inputs: q, k, their gradients, the weights; outputs: dq, dk, the weights' gradients
    const Rows in[4] = {{q, lq, q_stride * e}, {q_grad, lq, q_grad_stride * e}, {k, lk, k_stride * e}, {k_grad, lk, k_grad_stride * e}};
    const Rows out[2] = {{dq, lq, dq_stride * e}, {dk, lk, dk_stride * e}};
    for (int o = 0; o < 1 + keys; o++)
        for (int i = 0; i < 2 + 2 * keys; i++)
            if (clash(out[o], in[i], T, i / 2 == o)) return PP_ERR_INVALID_ARG;
    if (keys && clash(out[0], out[1], T, false)) return PP_ERR_INVALID_ARG;
    for (int o = 0; o < 1 + keys; o++)
        if (on_parameters(out[o], T, *norm, rot, positions, T, (int64_t)head_dim * e)) return PP_ERR_INVALID_ARG;
    const float* dg[2] = {dq_gamma, dk_gamma};
    for (int g = 0; g < 2; g++) {
        if (!dg[g]) continue;
        if (on_parameters({dg[g], lg, lg}, 1, *norm, rot, positions, T, (int64_t)head_dim * e)) return PP_ERR_INVALID_ARG;
        auto over = [&](const Rows& r) { // the rows' whole span
            return r.p && T > 0 && rows_overlap(dg[g], lg, lg, r.p, (int64_t)(T - 1) * r.stride + r.row, r.stride, 1);
        };
        for (int i = 0; i < 2 + 2 * keys; i++)
            if (over(in[i])) return PP_ERR_INVALID_ARG;
        for (int o = 0; o < 1 + keys; o++)
            if (over(out[o])) return PP_ERR_INVALID_ARG;
        if (ws && rows_overlap(dg[g], lg, lg, ws, (int64_t)norm_ws_bytes(head_dim), lg, 1)) return PP_ERR_INVALID_ARG;
    }
    if (dq_gamma && dk_gamma && rows_overlap(dq_gamma, lg, lg, dk_gamma, lg, lg, 1)) return PP_ERR_INVALID_ARG;
    if (dq_gamma || dk_gamma) {
        const int64_t n = (int64_t)norm_ws_bytes(head_dim);
        if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)n) return PP_ERR_WORKSPACE;
        // written while the others are still read
        for (int i = 0; i < 2 + 2 * keys; i++)
            if (touches(in[i], T, ws, n)) return PP_ERR_INVALID_ARG;
        for (int o = 0; o < 1 + keys; o++)
            if (touches(out[o], T, ws, n)) return PP_ERR_INVALID_ARG;
        if (on_parameters({ws, n, n}, 1, *norm, rot, positions, T, (int64_t)head_dim * e)) return PP_ERR_INVALID_ARG;
    }
    int sms = 0;
    PP_TRY(device_sms(&sms));
    NormArgs a = norm_args(norm, rot, positions, T, n_heads, n_kv_heads, head_dim);
    a.q = static_cast<const char*>(q);
    a.k = static_cast<const char*>(k);
    a.q_grad = static_cast<const char*>(q_grad);
    a.k_grad = static_cast<const char*>(k_grad);
    a.q_out = static_cast<char*>(dq);
    a.k_out = static_cast<char*>(dk);
    a.q_stride = q_stride * e;
    a.k_stride = k_stride * e;
    a.q_grad_stride = q_grad_stride * e;
    a.k_grad_stride = k_grad_stride * e;
    a.q_out_stride = dq_stride * e;
    a.k_out_stride = dk_stride * e;
    a.part = static_cast<float*>(ws);
    return cuda_status(norm_grad_launch(a, dtype, rot ? rot->layout : PP_ROPE_HALF, dq_gamma, dk_gamma, sms,
                                        static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
