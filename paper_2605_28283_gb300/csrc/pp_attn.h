// Internal launch interfaces of the attention side of a decode step: rotary
// positions, the paged key/value cache and attention over it.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "prunepath.h"

namespace pp {

// Grid bound of the attention kernels, and so of the partial results and
// counters in their workspace.
constexpr int kAttnMaxGrid = 608;      // CUDA-core kernel: up to 4 CTAs on each of 152 SMs
constexpr int kAttnSimtRows = 16;      // rows (token, head of the group) of its largest tile
constexpr int kAttnTcGrid = 152;       // tensor-core kernel: one CTA per SM ...
constexpr int kAttnTcRows = 256;       // ... and two tiles of 128 rows
constexpr int kAttnTail = 128;         // bytes of AttnArgs.tails per CTA

struct BatchArgs {
    const int32_t* q_start;
    const int32_t* ctx_len;
    const int32_t* pages;
    int n_seqs, n_tokens, max_pages, page_size, n_pages;
};

struct PageArgs {
    char* k;
    char* v;
    long long page_stride, token_stride, head_stride;  // bytes
};

// What is done to a head's row: norm (where `norm`) and rotation (where
// rot_dim > 0).  `group` lanes hold a row (pp_head.cuh).
struct HeadArgs {
    const int32_t* positions;
    const float* inv_freq;
    float scale, eps, inv_dim;  // inv_dim: 1 / head_dim
    int head_dim, rot_dim, group;
    bool norm;
};

struct NormArgs {
    HeadArgs head;
    const char *q, *k, *q_gamma, *k_gamma;
    const char *q_grad, *k_grad;  // gradients of the outputs (backward)
    char *q_out, *k_out;          // outputs, or the gradients of q and k
    long long q_stride, k_stride, q_grad_stride, k_grad_stride, q_out_stride, k_out_stride;  // bytes
    int n_tokens, n_heads, n_kv_heads;
    int ctas_q, ctas_k;  // backward: CTAs that take the rows of q and of k
    float* part;         // backward: sums of the weights' gradients, a row of head_dim a CTA
};

struct AppendArgs {
    BatchArgs batch;
    PageArgs cache;
    const int32_t* positions;
    const float* inv_freq;
    const char* q;
    const char* k;
    const char* v;
    char* q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;  // bytes
    int n_heads, n_kv_heads, head_dim, rot_dim;             // n_kv_heads 0: rotate q only, no cache
    float scale;
    int inverse;
    unsigned* status;
};

struct CommitArgs {
    BatchArgs batch;
    PageArgs cache;
    const int32_t* path;
    const int32_t* n_accept;
    int32_t* new_len;
    int max_path, n_layers;
    long long layer_stride;  // bytes
    int n_kv_heads, head_bytes;
    unsigned* status;
};

// Scales of an 8-bit cache (PageArgs then holds its codes).
struct ScaleArgs {
    float* k;
    float* v;
    int shift;   // block == 1 << shift
    int blocks;  // of a page
};

struct Append8Args {
    BatchArgs batch;
    PageArgs cache;
    ScaleArgs scales;
    HeadArgs head;
    const char *q, *k, *v, *q_gamma, *k_gamma;
    char* q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;  // bytes
    int n_heads, n_kv_heads;  // n_heads 0: no queries
    int slots, parts;         // blocks of tokens that may be new, CTAs of each
    int passes;               // of a CTA over heads' keys and values
    int team, split;          // threads of a token's queries, CTAs of them
    int stages, table_bytes;  // shared memory: units of keys and values on their way, behind the factors
    unsigned* status;
};

struct Read8Args {
    BatchArgs batch;
    PageArgs cache;
    ScaleArgs scales;
    char *k_out, *v_out;
    long long k_stride, v_stride;  // bytes
    int n_kv_heads, head_dim;
    unsigned* status;
};

struct Commit8Args {
    CommitArgs c;
    ScaleArgs scales;
    long long scale_layer_stride;  // floats
    int units;                     // of a CTA: one layer's and head's keys or values each
};

struct AttnArgs {
    BatchArgs batch;
    PageArgs cache;
    ScaleArgs scales;    // 8-bit cache
    const char* q;
    char* out;
    long long q_stride, out_stride;  // bytes
    const uint32_t* mask;
    int mask_words;
    int n_kv_heads, group, head_dim;
    unsigned min_rows, max_rows;  // query rows a key head of the sequences that this launch takes
    int head_shift;      // 1 << head_shift CTAs take as many key heads side by side (8-bit cache, few rows)
    int box;             // tokens of a TMA box of the cache, 0: copied row by row
    int q_box;           // whether the rows of q go by TMA
    float scale_log2;    // scale * log2(e): softmax in powers of two
    float* part;         // partial results of split items
    char* tails;         // [kAttnTcGrid] the split item that begins in each stretch (joined by a second kernel)
    int join_later;      // whether split items are joined by that kernel
    unsigned* counters;  // arrivals per split item, zero at rest
    unsigned* status;
    uint64_t timeout_ns;
};

constexpr int kNormGrid = 608;  // CTAs of the norms' backward pass at most
cudaError_t norm_launch(const NormArgs& a, int dtype, int layout, cudaStream_t st);
cudaError_t norm_grad_launch(NormArgs a, int dtype, int layout, float* q_gamma, float* k_gamma, int sms, cudaStream_t st);

cudaError_t append_launch(const AppendArgs& a, int dtype, int layout, cudaStream_t st);
cudaError_t commit_launch(const CommitArgs& a, cudaStream_t st);

cudaError_t append8_launch(const Append8Args& a, int dtype, int layout, int block, cudaStream_t st);
cudaError_t read8_launch(const Read8Args& a, int dtype, cudaStream_t st);
cudaError_t commit8_launch(Commit8Args a, cudaStream_t st);

size_t attn_part_floats(int head_dim);  // floats behind AttnArgs.part
cudaError_t attn_simt_launch(const AttnArgs& a, int sms, cudaStream_t st);  // fp32
cudaError_t attn_tc_launch(const AttnArgs& a, int sms, cudaStream_t st);    // bf16
cudaError_t attn8_simt_launch(const AttnArgs& a, int sms, cudaStream_t st);  // the same over 8-bit pages
cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st);
cudaError_t attn8_few_launch(const AttnArgs& a, int sms, cudaStream_t st);  // bf16, few rows a key head

}  // namespace pp
