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

struct AttnArgs {
    BatchArgs batch;
    PageArgs cache;
    const char* q;
    char* out;
    long long q_stride, out_stride;  // bytes
    const uint32_t* mask;
    int mask_words;
    int n_kv_heads, group, head_dim;
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

cudaError_t append_launch(const AppendArgs& a, int dtype, int layout, cudaStream_t st);
cudaError_t commit_launch(const CommitArgs& a, cudaStream_t st);

size_t attn_part_floats(int head_dim);  // floats behind AttnArgs.part
cudaError_t attn_simt_launch(const AttnArgs& a, int sms, cudaStream_t st);  // fp32
cudaError_t attn_tc_launch(const AttnArgs& a, int sms, cudaStream_t st);    // bf16

}  // namespace pp
