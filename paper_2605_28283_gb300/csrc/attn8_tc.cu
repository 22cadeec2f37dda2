// Attention over the paged cache on the tensor cores: pages of e4m3 codes, made
// bf16 on their way into shared memory; or, for few rows a key head, multiplied
// as they are (attn8_few.cu).
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // Rows that a sequence brings to a key head, on average: 64 sequences of 64 to 8191 entries, 32 heads on 8, codes
    // multiplied as they are / made bf16 first: 1 token each (4 rows) 99 / 252 us, 2 (8 rows) 110 / 254, 3 (two items of 8)
    // 194 / 267, 4 (16 rows) 203 / 268, 5 290 / 270, 8 (32 rows) 394 / 275.  4 sequences of 1000 to 4000: 18 / 23 at 4 rows,
    // 27 / 28 at 16, 32 / 35 at 32, 40 / 25 at 48.  One key head, 32 rows: 67 / 57.  Short contexts, where items cost more
    // than reading: 256 single tokens over 100 entries 77 / 60, 4 tokens each for 40 sequences of 100 to 500 58 / 35.
    constexpr long long kFew = 16, kLong = 512;
    const long long mean = mean_rows(a);
    if (mean > kFew) return launch<true>(a, mean, sms, st);
    // What the longest sequence brings if every one has a token.  Where that may be much, each kernel takes the sequences
    // that it is for: a prompt beside single tokens over 64 to 2000 entries, both / codes as they are / bf16 alone: 130
    // tokens beside 255 199 / 355 / 388 us, 160 beside 127 119 / 200 / 213, 765 beside 255 229 / 612 / 401, 1500 beside 511
    // 437 / 1205 / 722 (440 beside 63, 31 rows on average and so by bf16 alone: 127).  Two more launches cost 64 sequences
    // of 3 tokens 8 us of 194.
    const long long most = ((long long)a.batch.n_tokens - a.batch.n_seqs + 1) * a.group;
    if (most <= kLong) return attn8_few_launch(a, sms, st);
    AttnArgs part = a;
    part.max_rows = kFew;
    const cudaError_t e = attn8_few_launch(part, sms, st);
    if (e != cudaSuccess) return e;
    part.max_rows = a.max_rows;
    part.min_rows = kFew + 1;
    return launch<true>(part, most, sms, st);
}

}  // namespace pp
