// Attention over the paged cache on the tensor cores: pages of e4m3 codes, made
// bf16 on their way into shared memory; or, for few rows a key head, multiplied
// as they are (attn8_few.cu).
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // Rows a sequence brings to a key head on average, as in attn_tc.cuh.  64 sequences of 64 to 8191 entries, 32 heads on
    // 8, codes multiplied as they are / made bf16 first: 1 token each (4 rows) 99 / 252 us, 2 (8 rows) 110 / 254, 3 (two
    // items of 8) 194 / 267, 4 (16 rows) 203 / 268, 5 290 / 270, 8 (32 rows) 394 / 275.  4 sequences of 1000 to 4000: 18 /
    // 23 at 4 rows, 27 / 28 at 16, 32 / 35 at 32, 40 / 25 at 48.  One key head, 32 rows: 67 / 57.  A prompt beside single
    // tokens of 64 to 2000 entries, by the mean as well: 440 tokens beside 63 (31 rows) 230 / 127, 1024 beside 255 (20)
    // 702 / 385, 100 over 2000 entries beside 63 (10) 113 / 98, 50 beside 63 (7) 83 / 94.
    const long long rows = ((long long)a.batch.n_tokens * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
    if (rows <= 16) return attn8_few_launch(a, sms, st);
    return launch<true>(a, sms, st);
}

}  // namespace pp
