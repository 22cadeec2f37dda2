// Attention over the paged cache on the tensor cores: pages of e4m3 codes, made
// bf16 on their way into shared memory; or, for few rows a key head, multiplied
// as they are (attn8_few.cu).
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // Rows a sequence brings to a key head on average, as in attn_tc.cuh.  64 sequences of 64 to 8191 entries, 32 heads on
    // 8, codes multiplied as they are / made bf16 first: 1 token each (4 rows) 99 / 253 us, 4 (16 rows) 132 / 269, 5 217 /
    // 271, 8 (32 rows, two items of 16) 247 / 275, 12 368 / 278.  4 sequences of 1000 to 4000: 31 / 28 at 16 rows, 34 / 36
    // at 32, 37 / 26 at 48.
    const long long rows = ((long long)a.batch.n_tokens * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
    if (rows <= 32) return attn8_few_launch(a, sms, st);
    return launch<true>(a, sms, st);
}

}  // namespace pp
