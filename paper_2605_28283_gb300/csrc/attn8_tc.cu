// Attention over the paged cache on the tensor cores: pages of e4m3 codes, made
// bf16 on their way into shared memory; or, for few rows a key head, multiplied
// as they are (attn8_few.cu).
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) {
    // Rows a sequence brings to a key head on average, as in attn_tc.cuh.  64 single tokens (4 rows): multiplied as they
    // are 99 us, made bf16 first 333.
    const long long rows = ((long long)a.batch.n_tokens * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
    if (rows <= 16) return attn8_few_launch(a, sms, st);
    return launch<true>(a, sms, st);
}

}  // namespace pp
