// Attention over the paged cache on the tensor cores: pages of bf16.
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) { return launch<false>(a, mean_rows(a), sms, st); }

}  // namespace pp
