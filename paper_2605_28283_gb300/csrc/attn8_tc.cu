// Attention over the paged cache on the tensor cores: pages of e4m3 codes, made
// bf16 on their way into shared memory.
#include "attn_tc.cuh"

namespace pp {

cudaError_t attn8_tc_launch(const AttnArgs& a, int sms, cudaStream_t st) { return launch<true>(a, sms, st); }

}  // namespace pp
