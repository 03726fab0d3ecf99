// Attention of new tokens over a paged cache with capped scores.
//
// 64 tokens on 300 to 8192 keys each: 128 us, memory at 5.0 TB/s.  2048 tokens after their
// like: 168 us, 126 without caps: 16 caps a lane are vector instructions between two blocks of
// the pipeline, where this wave's matrix cores have nothing to do; 217 us where many scores
// are past 0.6 caps (see cap_scores).
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, true, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
