// Attention of new tokens over a paged cache with capped scores with a bias.
//
// 2048 tokens after their like: 233 us (172 without the cap); a batch of 24 (a prompt's 509 tokens and
// mostly single ones) 70 us (56): biases take far keys past 0.6 caps, which costs both formulas.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, true, true>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
