// Attention of new tokens over a paged cache with capped scores with a bias.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, true, true>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
