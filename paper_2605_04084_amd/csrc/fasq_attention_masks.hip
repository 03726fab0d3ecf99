// Attention of new tokens over a paged cache with masks of a call's own.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, false, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
