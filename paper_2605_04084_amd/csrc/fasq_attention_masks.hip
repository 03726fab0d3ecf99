// Attention of new tokens over a paged cache with masks of a call's own.
//
// A prompt of 4096 tokens in 11 documents (32 heads on 8 of 128): 59 us, 17 at the matrix
// product's rate; bound by what 1024 tiles of some 370 keys cost besides them.
// 2 trees of 64 nodes on 65536 to 131072 keys: 292 us, 706 TFLOP/s and 2.8 TB/s; bound by
// a wave's chain of steps, as the plain kernel is.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, false, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
