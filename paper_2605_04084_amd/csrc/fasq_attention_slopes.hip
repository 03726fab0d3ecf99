// Attention of new tokens over a paged cache with scores with a bias.
//
// One token on 1531 keys: 10.8 us and the join's 4.6, chains of reads (lengths, pages,
// keys).  A batch of 24 (a prompt's 509 tokens and mostly single ones): 52 us, some 10 us
// a tile of 128 rows besides its keys; single tokens of 3 rows are tiles of 128 rows too.
#include "fasq_attention_kernels.h"

namespace fasq {
template hipError_t launch_variant<Variant<true, false, true>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
}
