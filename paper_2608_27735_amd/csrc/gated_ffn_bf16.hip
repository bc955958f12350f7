// gated_ffn_bf16.hip -- the gated feed-forward block's kernels for __bf16.
#include "gated_ffn.h"

namespace abcd {
ABCD_FFN_KERNELS(bf16, __bf16)
}
