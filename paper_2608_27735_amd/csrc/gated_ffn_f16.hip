// gated_ffn_f16.hip -- the gated feed-forward block's kernels for _Float16.
#include "gated_ffn.h"

namespace abcd {
ABCD_FFN_KERNELS(f16, _Float16)
}
