// gated_ffn_f32.hip -- the gated feed-forward block's kernels for float.
#include "gated_ffn.h"

namespace abcd {
ABCD_FFN_KERNELS(f32, float)
}
