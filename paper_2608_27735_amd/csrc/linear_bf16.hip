// linear_bf16.hip -- the linear layer's kernels for __bf16.
#include "linear.h"

namespace abcd {
ABCD_LINEAR_KERNELS(bf16, __bf16)
}  // namespace abcd
