// residual_norm_bf16.hip -- the joint between two blocks, for __bf16.
#include "residual_norm.h"

namespace abcd {
ABCD_JOINT_KERNELS(bf16, __bf16)
}  // namespace abcd
