// residual_norm_f16.hip -- the joint between two blocks, for _Float16.
#include "residual_norm.h"

namespace abcd {
ABCD_JOINT_KERNELS(f16, _Float16)
}  // namespace abcd
