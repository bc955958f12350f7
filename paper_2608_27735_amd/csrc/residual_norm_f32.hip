// residual_norm_f32.hip -- the joint between two blocks, for float.
#include "residual_norm.h"

namespace abcd {
ABCD_JOINT_KERNELS(f32, float)
}  // namespace abcd
