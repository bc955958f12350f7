// linear_f32.hip -- the linear layer's kernels for float.
#include "linear.h"

namespace abcd {
ABCD_LINEAR_KERNELS(f32, float)
}  // namespace abcd
