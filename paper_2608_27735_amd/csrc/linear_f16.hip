// linear_f16.hip -- the linear layer's kernels for _Float16.
#include "linear.h"

namespace abcd {
ABCD_LINEAR_KERNELS(f16, _Float16)
}  // namespace abcd
