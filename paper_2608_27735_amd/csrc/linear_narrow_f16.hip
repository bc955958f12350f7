// linear_narrow_f16.hip -- the linear layer of narrow rows, for _Float16.
#include "linear_narrow.h"

namespace abcd {
ABCD_LINEAR_NARROW(f16, _Float16)
}  // namespace abcd
