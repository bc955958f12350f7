// linear_narrow_bf16.hip -- the linear layer of narrow rows, for __bf16.
#include "linear_narrow.h"

namespace abcd {
ABCD_LINEAR_NARROW(bf16, __bf16)
}  // namespace abcd
