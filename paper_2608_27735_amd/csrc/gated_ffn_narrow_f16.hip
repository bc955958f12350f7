// gated_ffn_narrow_f16.hip -- the narrow gated feed-forward block for _Float16.
#include "gated_ffn_narrow.h"

namespace abcd {
ABCD_FFN_NARROW(f16, _Float16)
}
