// gated_ffn_narrow_bf16.hip -- the narrow gated feed-forward block for __bf16.
#include "gated_ffn_narrow.h"

namespace abcd {
ABCD_FFN_NARROW(bf16, __bf16)
}
