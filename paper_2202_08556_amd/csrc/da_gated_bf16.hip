// The gated feed-forward block in bfloat16.
#include "da_gated_host.h"

namespace daspmm {
template size_t gated_forward_bytes<bf16>(const GatedShape&);
template size_t gated_backward_bytes<bf16>(const GatedShape&);
template void gated_forward<bf16>(const GatedCall&);
template void gated_backward<bf16>(const GatedCall&);
}  // namespace daspmm
