// The gated feed-forward block in float32.
#include "da_gated_host.h"

namespace daspmm {
template size_t gated_forward_bytes<float>(const GatedShape&);
template size_t gated_backward_bytes<float>(const GatedShape&);
template void gated_forward<float>(const GatedCall&);
template void gated_backward<float>(const GatedCall&);
}  // namespace daspmm
