// Attention backward, f32, head widths up to 32.
#include "attn_bwd.h"

namespace fo {
template fo_status attn_bwd_launch<float, 32>(const AttnArgs&, const BwdShape&, hipStream_t);
}  // namespace fo
