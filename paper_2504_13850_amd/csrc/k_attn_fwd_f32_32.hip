// Attention forward, f32, head widths up to 32.
#include "attn_fwd.h"

namespace fo {
template fo_status attn_fwd_launch<float, 32>(const AttnArgs&, const FwdShape&, hipStream_t);
}  // namespace fo
