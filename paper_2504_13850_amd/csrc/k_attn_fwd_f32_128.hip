// Attention forward, f32, head widths up to 128.
#include "attn_fwd.h"

namespace fo {
template fo_status attn_fwd_launch<float, 128>(const AttnArgs&, const FwdShape&, hipStream_t);
}  // namespace fo
