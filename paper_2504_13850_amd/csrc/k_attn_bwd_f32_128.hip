// Attention backward, f32, head widths up to 128.
#include "attn_bwd.h"

namespace fo {
template fo_status attn_bwd_launch<float, 128>(const AttnArgs&, const BwdShape&, hipStream_t);
}  // namespace fo
