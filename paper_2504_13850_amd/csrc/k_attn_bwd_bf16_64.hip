// Attention backward, bf16, head widths up to 64.
#include "attn_bwd.h"

namespace fo {
template fo_status attn_bwd_launch<bf16_t, 64>(const AttnArgs&, const BwdShape&, hipStream_t);
}  // namespace fo
