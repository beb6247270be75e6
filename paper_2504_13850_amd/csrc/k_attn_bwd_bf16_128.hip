// Attention backward, bf16, head widths up to 128.
#include "attn_bwd.h"

namespace fo {
template fo_status attn_bwd_launch<bf16_t, 128>(const AttnArgs&, const BwdShape&, hipStream_t);
}  // namespace fo
