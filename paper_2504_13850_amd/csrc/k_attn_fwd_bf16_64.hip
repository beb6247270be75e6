// Attention forward, bf16, head widths up to 64.
#include "attn_fwd.h"

namespace fo {
template fo_status attn_fwd_launch<bf16_t, 64>(const AttnArgs&, const FwdShape&, hipStream_t);
}  // namespace fo
