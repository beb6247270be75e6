// Attention backward for short sequences, bf16, head widths up to 64.
#include "attn_small.h"

namespace fo {
template fo_status small_bwd_launch<bf16_t, 64>(const AttnArgs&, hipStream_t);
}  // namespace fo
