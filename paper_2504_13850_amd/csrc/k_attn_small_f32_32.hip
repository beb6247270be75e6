// Attention backward for short sequences, f32, head widths up to 32.
#include "attn_small.h"

namespace fo {
template fo_status small_bwd_launch<float, 32>(const AttnArgs&, hipStream_t);
}  // namespace fo
