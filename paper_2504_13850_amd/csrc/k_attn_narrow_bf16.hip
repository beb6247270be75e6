// Attention for heads of up to eight columns, bf16.
#include "attn_narrow.h"

namespace fo {
#define FO_NARROW(D)                                                                            \
    template fo_status narrow_fwd_launch<bf16_t, D>(const AttnArgs&, const FwdShape&, hipStream_t); \
    template fo_status narrow_bwd_launch<bf16_t, D>(const AttnArgs&, const BwdShape&, hipStream_t)
FO_NARROW(2);
FO_NARROW(4);
FO_NARROW(8);
#undef FO_NARROW
}  // namespace fo
