// Backward pair of the learned relative position bias, bf16: odd or short rows and unaligned tensors.
#include "rpb_bf16_small.h"

namespace rib {
namespace rpb {
namespace bf {
hipError_t bwd_any(const Geo &g, const BwdArgs &a, Ws &ws)
{
    return g.d <= 32 ? launch_bwd<32, 1, kAny>(g, a, ws) : launch_bwd<64, 2, kAny>(g, a, ws);
}
}  // namespace bf
}  // namespace rpb
}  // namespace rib
