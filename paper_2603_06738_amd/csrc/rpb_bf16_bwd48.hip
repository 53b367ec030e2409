// Backward pair of the learned relative position bias, bf16: 48 columns, 2 block(s) of 32 channels.
#include "rpb_bf16_small.h"

namespace rib {
namespace rpb {
namespace bf {
hipError_t bwd48(const Geo &g, const BwdArgs &a, Ws &ws) { return launch_bwd<48, 2, kFast>(g, a, ws); }
}  // namespace bf
}  // namespace rpb
}  // namespace rib
