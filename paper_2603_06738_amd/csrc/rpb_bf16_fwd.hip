// Forward of the learned relative position bias, bf16, and the choice of the kernels' widths.
#include <initializer_list>

#include "rpb_bf16_small.h"

namespace rib {
namespace rpb {
namespace {
// Whether 16-byte pieces can be moved: rows of 8 or more values, all of it on 4-byte boundaries.
bool fast(const Geo &g, std::initializer_list<const void *> ptrs)
{
    if (g.d < 8 || (g.d & 1) || (g.tstride & 1)) return false;
    for (const void *p : ptrs)
        if (((uintptr_t)p & 3) != 0) return false;
    return true;
}
}  // namespace

using namespace bf;

hipError_t launch_fwd_bf16(const Geo &g, const FwdArgs &a)
{
    if (!fast(g, {a.q, a.k, a.v, a.out}))
        return g.d <= 32 ? launch_fwd_src<32, 1, true, kAny>(g, a) : launch_fwd_src<64, 2, true, kAny>(g, a);
    if (g.d < 32) return launch_fwd_src<32, 1, false, kFast>(g, a);
    if (g.d == 32) return launch_fwd_src<32, 1, true, kFast>(g, a);
    if (g.d <= 48) return launch_fwd_src<48, 2, false, kFast>(g, a);
    if (g.d < 64) return launch_fwd_src<64, 2, false, kFast>(g, a);
    return launch_fwd_src<64, 2, true, kFast>(g, a);
}

hipError_t launch_bwd_bf16(const Geo &g, const BwdArgs &a)
{
    Ws ws = ws_layout(g, RIB_BF16);
    hipError_t e;
    if (!fast(g, {a.q, a.k, a.v, a.out, a.dout, a.dq, a.dk, a.dv})) e = bwd_any(g, a, ws);
    else if (g.d <= 32) e = bwd32(g, a, ws);
    else if (g.d <= 48) e = bwd48(g, a, ws);
    else e = bwd64(g, a, ws);
    if (e != hipSuccess || a.dbias == nullptr) return e;
    return launch_reduce(g, RIB_BF16, ws, (const float *)((const char *)a.ws + ws.part), a.dbias, a.st);
}

}  // namespace rpb
}  // namespace rib
