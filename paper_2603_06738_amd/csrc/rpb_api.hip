// Host side of the learned relative position bias and of the 8-bit checkpoints (include/rib_attn.h): argument validation and
// launches.  Nothing here allocates device memory or synchronises.
#include <initializer_list>

#include "rpb_common.h"

namespace rib {
namespace rpb {
namespace {

bool aligned(std::initializer_list<const void *> ptrs, uintptr_t to)
{
    for (const void *p : ptrs)
        if (((uintptr_t)p & (to - 1)) != 0) return false;
    return true;
}
uintptr_t value_bytes(int dtype) { return dtype == RIB_BF16 ? 2 : 4; }
rib_status status_of(hipError_t e) { return e == hipSuccess ? RIB_OK : RIB_ERR_LAUNCH; }

// An attention call's parameters: those of the implicit bias without one, on the matrix cores.
rib_status attn_geo(const rib_params *p, Geo *g)
{
    const rib_status st = make_geo(p, g);
    if (st != RIB_OK) return st;
    if (p->r != 0 || (p->flags & ~RIB_FLAG_FORCE_ROW_MAX) != 0 || p->heads > 65535) return RIB_ERR_UNSUPPORTED;
    return RIB_OK;
}
rib_status check_table(const rib_rpb_params *p)
{
    if (p == nullptr) return RIB_ERR_NULL;
    if (p->window < 1 || p->window > 256 || p->heads < 1 || p->heads > 65535 || p->buckets < 1 || p->buckets > (1 << 24)) return RIB_ERR_SHAPE;
    if (p->dtype != RIB_F32 && p->dtype != RIB_BF16) return RIB_ERR_DTYPE;
    return RIB_OK;
}
rib_status run_bwd(const rib_params *p, const void *q, const void *k, const void *v, const void *ckpt, const float *bias, const void *out,
                   const void *d_out, const float *lse, void *dq, void *dk, void *dv, float *dbias, void *workspace, size_t workspace_bytes,
                   void *stream)
{
    Geo g;
    const rib_status st = attn_geo(p, &g);
    if (st != RIB_OK) return st;
    const bool packed = ckpt != nullptr;
    if ((!packed && (!q || !k || !v)) || !bias || !out || !d_out || !lse || !dq || !dk || !dv) return RIB_ERR_NULL;
    if (!aligned({q, k, v, out, d_out, dq, dk, dv}, value_bytes(p->dtype)) || !aligned({bias, lse, dbias}, 4) || !aligned({ckpt}, 16))
        return RIB_ERR_SHAPE;
    const Ws ws = ws_layout(g, p->dtype);
    if (!workspace || !aligned({workspace}, 256) || workspace_bytes < (dbias != nullptr ? ws.total : ws.part)) return RIB_ERR_WORKSPACE;
    const BwdArgs a{q, k, v, (const uint8_t *)ckpt, bias, out, d_out, lse, dq, dk, dv, dbias, workspace, (hipStream_t)stream};
    return status_of(p->dtype == RIB_BF16 ? launch_bwd_bf16(g, a) : launch_bwd_f32(g, a));
}

}  // namespace
}  // namespace rpb
}  // namespace rib

using namespace rib;
using namespace rib::rpb;

extern "C" {

rib_status rib_rpb_table_fwd(const rib_rpb_params *p, const void *table, const int32_t *index, float *bias, void *stream)
{
    const rib_status st = check_table(p);
    if (st != RIB_OK) return st;
    if (!table || !index || !bias) return RIB_ERR_NULL;
    if (!aligned({table}, value_bytes(p->dtype)) || !aligned({index, bias}, 4)) return RIB_ERR_SHAPE;
    return status_of(launch_table_fwd(p->window, p->heads, p->buckets, p->dtype, table, index, bias, (hipStream_t)stream));
}

rib_status rib_rpb_table_bwd(const rib_rpb_params *p, const float *dbias, const int32_t *index, void *dtable, void *stream)
{
    const rib_status st = check_table(p);
    if (st != RIB_OK) return st;
    if (!dbias || !index || !dtable) return RIB_ERR_NULL;
    if (!aligned({dtable}, value_bytes(p->dtype)) || !aligned({index, dbias}, 4)) return RIB_ERR_SHAPE;
    return status_of(launch_table_bwd(p->window, p->heads, p->buckets, p->dtype, dbias, index, dtable, (hipStream_t)stream));
}

rib_status rib_rpb_attn_fwd(const rib_params *p, const void *q, const void *k, const void *v, const float *bias, void *out, float *lse,
                            void *stream)
{
    Geo g;
    const rib_status st = attn_geo(p, &g);
    if (st != RIB_OK) return st;
    if (!q || !k || !v || !bias || !out) return RIB_ERR_NULL;
    if (!aligned({q, k, v, out}, value_bytes(p->dtype)) || !aligned({bias, lse}, 4)) return RIB_ERR_SHAPE;
    const FwdArgs a{q, k, v, bias, out, lse, (p->flags & RIB_FLAG_FORCE_ROW_MAX) != 0, (hipStream_t)stream};
    return status_of(p->dtype == RIB_BF16 ? launch_fwd_bf16(g, a) : launch_fwd_f32(g, a));
}

size_t rib_rpb_attn_bwd_workspace_bytes(const rib_params *p)
{
    Geo g;
    return attn_geo(p, &g) == RIB_OK ? ws_layout(g, p->dtype).total : 0;
}

rib_status rib_rpb_attn_bwd(const rib_params *p, const void *q, const void *k, const void *v, const float *bias, const void *out,
                            const void *d_out, const float *lse, void *dq, void *dk, void *dv, float *dbias, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    return run_bwd(p, q, k, v, nullptr, bias, out, d_out, lse, dq, dk, dv, dbias, workspace, workspace_bytes, stream);
}

rib_status rib_rpb_attn_bwd_ckpt(const rib_params *p, const void *ckpt, const float *bias, const void *out, const void *d_out,
                                 const float *lse, void *dq, void *dk, void *dv, float *dbias, void *workspace, size_t workspace_bytes,
                                 void *stream)
{
    if (p != nullptr && ckpt == nullptr) {
        Geo g;
        const rib_status st = attn_geo(p, &g);
        return st != RIB_OK ? st : RIB_ERR_NULL;
    }
    return run_bwd(p, nullptr, nullptr, nullptr, ckpt, bias, out, d_out, lse, dq, dk, dv, dbias, workspace, workspace_bytes, stream);
}

size_t rib_checkpoint_bytes(const rib_params *p)
{
    Geo g;
    return make_geo(p, &g) == RIB_OK ? (size_t)(3 * ckpt_rows(g)) * (ckpt_row(g.d) + 1) : 0;
}

rib_status rib_checkpoint_pack(const rib_params *p, const void *q, const void *k, const void *v, void *ckpt, void *stream)
{
    Geo g;
    const rib_status st = make_geo(p, &g);
    if (st != RIB_OK) return st;
    if (!q || !k || !v || !ckpt) return RIB_ERR_NULL;
    if (!aligned({q, k, v}, value_bytes(p->dtype)) || !aligned({ckpt}, 16)) return RIB_ERR_SHAPE;
    return status_of(launch_pack(g, p->dtype, q, k, v, (uint8_t *)ckpt, (hipStream_t)stream));
}

rib_status rib_checkpoint_unpack(const rib_params *p, const void *ckpt, void *q, void *k, void *v, void *stream)
{
    Geo g;
    const rib_status st = make_geo(p, &g);
    if (st != RIB_OK) return st;
    if (!q || !k || !v || !ckpt) return RIB_ERR_NULL;
    if (!aligned({q, k, v}, value_bytes(p->dtype)) || !aligned({ckpt}, 16)) return RIB_ERR_SHAPE;
    return status_of(launch_unpack(g, p->dtype, (const uint8_t *)ckpt, q, k, v, (hipStream_t)stream));
}

}  // extern "C"
