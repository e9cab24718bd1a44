// The cross entropy's products of bf16 operands.
#include "xent_tile.h"

namespace tgm {

tgm_status_t xent_sums_bf16(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<bf16, XentSums>(p, e, r);
}
tgm_status_t xent_grad_bf16(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<bf16, XentGrad>(p, e, r);
}
tgm_status_t xent_dx_bf16(const LinearProduct &p) { return xent_dx<bf16>(p); }
tgm_status_t xent_dw_bf16(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take)
{
    return xent_dw<bf16>(p, {x, ld, take});
}

}  // namespace tgm
