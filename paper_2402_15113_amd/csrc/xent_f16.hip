// The cross entropy's products of f16 operands.
#include "xent_tile.h"

namespace tgm {

tgm_status_t xent_sums_f16(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<f16, XentSums>(p, e, r);
}
tgm_status_t xent_grad_f16(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<f16, XentGrad>(p, e, r);
}
tgm_status_t xent_dx_f16(const LinearProduct &p) { return xent_dx<f16>(p); }
tgm_status_t xent_dw_f16(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take)
{
    return xent_dw<f16>(p, {x, ld, take});
}

}  // namespace tgm
