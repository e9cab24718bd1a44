// The cross entropy's products of f32 operands.
#include "xent_tile.h"

namespace tgm {

tgm_status_t xent_sums_f32(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<float, XentSums>(p, e, r);
}
tgm_status_t xent_grad_f32(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    return xent_product<float, XentGrad>(p, e, r);
}
tgm_status_t xent_dw_f32(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take)
{
    return xent_dw<float>(p, {x, ld, take});
}

}  // namespace tgm
