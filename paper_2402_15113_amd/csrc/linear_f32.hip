// Tiled products of fp32 operands.
#include "linear_tile.h"

namespace tgm {

namespace {
// The small tile gives every wavefront 64 columns and 16 rows: with a few thousand
// of them the SIMDs come out even (12,000 x 200 outputs of the framework's gates).
template <bool PK, bool QK, bool DIRECT> tgm_status_t go(const LinearProduct &p)
{
    const LinearPlan l = linear_plan(p.o.M, p.o.N, p.K, TGM_F32);
    return l.large ? launch_tile<float, float, PK, QK, 128, 128, 2, 2, DIRECT>(p, l.parts)
                   : launch_tile<float, float, PK, QK, 64, 64, 1, 4, DIRECT>(p, l.parts);
}
template <bool PK, bool QK> tgm_status_t go(const LinearProduct &p)
{
    return direct<float, PK, QK>(p) ? go<PK, QK, true>(p) : go<PK, QK, false>(p);
}
}  // namespace

tgm_status_t linear_tile_f32(const LinearProduct &p, int which, int)
{
    return which == 0 ? go<true, true>(p) : which == 1 ? go<false, true>(p) : go<false, false>(p);
}

}  // namespace tgm
