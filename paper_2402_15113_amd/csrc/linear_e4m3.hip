// Tiled products of 8-bit operands.
#include "linear_tile.h"

namespace tgm {

namespace {
template <class O> tgm_status_t go(const LinearProduct &p)
{
    const LinearPlan l = linear_plan(p.o.M, p.o.N, p.K, TGM_E4M3);
    if (!direct<e4m3, true, true>(p))
        return launch_tile<e4m3, O, true, true, 128, 128, 2, 2, false>(p, l.parts);
    return l.large ? launch_tile<e4m3, O, true, true, 256, 256, 2, 4, true>(p, l.parts)
                   : launch_tile<e4m3, O, true, true, 128, 128, 2, 2, true>(p, l.parts);
}
}  // namespace

tgm_status_t linear_tile_e4m3(const LinearProduct &p, int, int out)
{
    return out == TGM_F32 ? go<float>(p) : out == TGM_BF16 ? go<bf16>(p) : go<f16>(p);
}

}  // namespace tgm
