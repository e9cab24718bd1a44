// Tiled products of bf16 operands.
#include "linear_tile.h"

namespace tgm {

namespace {
// Operands that go through registers have none left for the large tile's.
template <bool PK, bool QK> tgm_status_t go(const LinearProduct &p)
{
    const LinearPlan l = linear_plan(p.o.M, p.o.N, p.K, TGM_BF16);
    if (!direct<bf16, PK, QK>(p))
        return launch_tile<bf16, bf16, PK, QK, 128, 128, 2, 2, false>(p, l.parts);
    return l.large ? launch_tile<bf16, bf16, PK, QK, 256, 256, 2, 4, true>(p, l.parts)
                   : launch_tile<bf16, bf16, PK, QK, 128, 128, 2, 2, true>(p, l.parts);
}
}  // namespace

tgm_status_t linear_tile_bf16(const LinearProduct &p, int which, int)
{
    return which == 0 ? go<true, true>(p) : which == 1 ? go<false, true>(p) : go<false, false>(p);
}

}  // namespace tgm
