// Tiled products of f16 operands.
#include "linear_tile.h"

namespace tgm {

tgm_status_t linear_tile_f16(const LinearProduct &p, int which, int)
{
    const int parts = linear_splits(p.o.M, p.o.N, p.K, TGM_F16);
    switch (which) {
    case 0: return launch_tile<f16, f16, true, true, 256, 256, 2, 4>(p, parts);
    case 1: return launch_tile<f16, f16, false, true, 256, 256, 2, 4>(p, parts);
    default: return launch_tile<f16, f16, false, false, 256, 256, 2, 4>(p, parts);
    }
}

}  // namespace tgm
