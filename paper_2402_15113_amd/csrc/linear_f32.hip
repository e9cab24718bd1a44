// Tiled products of fp32 operands.
#include "linear_tile.h"

namespace tgm {

tgm_status_t linear_tile_f32(const LinearProduct &p, int which, int)
{
    const int parts = linear_splits(p.o.M, p.o.N, p.K, TGM_F32);
    switch (which) {
    case 0: return launch_tile<float, float, true, true, 128, 64, 2, 2>(p, parts);
    case 1: return launch_tile<float, float, false, true, 128, 64, 2, 2>(p, parts);
    default: return launch_tile<float, float, false, false, 128, 64, 2, 2>(p, parts);
    }
}

}  // namespace tgm
