// Tiled products of 8-bit operands.
#include "linear_tile.h"

namespace tgm {

tgm_status_t linear_tile_e4m3(const LinearProduct &p, int, int out)
{
    const int parts = linear_splits(p.o.M, p.o.N, p.K, TGM_E4M3);
    switch (out) {
    case TGM_F32: return launch_tile<e4m3, float, true, true, 256, 256, 2, 4>(p, parts);
    case TGM_BF16: return launch_tile<e4m3, bf16, true, true, 256, 256, 2, 4>(p, parts);
    default: return launch_tile<e4m3, f16, true, true, 256, 256, 2, 4>(p, parts);
    }
}

}  // namespace tgm
