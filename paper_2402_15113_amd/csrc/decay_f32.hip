// The linear attention's chunks of f32 rows.
#include <algorithm>

#include "decay_tile.h"

namespace tgm {

tgm_status_t decay_f32(const DecayRun &r, int what, hipStream_t s)
{
    return run_decay<float>(r, what, s);
}

}  // namespace tgm
