// The linear attention's chunks of f16 rows.
#include <algorithm>

#include "decay_tile.h"

namespace tgm {

tgm_status_t decay_f16(const DecayRun &r, int what, hipStream_t s)
{
    return run_decay<f16>(r, what, s);
}

}  // namespace tgm
