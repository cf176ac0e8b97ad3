// Trees of drafted tokens: element type f16, head dim 128, streams.
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_f16_d128_tn64(int tile_m, const LaunchArgs &a);
int launch_tree_f16_d128_halves(int tile_m, const LaunchArgs &a);
int launch_tree_f16_d128(int tile_m, const LaunchArgs &a)
{
    return launch_tree<_Float16, 128>(tile_m, a, launch_tree_f16_d128_tn64, launch_tree_f16_d128_halves);
}
}  // namespace tsdpa
