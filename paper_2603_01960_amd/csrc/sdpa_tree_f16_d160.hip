// Trees of drafted tokens: element type f16, head dim 160, streams.
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_f16_d160_tn32(int tile_m, const LaunchArgs &a);
int launch_tree_f16_d160(int tile_m, const LaunchArgs &a)
{
    return launch_tree<_Float16, 160>(tile_m, a, launch_tree_f16_d160_tn32, nullptr);
}
}  // namespace tsdpa
