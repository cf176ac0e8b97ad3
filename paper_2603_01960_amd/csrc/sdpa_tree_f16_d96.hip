// Trees of drafted tokens: element type f16, head dim 96, streams.
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_f16_d96_tn64(int tile_m, const LaunchArgs &a);
int launch_tree_f16_d96_halves(int tile_m, const LaunchArgs &a);
int launch_tree_f16_d96(int tile_m, const LaunchArgs &a)
{
    return launch_tree<_Float16, 96>(tile_m, a, launch_tree_f16_d96_tn64, launch_tree_f16_d96_halves);
}
}  // namespace tsdpa
