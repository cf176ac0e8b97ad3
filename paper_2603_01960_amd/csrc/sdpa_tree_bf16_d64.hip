// Trees of drafted tokens: element type bf16, head dim 64, streams.
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_bf16_d64_tn64(int tile_m, const LaunchArgs &a);
int launch_tree_bf16_d64_halves(int tile_m, const LaunchArgs &a);
int launch_tree_bf16_d64(int tile_m, const LaunchArgs &a)
{
    return launch_tree<__bf16, 64>(tile_m, a, launch_tree_bf16_d64_tn64, launch_tree_bf16_d64_halves);
}
}  // namespace tsdpa
