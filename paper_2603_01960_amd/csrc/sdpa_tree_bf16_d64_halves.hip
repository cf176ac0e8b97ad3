// Trees of drafted tokens: element type bf16, head dim 64, 32 rows in four streams with weights in halves.
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_bf16_d64_halves(int tile_m, const LaunchArgs &a) { return launch_tree_halved<__bf16, 64>(tile_m, a); }
}  // namespace tsdpa
