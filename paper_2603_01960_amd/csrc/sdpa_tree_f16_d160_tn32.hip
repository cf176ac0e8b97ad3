// Trees of drafted tokens: element type f16, head dim 160, plain form (32-row K/V tiles).
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_f16_d160_tn32(int tile_m, const LaunchArgs &a) { return launch_tree_plain<_Float16, 160>(tile_m, a); }
}  // namespace tsdpa
