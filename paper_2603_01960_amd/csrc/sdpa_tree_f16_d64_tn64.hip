// Trees of drafted tokens: element type f16, head dim 64, plain form (64-row K/V tiles up to D = 128: see extra_flags in build.py).
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_f16_d64_tn64(int tile_m, const LaunchArgs &a) { return launch_tree_plain<_Float16, 64>(tile_m, a); }
}  // namespace tsdpa
