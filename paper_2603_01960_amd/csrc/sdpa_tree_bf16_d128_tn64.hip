// Trees of drafted tokens: element type bf16, head dim 128, plain form (64-row K/V tiles up to D = 128: see extra_flags in build.py).
#include "sdpa_tree_inst.h"

namespace tsdpa {
int launch_tree_bf16_d128_tn64(int tile_m, const LaunchArgs &a) { return launch_tree_plain<__bf16, 128>(tile_m, a); }
}  // namespace tsdpa
