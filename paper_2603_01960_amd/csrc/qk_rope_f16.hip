#include "qk_rope_kernel.h"

namespace tsdpa {
int launch_rope_f16(int D, bool cache, const RopeArgs &a) { return launch_rope<_Float16>(D, cache, a); }
int launch_rope_bwd_f16(int D, const RopeArgs &a) { return launch_rope_bwd<_Float16>(D, a); }
}  // namespace tsdpa
