#include "qk_rope_kernel.h"

namespace tsdpa {
int launch_rope_bf16(int D, bool cache, const RopeArgs &a) { return launch_rope<__bf16>(D, cache, a); }
int launch_rope_bwd_bf16(int D, const RopeArgs &a) { return launch_rope_bwd<__bf16>(D, a); }
}  // namespace tsdpa
