#include <mutex>

#include "sdpa_cache8_rows_kernel.h"

namespace tsdpa {
int launch_cache8_rows_bf16(int D, const Cache8Attend &x) { return launch_cache8_rows<__bf16>(D, x); }
}  // namespace tsdpa
