#include <mutex>

#include "sdpa_cache8_rows_kernel.h"

namespace tsdpa {
int launch_cache8_rows_f16(int D, const Cache8Attend &x) { return launch_cache8_rows<_Float16>(D, x); }
}  // namespace tsdpa
