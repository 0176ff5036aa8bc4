// Attention kernels, f16.
#include "attend_launch.hpp"

namespace tl {
ATT_INSTANCES(f16_t)
}  // namespace tl
