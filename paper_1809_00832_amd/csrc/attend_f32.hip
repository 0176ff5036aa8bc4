// Attention kernels, f32.
#include "attend_launch.hpp"

namespace tl {
ATT_INSTANCES(float)
}  // namespace tl
