// Attention kernels, bf16.
#include "attend_launch.hpp"

namespace tl {
ATT_INSTANCES(bf16_t)
}  // namespace tl
