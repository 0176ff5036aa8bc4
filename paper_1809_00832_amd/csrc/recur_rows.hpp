// Places of the recurrence that are counted in 64 bits, as plain C++.
#pragma once

namespace tl {

// Rows behind the last sentence: every wave clears each W slots-th one from a row of its own on.  (`tail` may be all but 2^31 and slots some 10^6: their sum is none of 32 bits.)
constexpr long long rec_behind(int tail, int slot, int wave, int slots) { return (long long)tail + slot + (long long)wave * slots; }

}  // namespace tl
