// What the C entry points of the operators without a context share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "treelstm.h"

namespace tl {

// Compute units of the current device (asked for once per device).
inline int compute_units()
{
    static int known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
    if (dev < 64 && __atomic_load_n(&known[dev], __ATOMIC_RELAXED)) return __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
    if (dev < 64) __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
    return n;
}

inline bool is_dtype(int dtype) { return dtype >= TL_DT_F32 && dtype <= TL_DT_F16; }
inline int element_size(int dtype) { return dtype == TL_DT_F32 ? 4 : 2; }
inline long long round16(long long x) { return (x + 15) & ~15ll; }

// A launch has fewer than 2^32 threads in all.
constexpr long long most_blocks(int threads) { return (1ll << 32) / threads - 1; }

// Rows of `cols` elements, `row` elements apart; an output's rows must not overlap.
inline bool check_matrix(const void *p, long long row, int dtype, long long rows, long long cols, bool out)
{
    if (rows == 0) return true;
    if (!p || ((uintptr_t)p & (element_size(dtype) - 1)) || row < 0) return false;
    return !out || rows <= 1 || row >= cols;
}

}  // namespace tl
