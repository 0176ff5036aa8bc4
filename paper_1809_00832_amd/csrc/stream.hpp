// Reads and writes of 16-byte pieces at any address of a type, kept in the caches or past them.
#pragma once

#include "attend.hpp"

namespace tl {

// ONCE: what is read or written needs no place in the caches (non-temporal instructions).
template <bool ONCE, typename P, typename T> __device__ inline void stream_load(P &to, const T *from)
{
    typedef u32x4 __attribute__((aligned(2))) Words;
    static_assert(sizeof(P) % 16 == 0, "whole pieces");
    if constexpr (ONCE) {
        u32x4 w[sizeof(P) / 16];
#pragma unroll
        for (size_t i = 0; i < sizeof(P) / 16; ++i) w[i] = __builtin_nontemporal_load(reinterpret_cast<const Words *>(from) + i);
        __builtin_memcpy(&to, w, sizeof(P));
    } else {
        __builtin_memcpy(&to, reinterpret_cast<const P *>(from), sizeof(P));
    }
}
template <bool ONCE, typename P, typename T> __device__ inline void stream_store(T *to, const P &from)
{
    typedef u32x4 __attribute__((aligned(2))) Words;
    static_assert(sizeof(P) % 16 == 0, "whole pieces");
    if constexpr (ONCE) {
        u32x4 w[sizeof(P) / 16];
        __builtin_memcpy(w, &from, sizeof(P));
#pragma unroll
        for (size_t i = 0; i < sizeof(P) / 16; ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<Words *>(to) + i);
    } else {
        __builtin_memcpy(reinterpret_cast<P *>(to), &from, sizeof(P));
    }
}

}  // namespace tl
