// Dropout whose mask is made anew wherever it is needed: y = residual + [kept] x 65536 / (65536 - t).
//
// Numbers: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3, 2011).  A counter of four words is put through ten
// rounds, each of two products of 32 by 32 bits whose high halves are mixed with the other words and a key that grows by a constant.  Counter
// (column / 8, row, step, step >> 32) under the key (seed, seed >> 32) gives 128 bits: eight pieces of 16 bits, low halves first, for eight columns side by
// side.  A value is dropped where its piece is below t = rint(65536 p).  16 bits instead of 32: half the products a value, which are what bounds the
// call at 16-bit types; the share of dropped values is then a multiple of 2^-16, and the factor is that share's own, so that the expectation is exact.
#pragma once

#include "stream.hpp"

namespace tl {

constexpr int DRO_THREADS = 256;

struct DropArgs {
    const void *x, *residual;
    void *y;
    long long x_row, r_row, y_row;
    const uint64_t *numbers;                    // seed, step
    long long first, end;                       // rows of the launch
    int cols, blocks;                           // blocks: of eight columns
    uint32_t t;
    float scale;
};

__device__ inline u32x4 dro_philox(u32x4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c = u32x4{(uint32_t)(b >> 32) ^ c[1] ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c[3] ^ k1, (uint32_t)a};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// A thread: eight columns of a row.
template <typename T, bool RESIDUAL, bool ONCE> __global__ __launch_bounds__(DRO_THREADS) void k_dropout(DropArgs a)
{
    struct __attribute__((packed, aligned(sizeof(T)))) Eight {
        T v[8];
    };
    const uint64_t seed = a.numbers[0], step = a.numbers[1];
    // thread numbers of a launch pass 32 bits nowhere; the workgroup's first one is divided once, its lanes add less than a workgroup
    const uint32_t begin = blockIdx.x * (uint32_t)DRO_THREADS, row0 = begin / (uint32_t)a.blocks;
    uint32_t block = begin - row0 * a.blocks + threadIdx.x;
    const uint32_t more = block / (uint32_t)a.blocks;
    block -= more * a.blocks;
    const long long row = a.first + row0 + more;
    if (row >= a.end) return;
    const int col = (int)block * 8, n = min(8, a.cols - col);
    const T *const x = static_cast<const T *>(a.x) + row * a.x_row + col;
    const T *const r = RESIDUAL ? static_cast<const T *>(a.residual) + row * a.r_row + col : nullptr;
    T *const y = static_cast<T *>(a.y) + row * a.y_row + col;
    Eight v, old = {};                                          // (read before the numbers are made: the rounds run while the values come)
    if (n == 8) {
        stream_load<ONCE>(v, x);
        if (RESIDUAL) stream_load<ONCE>(old, r);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v.v[j] = j < n ? x[j] : (T)0.f;
            if (RESIDUAL) old.v[j] = j < n ? r[j] : (T)0.f;
        }
    }
    const u32x4 w = dro_philox(u32x4{block, (uint32_t)row, (uint32_t)step, (uint32_t)(step >> 32)}, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t piece = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
        const float s = piece < a.t ? 0.f : (float)v.v[j] * a.scale;
        v.v[j] = (T)(RESIDUAL ? (float)old.v[j] + s : s);
    }
    if (n == 8) {
        *reinterpret_cast<Eight *>(y) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) y[j] = v.v[j];
    }
}

}  // namespace tl
