// One word per row of logits: temperature, top-k, top-p, min-p, then the inverse of the distribution function at a given number.
//
//   w_j = exp((x_j - max x) / T);  words in order of x, equal ones by index.  top-k keeps the first k of them; top-p, of those, each whose
//   mass before it is below p times their total; min-p those with w_j >= min_p.  The word drawn is the first one, by index, at
//   which the running sum of the kept weights exceeds u times their total.
//
// Which word that is hangs on sums over the whole row, so weights are taken in 64 bits and summed as whole multiples of 2^-shift (62
// bits for the sum of all): integers add up to the same total in any order, so that the result does not depend on which thread
// adds first.  No row is sorted: the last word that top-k or top-p keeps is found digit by digit (11 bits at a time) from histograms of
// counts and of weights over the ordered bit patterns of the logits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend.hpp"

namespace tl {

constexpr int SMP_THREADS = 1024;
constexpr int SMP_WAVES = SMP_THREADS / 64;
constexpr int SMP_BINS = 2048;
constexpr int SMP_TILE = SMP_THREADS * 4;       // words that a workgroup looks at in one step
constexpr int SMP_CHUNKS = 256;                 // pieces of a row whose weights are summed apart

struct SampleArgs {
    const void *logits;
    long long row;                              // elements from one row to the next
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    int vocab;
    int shift;                                  // weights are multiples of 2^-shift
    int vec;
};

// Bit patterns in the order of the values; -0 as 0, NaN as -infinity.
__device__ inline uint32_t smp_key(float x)
{
    x = x != x ? -INFINITY : x + 0.f;
    const uint32_t b = __float_as_uint(x);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ inline float smp_value(uint32_t key) { return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t SMP_KEY_NONE = 0x007fffffu;  // of -infinity

struct SmpWeight {
    double inv_t, max, one;
    uint32_t max_key;
    // (x - max) / T of a word above -infinity; beside a word at +infinity the others have no weight
    __device__ double exponent(uint32_t key) const
    {
        if (key == max_key) return 0.;
        return max == INFINITY ? -INFINITY : ((double)smp_value(key) - max) * inv_t;
    }
    // in units of 2^-shift
    __device__ uint64_t operator()(uint32_t key) const
    {
        if (key <= SMP_KEY_NONE) return 0;
        return (uint64_t)(exp(exponent(key)) * one + 0.5);
    }
};

template <typename V> __device__ inline V smp_wave_sum(V x)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Sum over the threads in front of this one (exclusive) and over all; `tmp` has SMP_WAVES words.  Everyone must call it.
template <typename V> __device__ inline V smp_scan(V x, V *tmp, V *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    V s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const V y = __shfl_up(s, o);
        if (lane >= o) s += y;
    }
    __syncthreads();
    if (lane == 63) tmp[wave] = s;
    __syncthreads();
    V before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < SMP_WAVES; ++w) {
        if (w < wave) before += tmp[w];
        all += tmp[w];
    }
    *total = all;
    return before + s - x;
}

struct SmpShared {
    uint64_t mass[SMP_BINS];
    uint32_t count[SMP_BINS];
    uint64_t chunk[SMP_CHUNKS];
    uint64_t tmp[SMP_WAVES];
    uint64_t tmp2[SMP_WAVES];
    uint64_t out[4];
    uint64_t best;
};

template <typename T> struct SmpRow {
    const T *p;
    int n, vec;
    // the four words from j on (keys; 0, which is no value's key, beyond the row)
    __device__ void keys4(int j, uint32_t (&k)[4]) const
    {
        if (vec && j + 3 < n) {
            T x[4];
            __builtin_memcpy(x, __builtin_assume_aligned(p + j, 4 * sizeof(T)), 4 * sizeof(T));
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = smp_key((float)x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = j + i < n ? smp_key((float)p[j + i]) : 0u;
        }
    }
};

// The last word, in the order of the values, that a filter keeps: its key, and how many of the words with that key it keeps.  BY_COUNT:
// the k-th word.  Else: the first word at which the running weight reaches `need`.  above: weight of the words with larger keys.
struct SmpCut {
    uint32_t key;
    uint32_t n, of;             // kept words with this key; all of them
    uint32_t count_above;
    uint64_t above;
};

template <typename T, bool BY_COUNT>
__device__ SmpCut smp_cut(const SmpRow<T> &row, const SmpWeight &weight, uint32_t k, double need, SmpShared &sh)
{
    constexpr int LEVELS = sizeof(T) == 4 ? 3 : 2;          // a 16-bit type's patterns end above the last 11 bits
    constexpr int shift_of[3] = {21, 10, 0};
    SmpCut c = {0, 0, 0, 0, 0};
    uint32_t prefix = 0;
    for (int level = 0; level < LEVELS; ++level) {
        const int sh_l = shift_of[level], bits = level == 2 ? 10 : 11, n_bins = 1 << bits;
        for (int b = threadIdx.x; b < n_bins; b += SMP_THREADS) {
            sh.mass[b] = 0;
            sh.count[b] = 0;
        }
        if (threadIdx.x == 0) sh.out[0] = ~0ull;
        __syncthreads();
        for (int j = threadIdx.x * 4; j < row.n; j += SMP_TILE) {
            uint32_t key[4];
            row.keys4(j, key);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (key[i] == 0u) continue;
                if (level > 0 && key[i] >> (sh_l + bits) != prefix) continue;
                const uint32_t b = key[i] >> sh_l & (n_bins - 1);
                atomicAdd(&sh.count[b], 1u);
                atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)weight(key[i]));
            }
        }
        __syncthreads();
        // from the largest key down: thread t holds bins n - 1 - 2 t and n - 2 - 2 t
        const int hi = n_bins - 1 - 2 * (int)threadIdx.x;
        const bool in = hi >= 0;
        const uint64_t m0 = in ? sh.mass[hi] : 0, m1 = in ? sh.mass[hi - 1] : 0;
        const uint32_t c0 = in ? sh.count[hi] : 0, c1 = in ? sh.count[hi - 1] : 0;
        uint64_t all_m, all_c;
        const uint64_t bm = smp_scan<uint64_t>(m0 + m1, sh.tmp, &all_m), bc = smp_scan<uint64_t>((uint64_t)c0 + c1, sh.tmp2, &all_c);
        // the first bin at which the bound is reached, or the last one that holds anything
        bool hit0, hit1;
        if (BY_COUNT) {
            hit0 = c0 && c.count_above + bc + c0 >= k;
            hit1 = c1 && c.count_above + bc + c0 + c1 >= k;
        } else {
            hit0 = c0 && ((double)(c.above + bm + m0) >= need || bc + c0 == all_c);
            hit1 = c1 && ((double)(c.above + bm + m0 + m1) >= need || bc + c0 + c1 == all_c);
        }
        if (hit0) atomicMin((unsigned long long *)&sh.out[0], (unsigned long long)(2 * threadIdx.x));
        else if (hit1) atomicMin((unsigned long long *)&sh.out[0], (unsigned long long)(2 * threadIdx.x + 1));
        __syncthreads();
        const uint64_t at = sh.out[0];
        if (at >> 1 == threadIdx.x) {
            sh.out[1] = at & 1 ? bm + m0 : bm;
            sh.out[2] = at & 1 ? bc + c0 : bc;
            sh.out[3] = at & 1 ? c1 : c0;
        }
        __syncthreads();
        c.above += sh.out[1];
        c.count_above += (uint32_t)sh.out[2];
        c.of = (uint32_t)sh.out[3];
        prefix = prefix << bits | (uint32_t)(n_bins - 1 - (int)at);
        __syncthreads();
    }
    c.key = prefix;
    if (LEVELS == 2) {
        // 22 bits of the pattern; the rest are all zeros, or all ones of a negative value
        c.key = prefix << 10;
        if (!(c.key >> 31)) c.key |= 0x3ffu;
    }
    if (BY_COUNT) {
        c.n = k - c.count_above;
    } else {
        const double w = (double)weight(c.key), left = need - (double)c.above;
        const double n = w > 0. ? ceil(left / w) : (double)c.of;
        c.n = n < 1. ? 1u : n > (double)c.of ? c.of : (uint32_t)n;
    }
    return c;
}

// The first word, by index, at which the running sum of f over the words in front of and at it exceeds `target(sum of all)`; also that
// sum.  -1 if it is never exceeded.
template <typename T, typename F, typename G>
__device__ int smp_locate(const SmpRow<T> &row, F f, G target, uint64_t *sum, SmpShared &sh)
{
    const int lane = threadIdx.x & 63;
    const int n_tiles = (row.n + SMP_TILE - 1) / SMP_TILE;
    const int per = (n_tiles + SMP_CHUNKS - 1) / SMP_CHUNKS;         // tiles of a chunk
    for (int b = threadIdx.x; b < SMP_CHUNKS; b += SMP_THREADS) sh.chunk[b] = 0;
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int j = t * SMP_TILE + threadIdx.x * 4;
        uint64_t s = 0;
        if (j < row.n) {
            uint32_t key[4];
            row.keys4(j, key);
#pragma unroll
            for (int i = 0; i < 4; ++i) s += key[i] ? f(key[i], j + i) : 0;
        }
        s = smp_wave_sum(s);
        if (lane == 0) atomicAdd((unsigned long long *)&sh.chunk[t / per], (unsigned long long)s);
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.out[0] = ~0ull;
    uint64_t all;
    const uint64_t mine = threadIdx.x < SMP_CHUNKS ? sh.chunk[threadIdx.x] : 0;
    const uint64_t before = smp_scan<uint64_t>(mine, sh.tmp, &all);
    const uint64_t goal = target(all);
    if (before <= goal && goal < before + mine) {
        sh.out[0] = threadIdx.x;
        sh.out[1] = before;
    }
    __syncthreads();
    *sum = all;
    const uint64_t chunk = sh.out[0];
    uint64_t run = sh.out[1];
    __syncthreads();
    if (chunk == ~0ull) return -1;
    if (threadIdx.x == 0) sh.out[0] = ~0ull;
    for (int t = (int)chunk * per; t < min((int)(chunk + 1) * per, n_tiles); ++t) {
        const int j = t * SMP_TILE + threadIdx.x * 4;
        uint64_t w[4] = {0, 0, 0, 0};
        if (j < row.n) {
            uint32_t key[4];
            row.keys4(j, key);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = key[i] ? f(key[i], j + i) : 0;
        }
        uint64_t here;
        uint64_t at = run + smp_scan<uint64_t>(w[0] + w[1] + w[2] + w[3], sh.tmp, &here);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at <= goal && goal < at + w[i]) sh.out[0] = (uint64_t)(j + i);
            at += w[i];
        }
        run += here;
        __syncthreads();
        if (run > goal) break;
    }
    const int found = (int)sh.out[0];
    __syncthreads();
    return found;
}

template <typename T> __global__ __launch_bounds__(SMP_THREADS) void k_sample(const SampleArgs a)
{
    __shared__ SmpShared sh;
    const int r = blockIdx.x;
    SmpRow<T> row;
    row.p = static_cast<const T *>(a.logits) + (long long)r * a.row;
    row.n = a.vocab;
    row.vec = a.vec;

    // the largest value and its first index: keys above, complements of the indexes below
    if (threadIdx.x == 0) sh.best = 0;
    __syncthreads();
    uint64_t best = 0;
    for (int j = threadIdx.x * 4; j < row.n; j += SMP_TILE) {
        uint32_t key[4];
        row.keys4(j, key);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t x = (uint64_t)key[i] << 32 | (uint32_t)~(j + i);
            best = x > best ? x : best;
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const uint64_t x = __shfl_xor(best, o);
        best = x > best ? x : best;
    }
    if ((threadIdx.x & 63) == 0) atomicMax((unsigned long long *)&sh.best, (unsigned long long)best);
    __syncthreads();
    best = sh.best;
    const uint32_t max_key = (uint32_t)(best >> 32);
    const float temperature = a.temperature ? a.temperature[r] : 1.f;
    if (max_key <= SMP_KEY_NONE || !(temperature > 0.f)) {
        const bool none = max_key <= SMP_KEY_NONE;
        if (threadIdx.x == 0) {
            a.token[r] = none ? -1 : (int32_t)~(uint32_t)best;
            if (a.logprob) a.logprob[r] = none ? -INFINITY : 0.f;
            if (a.kept) a.kept[r] = none ? 0 : 1;
        }
        return;
    }
    SmpWeight weight;
    weight.inv_t = 1. / (double)temperature;
    weight.max = (double)smp_value(max_key);
    weight.one = (double)(1ull << a.shift);
    weight.max_key = max_key;

    SmpCut cut = {SMP_KEY_NONE + 1, 0, 0, 0, 0};              // words with keys above, and cut.n of those with cut.key
    cut.n = cut.of = ~0u;
    uint64_t total = 0;
    bool have_total = false;
    const int k = a.top_k ? a.top_k[r] : 0;
    if (k > 0 && k < row.n) {
        cut = smp_cut<T, true>(row, weight, (uint32_t)k, 0., sh);
        if (cut.key <= SMP_KEY_NONE) {                        // fewer than k words above -infinity
            cut.key = SMP_KEY_NONE + 1;
            cut.n = cut.of = ~0u;
        } else {
            total = cut.above + cut.n * weight(cut.key);
            have_total = true;
        }
    }
    const float p = a.top_p ? a.top_p[r] : 1.f;
    if (p < 1.f) {
        if (!have_total) {
            uint64_t s = 0;
            for (int j = threadIdx.x * 4; j < row.n; j += SMP_TILE) {
                uint32_t key[4];
                row.keys4(j, key);
#pragma unroll
                for (int i = 0; i < 4; ++i) s += weight(key[i]);
            }
            smp_scan<uint64_t>(s, sh.tmp, &total);
            __syncthreads();
        }
        const SmpCut c = smp_cut<T, false>(row, weight, 0, (double)p * (double)total, sh);
        if (c.key > cut.key) cut = c;
        else if (c.key == cut.key) cut.n = min(cut.n, c.n);
    }
    // of words that tie at the cut, the first ones by index
    int last_tie = row.n;
    uint64_t sum;
    if (cut.n < cut.of) {
        const uint32_t key = cut.key;
        const uint64_t n = cut.n;
        last_tie = smp_locate(row, [key](uint32_t x, int) { return (uint64_t)(x == key); }, [n](uint64_t) { return n - 1; }, &sum, sh);
    }
    const double floor_e = a.min_p ? log((double)a.min_p[r]) : -INFINITY;      // w >= min_p, of the exponents (a NaN keeps every word)
    const double u = (double)a.u[r];
    uint32_t n_kept = 0;
    bool counting = true;
    auto kept_weight = [&](uint32_t key, int j) -> uint64_t {
        if (key < cut.key || (key == cut.key && j > last_tie)) return 0;
        if (key != max_key && weight.exponent(key) < floor_e) return 0;
        if (counting) ++n_kept;
        return weight(key);
    };
    int token = smp_locate(row, kept_weight, [&](uint64_t s) {
        counting = false;
        const double x = u * (double)s;
        const uint64_t t = x > 0. ? (uint64_t)x : 0;
        return t >= s ? s - 1 : t;
    }, &sum, sh);
    uint32_t all_kept;
    smp_scan<uint32_t>(n_kept, (uint32_t *)sh.tmp2, &all_kept);
    if (threadIdx.x == 0) {
        a.token[r] = token;
        if (a.logprob) a.logprob[r] = (float)log((double)weight(smp_key((float)row.p[token])) / (double)sum);
        if (a.kept) a.kept[r] = (int32_t)all_kept;
    }
}

}  // namespace tl
