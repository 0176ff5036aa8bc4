// One word per row of logits: temperature, top-k, top-p, min-p, then the inverse of the distribution function at a given number.
//
//   w_j = exp((x_j - max x) / T);  words in order of x, equal ones by index.  top-k keeps the first k of them; top-p, of those, each whose
//   mass before it is below p times their total; min-p those with w_j >= min_p.  The word drawn is the first one, by index, at
//   which the running sum of the kept weights exceeds u times their total.
//
// Which word that is hangs on sums over the whole row, so weights are taken in 64 bits and summed as whole multiples of 2^-shift (62
// bits for the sum of all): integers add up to the same total in any order, so the result does not depend on which thread adds
// first.  No row is sorted.  One workgroup walks a row two to four times: the largest and smallest value; a histogram over 2048 equal
// steps of the value; the words of the step in which a filter ends, which are sorted in LDS; the kept weights per piece
// of the row, of which one wave then walks the piece that holds the draw.  (Without top-k and top-p the second and third are left out; both with more words
// than the list holds: six walks; 16-bit rows with a NaN: one more; each filter that goes by digits, below: two to four more.)  Equal steps of the value spread a row's words evenly enough that the
// additions of a wave seldom meet in one counter, which steps of the bit pattern do not (few exponents).  top-k counts words,
// which needs no weights, and where it leaves no more words than the list holds, top-p is answered from the list; else a histogram
// of weights follows.  A step that holds more words than the list (long runs of equal values) is resolved digit by digit of the bit pattern.
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attend.hpp"

namespace tl {

constexpr int SMP_THREADS = 1024;
constexpr int SMP_WAVES = SMP_THREADS / 64;
constexpr int SMP_BINS = 2048;
constexpr int SMP_LIST = 4096;                  // words of one step that are sorted in LDS; also the pieces of a row whose weights are summed apart
constexpr int SMP_VALUES = 4096;                // bf16: values whose words are counted one by one
constexpr double SMP_REACH = 40.;               // steps cover weights down to e^-40; what lies below is in the last one

struct SampleArgs {
    const void *logits;
    long long row;                              // elements from one row to the next
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *token, *kept;
    float *logprob;
    int vocab;
    int shift;                                  // weights are multiples of 2^-shift, shift <= 51
};

struct SmpShared {
    union {
        struct {
            uint64_t mass[SMP_BINS];
            uint32_t count[SMP_BINS];
        };
        uint64_t piece[SMP_LIST];               // (the histogram is over when the pieces are summed)
    };
    union {
        uint64_t list[SMP_LIST];
        uint32_t equal[SMP_VALUES];             // bf16: words of each value (see smp_histogram)
        float packed[SMP_WAVES][512];           // kept words of a wave's piece, side by side
    };
    uint64_t tmp[SMP_WAVES];
    uint64_t out[4];
    uint64_t best;
    uint32_t low, listed, kept;
};
extern __shared__ __align__(16) unsigned char smp_lds[];
__device__ inline SmpShared &smp_shared() { return *reinterpret_cast<SmpShared *>(smp_lds); }

// The phases are functions of their own, called, so that each has the registers to itself (inlined into one kernel they spill); what they are
// given is the same in every lane, and is put into scalar registers again.
template <typename S> __device__ inline S smp_uniform(S x)
{
    static_assert(sizeof(S) % 4 == 0, "whole words");
    uint32_t w[sizeof(S) / 4];
    __builtin_memcpy(w, &x, sizeof(S));
#pragma unroll
    for (size_t i = 0; i < sizeof(S) / 4; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    __builtin_memcpy(&x, w, sizeof(S));
    return x;
}

// Bit patterns in the order of the values (of numbers; -0 as 0).
constexpr uint32_t SMP_KEY_NONE = 0x007fffffu;  // of -infinity
__device__ inline uint32_t smp_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ inline float smp_value(uint32_t key) { return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xffffffffu)); }

// log2 of a word's weight is (x - max) per_t.  Where a word is at +infinity, max lies far beyond all other words, so that they
// have no weight, and what is above 0 counts as 0.
struct SmpWeight {
    double per_t, max;                          // log2(e) / T, the row's largest value
    int shift, pad;
    __device__ double exponent(float x) const { return ((double)x - max) * per_t; }
};

// Weights in units of 2^-shift.  2^t = 2^k 2^r with k the nearest whole number to t, found by adding 1.5 * 2^52; 2^r on [-1/2, 1/2] as 1 + r q(r), q the
// polynomial of degree 8 through (2^r - 1) / r at the nine Chebyshev nodes: good to 4e-14, and exactly 1 at 0; adding 2^52 rounds to whole units and leaves them in the
// mantissa.  (A table of powers and a shorter polynomial would cost a scattered LDS read a word beside the histogram's additions.)
// The coefficients are made opaque so that they stay in scalar registers, where a multiply-add takes them from: the compiler would
// copy each to vector registers for each word.
struct SmpSeries {
    double c[10];
    SmpWeight w;
    __device__ explicit SmpSeries(const SmpWeight &weight)
        : c{1., 6.93147180559945286e-01, 2.40226506958129887e-01, 5.55041086647608192e-02, 9.61812915940255843e-03, 1.33335581789866269e-03,
            1.54034558524538382e-04, 1.52526868763930427e-05, 1.32552248786688168e-06, 1.02031157077784712e-07},
          w(weight)
    {
#pragma unroll
        for (int i = 0; i < 10; ++i) asm volatile("" : "+s"(c[i]));
    }
    // 0 for a NaN and for -infinity
    __device__ uint64_t operator()(float x) const
    {
        const double t = fmin(fmax(w.exponent(x), -64.), 0.);
        const double magic = 6755399441055744.;
        const double a = t + magic;
        const double r = t - (a - magic);
        double e = c[9];
#pragma unroll
        for (int i = 8; i >= 0; --i) e = fma(e, r, c[i]);
        const int k = (int)(uint32_t)__double_as_longlong(a);
        const uint64_t y = __double_as_longlong(e) + ((uint64_t)(uint32_t)(k + w.shift) << 52);
        return (uint64_t)__double_as_longlong(__longlong_as_double((long long)y) + 4503599627370496.) & 0xfffffffffffffull;
    }
};

// The share p of a sum, rounded down or up, exactly: a draw or a filter may end right at a border between words.
__device__ inline uint64_t smp_share(float p, uint64_t of, bool up)
{
    if (!(p > 0.f)) return 0;
    const uint32_t b = __float_as_uint(p), e = b >> 23;
    const uint64_t m = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
    const int s = 150 - (int)(e ? e : 1);                       // p = m 2^-s
    if (s <= 0) return ~0ull;                                   // (2^23 and more)
    const uint64_t lo = of * m, hi = __umul64hi(of, m);
    const uint64_t whole = s < 64 ? hi << (64 - s) | lo >> s : s < 128 ? hi >> (s - 64) : 0;
    const uint64_t rest = s < 64 ? lo << (64 - s) : lo | (s > 64 ? s < 128 ? hi << (128 - s) : hi : 0);
    return whole + (up && rest ? 1 : 0);
}

// ---- sums over lanes --------------------------------------------------------------------

// What lane l - n of the row of 16 (or the last lane of the rows in front) holds; zero where there is none.
template <int CTRL, int ROWS> __device__ inline uint64_t smp_from(uint64_t x)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}
__device__ inline uint64_t smp_row_scan(uint64_t x)
{
    x += smp_from<0x111, 0xf>(x);
    x += smp_from<0x112, 0xf>(x);
    x += smp_from<0x114, 0xf>(x);
    x += smp_from<0x118, 0xf>(x);
    return x;
}
// Sum over this lane and those in front of it.
__device__ inline uint64_t smp_wave_scan(uint64_t x)
{
    x = smp_row_scan(x);
    x += smp_from<0x142, 0xa>(x);
    x += smp_from<0x143, 0xc>(x);
    return x;
}
// The same for counts.
__device__ inline uint32_t smp_wave_count(uint32_t x)
{
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
    return x;
}
__device__ inline uint64_t smp_lane(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

// Sum over the threads in front of this one and over all.  Everyone must call it.
__device__ inline uint64_t smp_scan(uint64_t x, uint64_t *total, SmpShared &sh)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t s = smp_wave_scan(x);
    __syncthreads();
    if (lane == 63) sh.tmp[wave] = s;
    __syncthreads();
    const uint64_t w = smp_row_scan(sh.tmp[lane & (SMP_WAVES - 1)]);
    *total = smp_lane(w, SMP_WAVES - 1);
    return (wave ? smp_lane(w, wave - 1) : 0) + s - x;
}

// ---- a row ------------------------------------------------------------------------------

// A row, walked in steps of SMP_THREADS times W words, 16 bytes a thread; W words from a 16-byte boundary on, so that rows of any length
// and distance are read in such pieces.  Words outside the row read as -infinity.
template <typename T> struct SmpRow {
    static constexpr int W = 16 / (int)sizeof(T);
    static constexpr int STEP = SMP_THREADS * W;
    static constexpr int PIECE = 64 * W;        // words of a wave in one step
    static constexpr int BATCH = 4;             // requests in flight (a short row is bound by their latency)
    const T *p;
    int n, ahead;                               // words, and how many the first 16 bytes hold in front of them

    SmpRow() = default;
    __device__ SmpRow(const T *row, int words) : p(row), n(words), ahead((int)(((uintptr_t)row & 15) / sizeof(T))) {}
    __device__ int pieces() const { return (n + ahead + PIECE - 1) / PIECE; }
    // words j .. j + W - 1, as they are
    __device__ void raw(int j, T (&v)[W]) const
    {
        typedef const __attribute__((address_space(1))) T *global;
        const global g = (global)p;
        if (j >= 0 && j + W <= n) {
            const u32x4 x = *(const __attribute__((address_space(1))) u32x4 *)(g + j);
            __builtin_memcpy(v, &x, 16);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const T x = g[min(max(j + i, 0), n - 1)];
                v[i] = (unsigned)(j + i) < (unsigned)n ? x : (T)-INFINITY;
            }
        }
    }
    // f(W words, index of the first, piece); every lane of a wave calls it equally often.
    template <typename F> __device__ void each(F f) const
    {
        each_raw([&](const T (&v)[W], int j, int q) {
            float x[W];
#pragma unroll
            for (int i = 0; i < W; ++i) x[i] = (float)v[i];
            f(x, j, q);
        });
    }
    template <typename F> __device__ void each_raw(F f) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_pieces = pieces();
        for (int q = wave; q < n_pieces; q += BATCH * SMP_WAVES) {
            const int j = (q * 64 + (int)(threadIdx.x & 63)) * W - ahead;
            T v[BATCH][W];
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (q + b * SMP_WAVES < n_pieces) raw(j + b * STEP, v[b]);
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (q + b * SMP_WAVES < n_pieces) f(v[b], j + b * STEP, q + b * SMP_WAVES);
        }
    }
};

// The last word that a filter keeps, in the order of values and indexes: a word is kept if it stands at or before it.
struct SmpCut {
    float x;
    int j;
    uint64_t mass;              // weight of the words up to it
    __device__ bool keeps(float y, int i) const { return (y > x) | ((y == x) & (i <= j)); }
};

// ---- the cut ----------------------------------------------------------------------------

// Step of a value: 0 for the largest, never smaller for a smaller one.  (+infinity is in front of the largest number; a NaN's step is not asked for.)
struct SmpSteps {
    float max, per;
    __device__ float place(float x) const { return __builtin_amdgcn_fmed3f((max - x) * per, 0.f, (float)(SMP_BINS - 1)); }
    __device__ int operator()(float x) const { return (int)place(x); }
};

// The histogram of weights of a long row of bf16: a row's words share few values, so words are counted per value and a weight is worked out once for each
// value that occurs.  Counted are magnitudes of 2^-10 to 2^6; the few words outside that have a weight at all are added by themselves.  The sums are whole
// numbers, so they are the same as word by word.  (A word costs some 9 instructions instead of 30: 512 rows of 131 072, top-p alone, 168 -> 142 us.  The same
// rows 60 or 100 higher, where bf16 has few values: 530 and 960, word by word 555 and 929, most of it additions that meet in one counter.)
static __device__ void smp_histogram_of_values(const SmpRow<bf16_t> &row, const SmpWeight &weight, const SmpSteps &step)
{
    constexpr int W = SmpRow<bf16_t>::W;
    constexpr uint32_t LOW = 0x3a80, HALF = SMP_VALUES / 2;     // 2^-10; values of one sign
    SmpShared &sh = smp_shared();
    for (int b = threadIdx.x; b < SMP_VALUES; b += SMP_THREADS) sh.equal[b] = 0;
    __syncthreads();
    const SmpSeries series(weight);
    // far below the largest value weights are zero (2^-64 and less)
    const float skip = weight.max < 1e300 ? fmaxf((float)(weight.max - 64. / weight.per_t), -FLT_MAX) : -FLT_MAX;
    row.each_raw([&](const bf16_t (&v)[W], int j, int) {
        unsigned others = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint32_t bits = __builtin_bit_cast(uint16_t, v[i]), at = (bits & 0x7fffu) - LOW;
            if (at < HALF) atomicAdd(&sh.equal[at | (bits >> 15) * HALF], 1u);
            else others |= (float)v[i] >= skip ? 1u << i : 0u;
        }
        while (others) {
            const float x = (float)row.p[j + __ffs(others) - 1];
            others &= others - 1;
            const uint64_t w = series(x);
            if (w) atomicAdd((unsigned long long *)&sh.mass[step(x)], (unsigned long long)w);
        }
    });
    __syncthreads();
    for (int b = threadIdx.x; b < SMP_VALUES; b += SMP_THREADS) {
        const uint32_t n = sh.equal[b];
        if (!n) continue;
        const float x = __uint_as_float(((uint32_t)b % HALF + LOW) << 16 | ((uint32_t)b / HALF) << 31);
        const uint64_t w = series(x) * n;
        if (w) atomicAdd((unsigned long long *)&sh.mass[step(x)], (unsigned long long)w);
    }
    __syncthreads();
}

// Histogram over the steps: of the words above -infinity, or of the weights.
template <typename T, bool BY_COUNT> __device__ __noinline__ void smp_histogram(SmpRow<T> row, SmpWeight weight, SmpSteps step)
{
    constexpr int W = SmpRow<T>::W;
    SmpShared &sh = smp_shared();
    row = smp_uniform(row);
    weight = smp_uniform(weight);
    step = smp_uniform(step);
    __syncthreads();
    for (int b = threadIdx.x; b < SMP_BINS; b += SMP_THREADS) {
        if (BY_COUNT) sh.count[b] = 0;
        else sh.mass[b] = 0;
    }
    __syncthreads();
    const SmpSeries series(weight);
    if constexpr (!BY_COUNT && std::is_same<T, bf16_t>::value) {
        if (row.n >= 2 * SMP_VALUES) {
            smp_histogram_of_values(row, weight, step);
            return;
        }
    }
    row.each([&](const float (&x)[W], int, int) {
        uint64_t w[W];
        if (!BY_COUNT) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = series(x[i]);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int b = step(x[i]);
            if (BY_COUNT) {
                if (x[i] > -INFINITY) atomicAdd(&sh.count[b], 1u);
            } else {
                if (w[i]) atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)w[i]);
            }
        }
    });
    __syncthreads();
}

// The first step, from the largest values on, at which `goal` words are reached, or the share `p` of the weight `of` (0: of the whole); the last one that
// holds anything where they never are.
struct SmpAt {
    int at;
    uint32_t here;              // BY_COUNT: words in it
    uint64_t above;             // in the steps in front of it
    uint64_t need;              // weight that is to be reached
};
template <bool BY_COUNT> __device__ __noinline__ SmpAt smp_step(uint32_t goal, float p, uint64_t of)
{
    SmpShared &sh = smp_shared();
    goal = smp_uniform(goal);
    p = smp_uniform(p);
    of = smp_uniform(of);
    const int b = 2 * threadIdx.x;
    const uint64_t m0 = BY_COUNT ? sh.count[b] : sh.mass[b], m1 = BY_COUNT ? sh.count[b + 1] : sh.mass[b + 1];
    uint64_t all;
    const uint64_t before = smp_scan(m0 + m1, &all, sh);
    const uint64_t at0 = before + m0, at1 = at0 + m1;
    const uint64_t need = smp_share(p, of ? of : all, true);
    auto short_of = [&](uint64_t x) { return x == 0 || (BY_COUNT ? x < goal : x < need); };
    // (one step alone: sums in front of it fall short, its own reaches or is the last)
    if (m0 && short_of(before) && (!short_of(at0) || at0 == all)) {
        sh.out[0] = b;
        sh.out[1] = before;
    }
    if (m1 && short_of(at0) && (!short_of(at1) || at1 == all)) {
        sh.out[0] = b + 1;
        sh.out[1] = at0;
    }
    __syncthreads();
    const int at = (int)sh.out[0];
    const SmpAt r = {at, BY_COUNT ? sh.count[at] : 0, sh.out[1], need};
    __syncthreads();
    return r;
}

// Lists the words of steps from .. to; how many they are (beyond SMP_LIST: not all are listed).
template <typename T> __device__ __noinline__ int smp_collect(SmpRow<T> row, SmpSteps step, int from, int to)
{
    constexpr int W = SmpRow<T>::W;
    SmpShared &sh = smp_shared();
    row = smp_uniform(row);
    step = smp_uniform(step);
    const float first = (float)smp_uniform(from), behind = (float)smp_uniform(to) + 1.f;
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    row.each([&](const float (&x)[W], int j, int) {
        unsigned hit = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float at = step.place(x[i]);
            hit |= (at >= first) & (at < behind) & (x[i] > -INFINITY) ? 1u << i : 0u;
        }
        if (__any(hit != 0)) {
            const uint32_t upto = smp_wave_count(__popc(hit)), all = __builtin_amdgcn_readlane(upto, 63);
            uint32_t at = 0;
            if ((threadIdx.x & 63) == 0) at = atomicAdd(&sh.listed, all);
            at = __builtin_amdgcn_readfirstlane(at) + upto - __popc(hit);
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (hit >> i & 1) {
                    if (at < SMP_LIST) sh.list[at] = (uint64_t)smp_key(x[i]) << 32 | (uint32_t)~(j + i);
                    ++at;
                }
        }
    });
    __syncthreads();
    return (int)sh.listed;
}

// Sorts the list by value, then index: a few words by how many are larger; else exchanges at a distance below 64 stay within a wave, without barriers.
static __device__ __noinline__ void smp_sort(int n)
{
    SmpShared &sh = smp_shared();
    n = smp_uniform(n);
    const int lane = threadIdx.x & 63;
    if (n <= 64) {
        if (threadIdx.x < 64) {
            const uint64_t mine = lane < n ? sh.list[lane] : 0;
            int larger = 0;
            for (int i = 0; i < n; ++i) larger += smp_lane(mine, i) > mine ? 1 : 0;
            __builtin_amdgcn_wave_barrier();
            if (lane < n) sh.list[larger] = mine;
        }
        __syncthreads();
        return;
    }
    int size = 64;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += SMP_THREADS) sh.list[i] = 0;
    for (int run = 64; run <= size; run *= 2) {
        for (int d = run / 2; d >= 64; d /= 2) {
            __syncthreads();
            for (int e = threadIdx.x; e < size / 2; e += SMP_THREADS) {
                const int i = 2 * e - (e & (d - 1)), o = i + d;
                const uint64_t a = sh.list[i], b = sh.list[o];
                if ((a < b) == ((i & run) == 0)) {
                    sh.list[i] = b;
                    sh.list[o] = a;
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < size; i += SMP_THREADS) {
            uint64_t a = sh.list[i];
            for (int r = run == 64 ? 2 : run; r <= run; r *= 2)          // (the first 21 stages are one walk within waves)
                for (int d = min(r / 2, 32); d >= 1; d /= 2) {
                    const uint64_t b = __shfl_xor(a, d);
                    // the lower place of a pair keeps the larger one where its run descends
                    const bool keep_larger = ((lane & d) == 0) == ((i & r) == 0);
                    a = (a > b) == keep_larger ? a : b;
                }
            sh.list[i] = a;
        }
    }
    __syncthreads();
}

// The cut inside a sorted list of n words that stand behind `count_above` words of weight `above`.
template <bool BY_COUNT> __device__ __noinline__ SmpCut smp_cut_list(int n, SmpWeight weight, uint32_t k, uint64_t need, uint64_t above, uint32_t count_above)
{
    SmpShared &sh = smp_shared();
    n = smp_uniform(n);
    const SmpSeries series(smp_uniform(weight));
    constexpr int EACH = SMP_LIST / SMP_THREADS;
    uint64_t w[EACH] = {}, s = 0;
    if (EACH * ((int)threadIdx.x & ~63) < n) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = EACH * threadIdx.x + i;
            const uint64_t y = series(smp_value((uint32_t)(sh.list[e] >> 32)));
            s += w[i] = e < n ? y : 0;
        }
    }
    uint64_t all;
    uint64_t run = above + smp_scan(s, &all, sh);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = EACH * threadIdx.x + i;
        const bool short_before = e == 0 || (BY_COUNT ? count_above + (uint32_t)e < k : run < need);
        run += w[i];
        const bool reached = BY_COUNT ? count_above + (uint32_t)e + 1 >= k : run >= need;
        if (e < n && short_before && (reached || e == n - 1)) {
            sh.out[0] = e;
            sh.out[1] = run;
        }
    }
    __syncthreads();
    const uint64_t e = sh.list[sh.out[0]];
    const SmpCut c = {smp_value((uint32_t)(e >> 32)), (int)~(uint32_t)e, sh.out[1]};
    __syncthreads();
    return c;
}

// The least value above -infinity whose exponent is not below `least`, for a `least` up to 0: a search over the bit patterns, 64 at a time.
__device__ inline float smp_least_value(const SmpWeight &weight, float max, double least)
{
    uint32_t lo = SMP_KEY_NONE + 1, hi = smp_key(max);                   // hi fits
    while (lo < hi) {
        const uint32_t step = (hi - lo) / 64 + 1;
        const uint64_t at = (uint64_t)lo + (uint64_t)step * (threadIdx.x & 63);
        const bool fits = at >= hi || !(weight.exponent(smp_value((uint32_t)at)) < least);
        const int first = __ffsll(__ballot(fits)) - 1;                   // 0: lo itself; -1: beyond the last one
        if (first == 0) return smp_value(lo);
        const uint64_t below = (uint64_t)lo + (uint64_t)step * (first < 0 ? 63 : first - 1);
        if (first >= 0) hi = (uint32_t)min((uint64_t)hi, below + step);
        lo = (uint32_t)below + 1;
    }
    return smp_value(lo);
}

// ---- the draw ---------------------------------------------------------------------------

// The words that add to the running sum in which the draw is located: with their weights, those that the filters keep; or, to find one of many
// equal words, each of these with one.
struct SmpKept {
    SmpCut cut;
    SmpWeight weight;
    float u;                    // the draw, a share of the sum
    int equal;                  // or 1 + which of the equal words
    __device__ bool operator()(float x, int j) const { return cut.keeps(x, j) & ((x == cut.x) | !equal); }
};

struct SmpDraw {
    int word, kept;
    uint64_t sum, weight;       // of all, of the word
};

// The word, by index, at which the running sum first exceeds the draw; the sum of all and how many words add to it.
template <typename T> __device__ __noinline__ SmpDraw smp_locate(SmpRow<T> row, SmpKept f)
{
    typedef SmpRow<T> R;
    constexpr int W = R::W;
    SmpShared &sh = smp_shared();
    row = smp_uniform(row);
    f = smp_uniform(f);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_pieces = row.pieces();
    int group = 0;                                              // 2^group pieces are summed together
    while (n_pieces >> group >= SMP_LIST) ++group;
    __syncthreads();
    for (int i = threadIdx.x; i <= n_pieces >> group; i += SMP_THREADS) sh.piece[i] = 0;
    if (threadIdx.x == 0) {
        sh.out[0] = ~0ull;
        sh.kept = 0;
    }
    __syncthreads();
    const SmpSeries series(f.weight);
    const float above_cut = smp_value(smp_key(f.cut.x) + 1);   // the next larger value (of +infinity: a NaN)
    uint32_t kept = 0;
    row.each([&](const float (&x)[W], int j, int q) {
        unsigned mine = 0;
        const int first = q * R::PIECE - row.ahead;
        if (f.equal || (f.cut.j >= first && f.cut.j < first + R::PIECE)) {
#pragma unroll
            for (int i = 0; i < W; ++i) mine |= f(x[i], j + i) ? 1u << i : 0u;
        } else {
            // (the piece stands on one side of the cut's index: equal values are kept, or not)
            const float least = first <= f.cut.j ? f.cut.x : above_cut;
#pragma unroll
            for (int i = 0; i < W; ++i) mine |= x[i] >= least ? 1u << i : 0u;
        }
        if (!__any(mine != 0)) return;
        const uint32_t count = __popc(mine), upto = smp_wave_count(count), all = __builtin_amdgcn_readlane(upto, 63);
        kept += all;
        uint64_t s = 0;
        if (f.equal) {
            s = count;
        } else if (4 * all > 3 * R::PIECE) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint64_t y = series(x[i]);
                s += mine >> i & 1 ? y : 0;
            }
        } else {
            // few: put side by side first, so that a weight is worked out for them alone
            float *packed = sh.packed[wave];
            uint32_t at = upto - count;
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (mine >> i & 1) packed[at++] = x[i];
            __builtin_amdgcn_wave_barrier();
            for (uint32_t e = lane; e < ((all + 63) & ~63u); e += 64) {
                const uint64_t y = series(e < all ? packed[e] : -INFINITY);
                s += y;
            }
            __builtin_amdgcn_wave_barrier();
        }
        s = smp_lane(smp_wave_scan(s), 63);
        if (lane == 0) atomicAdd((unsigned long long *)&sh.piece[q >> group], (unsigned long long)s);
    });
    if (lane == 0) atomicAdd(&sh.kept, kept);
    __syncthreads();
    constexpr int EACH = SMP_LIST / SMP_THREADS;
    uint64_t w[EACH], s = 0, all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = EACH * threadIdx.x + i;
        s += w[i] = e <= n_pieces >> group ? sh.piece[e] : 0;
    }
    uint64_t run = smp_scan(s, &all, sh);
    // exceeded for good: the largest whole number below what the sum has to pass
    uint64_t goal = 0;
    if (f.equal) {
        goal = (uint64_t)f.equal - 1;
    } else {
        goal = smp_share(f.u, all, false);
        goal = goal >= all ? all - 1 : goal;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (run <= goal && goal < run + w[i]) {
            sh.out[0] = EACH * threadIdx.x + i;
            sh.out[1] = run;
        }
        run += w[i];
    }
    __syncthreads();
    SmpDraw d = {0, (int)sh.kept, all, 0};
    const uint64_t hit = sh.out[0];
    if (hit == ~0ull) return d;
    if (wave == 0) {
        uint64_t at = sh.out[1];
        for (int q = (int)hit << group; q < min((int)(hit + 1) << group, n_pieces); ++q) {
            const int j = (q * 64 + lane) * W - row.ahead;
            T x[W];
            row.raw(j, x);
            uint64_t v[W], t = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint64_t y = f.equal ? 1 : series((float)x[i]);
                t += v[i] = f((float)x[i], j + i) ? y : 0;
            }
            const uint64_t scan = smp_wave_scan(t);
            uint64_t here = at + scan - t;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (here <= goal && goal < here + v[i]) {
                    sh.out[2] = (uint64_t)(j + i);
                    sh.out[3] = v[i];
                }
                here += v[i];
            }
            at += smp_lane(scan, 63);
            if (at > goal) break;
        }
    }
    __syncthreads();
    d.word = (int)sh.out[2];
    d.weight = sh.out[3];
    __syncthreads();
    return d;
}

// The cut of any row, by the bit patterns of its values, 11, 11 and 10 bits at a time; for steps that hold more words than the list.
template <typename T, bool BY_COUNT> __device__ __noinline__ SmpCut smp_cut_by_digits(SmpRow<T> row, SmpWeight weight, uint32_t k, uint64_t need)
{
    constexpr int W = SmpRow<T>::W;
    SmpShared &sh = smp_shared();
    row = smp_uniform(row);
    weight = smp_uniform(weight);
    k = smp_uniform(k);
    need = smp_uniform(need);
    const SmpSeries series(weight);
    uint32_t prefix = 0, count_above = 0, of = 0;
    uint64_t above = 0;
    for (int level = 0; level < 3; ++level) {
        const int sh_l = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11, n_bins = 1 << bits;
        __syncthreads();
        for (int b = threadIdx.x; b < SMP_BINS; b += SMP_THREADS) {
            sh.mass[b] = 0;
            sh.count[b] = 0;
        }
        __syncthreads();
        row.each([&](const float (&x)[W], int, int) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint32_t key = smp_key(x[i]);
                if (!(x[i] > -INFINITY) || (level > 0 && key >> (sh_l + bits) != prefix)) continue;
                const uint32_t b = n_bins - 1 - (key >> sh_l & (n_bins - 1));
                atomicAdd(&sh.count[b], 1u);
                atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)series(x[i]));
            }
        });
        __syncthreads();
        const SmpAt s = smp_step<BY_COUNT>(k - count_above, 1.f, BY_COUNT || need <= above ? 1 : need - above);
        uint64_t c = 0, m = 0, all_c, all_m;                    // of the larger digits
        for (int i = threadIdx.x; i < s.at; i += SMP_THREADS) {
            c += sh.count[i];
            m += sh.mass[i];
        }
        smp_scan(c, &all_c, sh);
        smp_scan(m, &all_m, sh);
        of = sh.count[s.at];
        above += all_m;
        count_above += (uint32_t)all_c;
        prefix = prefix << bits | (uint32_t)(n_bins - 1 - s.at);
    }
    SmpCut c = {smp_value(prefix), row.n, 0};
    const uint64_t w = series(c.x);
    uint32_t n = of;                                            // words of this value that are kept: the first ones by index
    if (BY_COUNT) {
        n = min(k - count_above, of);
    } else if (w) {
        const uint64_t left = need > above ? (need - above + w - 1) / w : 1;
        n = left > of ? of : (uint32_t)left;
    }
    c.mass = above + n * w;
    if (n < of) {
        SmpKept f = {};
        f.cut = c;
        f.equal = (int)n;
        c.j = smp_locate(row, f).word;
    }
    return c;
}

// The largest value (its key in the upper half of sh.best, which is zero where no word is above -infinity), with INDEX its first index (~ in the lower half), and the
// smallest value.  16-bit types without INDEX: whole numbers in the order of the values, two in an instruction; a row that holds a NaN is walked again.
template <typename T, bool INDEX> __device__ __noinline__ void smp_extremes(SmpRow<T> row)
{
    constexpr int W = SmpRow<T>::W;
    SmpShared &sh = smp_shared();
    row = smp_uniform(row);
    if (threadIdx.x == 0) {
        sh.best = 0;
        sh.low = ~0u;
        sh.kept = 0;
    }
    __syncthreads();
    float top = -INFINITY, low = INFINITY;
    int at = 0;
    bool done = false;
    if constexpr (sizeof(T) == 2 && !INDEX) {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
        constexpr short INF = std::is_same<T, bf16_t>::value ? 0x7f80 : 0x7c00, NEG_INF = (short)~INF;
        s16x2 high = {-32768, -32768}, least = {32767, 32767};
        row.each_raw([&](const T (&v)[W], int, int) {
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                const s16x2 b = {__builtin_bit_cast(short, v[i]), __builtin_bit_cast(short, v[i + 1])};
                const s16x2 key = b ^ ((b >> 15) & (short)0x7fff);
                high = __builtin_elementwise_max(high, key);
                least = __builtin_elementwise_min(least, key);
            }
        });
        const short h = high[0] > high[1] ? high[0] : high[1], l = least[0] < least[1] ? least[0] : least[1];
        // (a thread without words leaves the bounds)
        if (h >= l && (h > INF || l < NEG_INF)) sh.kept = 1;
        if (h >= l) {
            top = (float)__builtin_bit_cast(T, (short)(h ^ ((h >> 15) & 0x7fff)));
            low = (float)__builtin_bit_cast(T, (short)(l ^ ((l >> 15) & 0x7fff)));
        }
        __syncthreads();
        done = sh.kept == 0;
        if (!done) {
            top = -INFINITY;
            low = INFINITY;
        }
    }
    if (!done) {
        row.each([&](const float (&x)[W], int j, int) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (INDEX) at = x[i] > top ? j + i : at;
                top = fmaxf(top, x[i]);
                low = fminf(low, x[i]);
            }
        });
    }
    uint64_t best = top > -INFINITY ? (uint64_t)smp_key(top) << 32 | (uint32_t)~at : 0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const uint64_t y = __shfl_xor(best, o);
        best = y > best ? y : best;
        low = fminf(low, __shfl_xor(low, o));
    }
    if ((threadIdx.x & 63) == 0) {
        atomicMax((unsigned long long *)&sh.best, (unsigned long long)best);
        atomicMin(&sh.low, smp_key(low));
    }
    __syncthreads();
}

// One workgroup a row, two rows a compute unit: registers are held to 64 for that.  Bound by the instructions of the weights (vector unit 73 % busy in 512 rows of bf16), not by
// memory, which the second and later walks find in the L2.  us: a row of 20 000 words (fp32, top-p) 26, of which 9 for the draw's walk and 7 for
// the histogram; 256 rows of 50 000 (fp32, all filters) 46; 512 rows of 131 072 (bf16, top-p) 141, 0.95 TB/s.
template <typename T> __global__ __launch_bounds__(SMP_THREADS, 8) void k_sample(const SampleArgs a)
{
    SmpShared &sh = smp_shared();
    const int r = blockIdx.x;
    const SmpRow<T> row(static_cast<const T *>(a.logits) + (long long)r * a.row, a.vocab);

    const float temperature = a.temperature ? a.temperature[r] : 1.f;
    const bool greedy = !(temperature > 0.f);
    if (greedy) smp_extremes<T, true>(row);
    else smp_extremes<T, false>(row);
    const uint64_t best = sh.best;
    if (best == 0 || greedy) {
        if (threadIdx.x == 0) {
            a.token[r] = best ? (int32_t)~(uint32_t)best : -1;
            if (a.logprob) a.logprob[r] = best ? 0.f : -INFINITY;
            if (a.kept) a.kept[r] = best ? 1 : 0;
        }
        return;
    }
    SmpWeight weight;
    const float max = smp_value((uint32_t)(best >> 32));
    weight.per_t = max < INFINITY ? 1.4426950408889634 / (double)temperature : 1.;
    weight.max = max < INFINITY ? (double)max : 1e300;
    weight.shift = a.shift;
    weight.pad = 0;

    SmpCut cut = {smp_value(SMP_KEY_NONE + 1), row.n, 0};       // every word above -infinity
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f;
    const bool by_count = k > 0 && k < row.n;
    bool by_mass = p < 1.f;
    if (by_count || by_mass) {
        SmpSteps step;
        step.max = fminf(max, FLT_MAX);
        const float range = fminf(step.max - smp_value(sh.low), (float)(SMP_REACH * (double)temperature));
        step.per = range > 0.f && range < INFINITY ? fminf((float)SMP_BINS / range, FLT_MAX) : 0.f;
        if (by_count) {
            smp_histogram<T, true>(row, weight, step);
            const SmpAt s = smp_step<true>((uint32_t)k, 0.f, 0);
            const bool all = s.above + s.here <= SMP_LIST;      // the list holds every word that top-k may keep
            if (s.here <= SMP_LIST) {
                uint64_t mass_above = 0;
                if (by_mass && !all) {
                    smp_histogram<T, false>(row, weight, step);
                    uint64_t m = 0;
                    for (int i = threadIdx.x; i < s.at; i += SMP_THREADS) m += sh.mass[i];
                    smp_scan(m, &mass_above, sh);
                }
                const int n = smp_collect(row, step, all ? 0 : s.at, s.at);
                smp_sort(n);
                cut = smp_cut_list<true>(n, weight, (uint32_t)k, 0, mass_above, all ? 0 : (uint32_t)s.above);
                if (by_mass && all) {
                    const SmpCut c = smp_cut_list<false>(n, weight, 0, smp_share(p, cut.mass, true), 0, 0);
                    if (cut.keeps(c.x, c.j)) cut = c;
                    by_mass = false;
                }
            } else {
                cut = smp_cut_by_digits<T, true>(row, weight, (uint32_t)k, 0);
                if (by_mass) smp_histogram<T, false>(row, weight, step);
            }
        } else {
            smp_histogram<T, false>(row, weight, step);
        }
        if (by_mass) {
            const SmpAt s = smp_step<false>(0, p, cut.mass);
            const int n = smp_collect(row, step, s.at, s.at);
            SmpCut c;
            if (n <= SMP_LIST) {
                smp_sort(n);
                c = smp_cut_list<false>(n, weight, 0, s.need, s.above, 0);
            } else {
                c = smp_cut_by_digits<T, false>(row, weight, 0, s.need);
            }
            if (cut.keeps(c.x, c.j)) cut = c;
        }
    }
    // w >= min_p, of the exponents, as a bound of the values.  A min_p not above 0, or a NaN, keeps every word; its logarithm is not asked for (a
    // NaN, which fmin would take for the bound of the largest value).
    const float m = a.min_p ? a.min_p[r] : 0.f;
    if (m > 0.f) {
        const float x = smp_least_value(weight, max, fmin(log2((double)m), 0.));
        if (x > cut.x) {
            cut.x = x;
            cut.j = row.n;
        }
    }
    SmpKept f = {};
    f.cut = cut;
    f.weight = weight;
    f.u = a.u[r];
    const SmpDraw d = smp_locate(row, f);
    if (threadIdx.x == 0) {
        a.token[r] = d.word;
        if (a.logprob) a.logprob[r] = (float)log((double)d.weight / (double)d.sum);
        if (a.kept) a.kept[r] = d.kept;
    }
}

}  // namespace tl
