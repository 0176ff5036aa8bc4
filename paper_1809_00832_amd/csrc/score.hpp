// Log probabilities of given words, entropies and the most probable words of rows of logits; the gradient of the first two.
//
//   m = max x,  z = sum_j exp(x_j - m),  log p_j = x_j - m - log z,  H = log z - sum_j exp(x_j - m) (x_j - m) / z
//   d_j = dl ([j = w] - p_j) - dH p_j (log p_j + H)
//
// One pass over a row: every lane keeps the largest value so far and the sums of e and e d for weights e = 2^d relative to a reference, which is raised
// when values come far above it.  The most probable words are kept in the same pass: words as 64-bit numbers (the value's bits in the order
// of values, then the complement of the word's index, so that no two are equal and equal values go by index), a sorted list of 64 per wave, a lane each, and
// a border below which a word cannot be among the first.  What lies above the border is put into LDS; when 64 are there they are sorted and
// joined to the list, so that a row in ascending order costs a sort per 64 words and not a step per word.
#pragma once

#include "attend.hpp"
#include "sample.hpp"
#include "stream.hpp"

namespace tl {

constexpr float SCO_LOG2_E = 1.4426950408889634f, SCO_LN_2 = 0.6931471805599453f;
constexpr float SCO_FAR = -150.f;               // 2^-150 is zero in fp32, and a finite number times zero is zero
constexpr uint64_t SCO_NONE = 0;                // no word: below every word's number
constexpr int SCO_TOP = 64;

struct ScoreArgs {
    const void *logits;
    long long row;
    const int32_t *word;
    float *logprob, *stats, *top_logprob;
    int32_t *top_word;
    float *part;                                // parts > 1: m, z, sum of e d and nothing for every row and part, then lists of 64 words
    int n_rows, vocab, top, parts;
    const float *d_logprob, *d_entropy;
    void *d_logits;
    long long d_row;
    long long first;                            // row of the launch's first workgroup
};

// ---- 64 words, a lane each, largest first --------------------------------------------------------

// The value of lane `lane ^ D`, without LDS.
template <int D> __device__ inline uint32_t sco_swap(uint32_t x)
{
    if constexpr (D == 1) return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);             // quad_perm 1 0 3 2
    else if constexpr (D == 2) return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);        // quad_perm 2 3 0 1
    else if constexpr (D == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);   // row_half_mirror (xor 7), quad_perm 3 2 1 0 (xor 3)
    else if constexpr (D == 8) return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);       // row_ror 8
    else if constexpr (D == 15) return __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true);      // row_mirror
    else {
        static_assert(D == 16 || D == 32, "a power of two of lanes");
        // [0]: the upper half of every 2 D lanes holds the lower one's values, [1]: the other way round
        const auto p = D == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & D ? p[0] : p[1];
    }
}
template <int D> __device__ inline uint64_t sco_swap(uint64_t x) { return (uint64_t)sco_swap<D>((uint32_t)(x >> 32)) << 32 | sco_swap<D>((uint32_t)x); }
template <int D> __device__ inline float sco_swap(float x) { return __uint_as_float(sco_swap<D>(__float_as_uint(x))); }

template <int D, typename X> __device__ inline X sco_step(X x, bool largest)
{
    const X y = sco_swap<D>(x);
    return (x > y) == largest ? x : y;
}
// Runs of 2 D lanes, each first rising and then falling or the other way round, to runs that fall (or, where `down` is false, rise).
template <int D, typename X> __device__ inline X sco_runs(X x, bool down)
{
    x = sco_step<D>(x, ((threadIdx.x & D) == 0) == down);
    if constexpr (D > 1) x = sco_runs<D / 2>(x, down);
    return x;
}
template <typename X> __device__ inline X sco_sort(X x)
{
    const int lane = threadIdx.x & 63;
    x = sco_runs<1>(x, (lane & 2) == 0);
    x = sco_runs<2>(x, (lane & 4) == 0);
    x = sco_runs<4>(x, (lane & 8) == 0);
    x = sco_runs<8>(x, (lane & 16) == 0);
    x = sco_runs<16>(x, (lane & 32) == 0);
    return sco_runs<32>(x, true);
}

// The largest 64 of two sorted lists.
__device__ inline uint64_t sco_merge(uint64_t x, uint64_t y)
{
    const uint64_t r = sco_swap<32>(sco_swap<16>(sco_swap<15>(y)));                 // lane 63 - l
    return sco_runs<32>(x > r ? x : r, true);
}

__device__ inline uint64_t sco_number(float x, int index)
{
    return (uint64_t)smp_key(fmaxf(x, -INFINITY)) << 32 | (uint32_t)~index;         // (a NaN as -infinity)
}
constexpr uint64_t SCO_LEAST = (uint64_t)SMP_KEY_NONE << 32 | 0xffffffffu;      // words at -infinity, and all of them

// A list with the first 64 of the words that wait, which are taken out.  (Called, not inlined: it is rare, and a piece has many places that need it.)
__device__ __noinline__ uint64_t sco_join(uint64_t list, uint64_t *wait, int waiting)
{
    const int lane = threadIdx.x & 63;
    const uint64_t x = lane < waiting ? wait[lane] : SCO_NONE, rest = lane + 64 < waiting ? wait[lane + 64] : SCO_NONE;
    wait[lane] = rest;
    return sco_merge(list, sco_sort(x));
}

// A wave's list and the words that wait to join it.
struct ScoList {
    uint64_t list, border;                      // border: only words above it can be among the first `top`
    float least;                                // ... and their values are not below this
    int waiting, top;
    uint64_t *wait;                             // [128] in LDS

    __device__ void init(uint64_t *lds, int n)
    {
        list = SCO_NONE;
        border = SCO_LEAST;
        least = -FLT_MAX;
        waiting = 0;
        top = n;
        wait = lds;
    }
    __device__ void raise(uint64_t to)
    {
        if (to <= border) return;
        border = to;
        least = smp_value((uint32_t)(to >> 32));
    }
    // Largest values of 64 groups of words, a lane each: the first `top` of them are `top` words, and none of these is below the last one.
    __device__ void prime(float largest)
    {
        const uint32_t at = __shfl(sco_sort(smp_key(fmaxf(largest, -INFINITY))), top - 1, 64);
        raise(((uint64_t)at << 32) - 1);        // (any word of that very value may still be one of them)
    }
    __device__ void join()
    {
        list = sco_join(list, wait, waiting);
        waiting = max(waiting - 64, 0);
        const uint64_t last = __shfl((unsigned long long)list, top - 1, 64);
        if (last != SCO_NONE) raise(last - 1);
    }
    __device__ void push(float x, int index)
    {
        const uint64_t k = sco_number(x, index);
        const unsigned long long mask = __ballot(k > border);
        if (!mask) return;
        if (k > border) wait[waiting + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1))] = k;
        waiting += __popcll(mask);
        if (waiting >= 64) join();
    }
};

// ---- sums --------------------------------------------------------------------------------------
//
// A lane's weights are 2^d with d = x log2(e) - r, one multiply-add: r is the rounded product of some logit and log2(e), raised when a logit lies more than
// SCO_LAG above it.  What rounding r did is the same for all words and is taken out again at the end, when the sums are brought to the row's
// largest logit itself.  It is below 2^-7 for logits up to SCO_LARGE; rows whose largest logit lies outside are walked once more, with differences.  Words
// far below -SCO_LARGE weigh nothing in the others: no reference is lower.

constexpr float SCO_LAG = 16.f, SCO_LARGE = 1e5f;

struct ScoSums {
    float r, z, t;                              // reference, sum of e, sum of e d
    __device__ void scale(float to)
    {
        const float d = fmaxf(r - to, SCO_FAR), c = __builtin_amdgcn_exp2f(d);
        t = c * fmaf(d, z, t);
        z *= c;
        r = to;
    }
    __device__ void add(float x)
    {
        const float d = fmaxf(fmaf(x, SCO_LOG2_E, -r), SCO_FAR), e = __builtin_amdgcn_exp2f(d);
        z += e;
        t = fmaf(e, d, t);
    }
    // by the difference from the row's largest logit, whatever that is
    __device__ void add_far(float x, float m)
    {
        const float d = x == m ? 0.f : fmaxf((x - m) * SCO_LOG2_E, SCO_FAR), e = __builtin_amdgcn_exp2f(d);
        z += e;
        t = fmaf(e, d, t);
    }
};

template <int D = 32> __device__ inline float sco_sum(float x)
{
    x += sco_swap<D>(x);
    if constexpr (D > 1) x = sco_sum<D / 2>(x);
    return x;
}
template <int D = 32> __device__ inline float sco_max(float x)
{
    x = fmaxf(x, sco_swap<D>(x));
    if constexpr (D > 1) x = sco_max<D / 2>(x);
    return x;
}

// The largest of three numbers, NaN if one of them is, whichever kind of NaN.  (The other maximum leaves a quiet NaN out, but of a signalling one and a number makes a NaN, which hides the
// number from the next step; and fmaxf of a number that was just read would first be made quiet, an instruction each.)
__device__ inline float sco_max3(float a, float b, float c)
{
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// What a row is known by: its largest logit, and relative to it the sum of e and of e d.
struct ScoRow {
    float m, z, t;
};

template <typename T> __device__ inline float sco_logit(const ScoreArgs &a, long long row, int j) { return (float)static_cast<const T *>(a.logits)[row * a.row + j]; }

// What is said of a row, from its sums and its list; one wave.
template <typename T> __device__ inline void sco_answer(const ScoreArgs &a, long long row, const ScoRow &s, uint64_t list)
{
    const int lane = threadIdx.x & 63;
    const bool some = s.m > -INFINITY;
    const float log_z = some ? logf(s.z) : -INFINITY;
    auto log_p = [&](float x) { return !some || !(x > -INFINITY) ? -INFINITY : x == s.m ? -log_z : x - s.m - log_z; };
    if (lane == 0) {
        if (a.logprob) {
            const int w = a.word[row];
            a.logprob[row] = w >= 0 && w < a.vocab ? log_p(sco_logit<T>(a, row, w)) : 0.f;
        }
        if (a.stats) {
            a.stats[row] = s.m;
            a.stats[a.n_rows + row] = some ? s.z : 0.f;
            a.stats[2ll * a.n_rows + row] = some ? fmaxf(log_z - SCO_LN_2 * (s.t / s.z), 0.f) : 0.f;
        }
    }
    if (lane < a.top) {
        const bool there = list > SCO_LEAST;
        a.top_word[row * a.top + lane] = there ? (int)~(uint32_t)list : -1;
        a.top_logprob[row * a.top + lane] = there ? log_p(smp_value((uint32_t)(list >> 32))) : -INFINITY;
    }
}

// ---- one row, or one part of it, per workgroup ------------------------------------------------------

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) ScoAny {
    T v[16 / sizeof(T)];
};

template <typename T, int NT, bool TOP, bool ONCE> __global__ __launch_bounds__(NT) void k_score(ScoreArgs a)
{
    constexpr int E = 16 / (int)sizeof(T), U = 16 / E, WAVES = NT / 64;
    __shared__ uint64_t wait[TOP ? WAVES : 1][128], all_words[TOP ? WAVES * 128 : 1];
    __shared__ float maxima[TOP ? 3 : 1][WAVES][64];
    __shared__ ScoSums sums[WAVES];
    __shared__ float largest[WAVES];
    __shared__ int taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long row = a.first + blockIdx.x / a.parts;
    const int part = blockIdx.x - (int)(blockIdx.x / a.parts) * a.parts;
    // parts are of whole pieces
    const int size = (((a.vocab + a.parts - 1) / a.parts) + E - 1) / E * E;
    const int begin = (int)min((long long)part * size, (long long)a.vocab), n = min(size, a.vocab - begin);
    const T *const p = static_cast<const T *>(a.logits) + row * a.row + begin;
    const int pieces = n / E, edge = n - pieces * E;            // (16 bytes at any address: what a row gives does not depend on where it lies)
    ScoSums s = {-SCO_LARGE * SCO_LOG2_E, 0.f, 0.f};
    float m = -INFINITY;
    ScoList top;
    if (TOP) top.init(wait[TOP ? wave : 0], a.top);
    auto take = [&](float (&v)[U][E], const int (&at)[U]) {         // at: index of each piece's first word
        float most[U], all;
        auto largest_of = [&]() {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                most[u] = v[u][0];
#pragma unroll
                for (int e = 1; e < E; e += 2) most[u] = sco_max3(most[u], v[u][e], v[u][e + 1 < E ? e + 1 : e]);
                all = u ? sco_max3(all, most[u], most[u]) : most[u];
            }
        };
        largest_of();
        if (__any(!(fmaf(all, SCO_LOG2_E, -s.r) <= SCO_LAG))) {
            if (__any(all != all)) {                            // (NaN as -infinity)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[u][e] = v[u][e] == v[u][e] ? v[u][e] : -INFINITY;
                largest_of();
            }
            if (__any(fmaf(all, SCO_LOG2_E, -s.r) > SCO_LAG)) s.scale(fmaxf(s.r, all * SCO_LOG2_E));
        }
        m = fmaxf(m, all);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) s.add(v[u][e]);
        if constexpr (TOP) {
            if (top.border == SCO_LEAST) top.prime(all);            // (nothing better is known yet)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (__any(most[u] >= top.least))
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (__any(v[u][e] >= top.least)) top.push(v[u][e], at[u] + e);
        }
    };
    // The border from the largest values of all waves' lanes so far, 64 groups of the words that the workgroup has read: some 1.2 times `top` words lie above it for
    // `top` = 20 (64 ln(64 / (64 - top)) of them), where a wave's own words alone would let eight times as many through.
    auto prime_all = [&](int n) {
        maxima[n][wave][lane] = m;
        __syncthreads();
        float x = maxima[n][0][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x = fmaxf(x, maxima[n][w][lane]);
        top.prime(x);
    };
    float v[U][E];
    int at[U];
    if (wave == 0 && edge > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) v[u][e] = -INFINITY;
        at[0] = pieces * E + tid;
#pragma unroll
        for (int u = 1; u < U; ++u) at[u] = 0;
        if (tid < edge) v[0][0] = (float)p[at[0]];
        at[0] += begin;
        take(v, at);
    }
    ScoAny<T> next[U];
    auto load = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < pieces) stream_load<ONCE>(next[u], p + (i + u * NT) * E);
    };
    load(tid);
    for (int g = wave * 64; g < pieces; g += U * NT) {          // (the same in all lanes of a wave)
        const int i = g + lane;
        if (g + (U - 1) * NT + 64 > pieces)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e) next[u].v[e] = i + u * NT < pieces ? next[u].v[e] : (T)-INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[u][e] = (float)next[u].v[e];
            at[u] = begin + (i + u * NT) * E;
        }
        load(i + U * NT);
        // (once a first round of pieces is there, and once a fourth is: rounds that all lanes take part in)
        if constexpr (TOP) {
            const int round = (g - wave * 64) / (U * NT);
            if ((round == 0 || round == 3) && (round + 1) * U * NT <= pieces) {
                if (round == 0) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < E; ++e) m = fmaxf(m, v[u][e]);
                }
                prime_all(round == 0 ? 0 : 1);
            }
        }
        take(v, at);
    }
    if (TOP) prime_all(2);
    m = sco_max(m);
    s.scale(sco_max(s.r));
    s.z = sco_sum(s.z);
    s.t = sco_sum(s.t);
    if (lane == 0) {
        sums[wave] = s;
        largest[wave] = m;
    }
    if (tid == 0) taken = 0;
    __syncthreads();
    // waves' sums, a lane each
    m = sco_max(largest[lane < WAVES ? lane : 0]);
    ScoSums x = sums[lane < WAVES ? lane : 0];
    ScoRow of = {m, 0.f, 0.f};
    if (fabsf(m) <= SCO_LARGE) {
        if (wave == 0) {                                        // (which alone answers)
            const float r = sco_max(x.r);
            x.scale(r);
            const float z = sco_sum(lane < WAVES ? x.z : 0.f), t = sco_sum(lane < WAVES ? x.t : 0.f);
            // ... and relative to m itself
            const float lag = fmaf(m, SCO_LOG2_E, -r), c = __builtin_amdgcn_exp2f(-lag);
            of.t = c * fmaf(-lag, z, t);
            of.z = fmaxf(c * z, 1.f);                           // (m's own weight is one; c is rounded, and no log probability may come out above zero)
        }
    } else if (m > -INFINITY) {                                 // (words at infinity share the mass)
        x = {0.f, 0.f, 0.f};
        for (int j = tid; j < n; j += NT) x.add_far((float)p[j], m);
        x.z = sco_sum(x.z);
        x.t = sco_sum(x.t);
        __syncthreads();
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        of.z = sco_sum(lane < WAVES ? sums[lane].z : 0.f);
        of.t = sco_sum(lane < WAVES ? sums[lane].t : 0.f);
    }
    uint64_t list = SCO_NONE;
    if (TOP) {
        // the words above the last border, which wave 0 sorts
        const uint64_t first = lane < top.waiting ? top.wait[lane] : SCO_NONE;          // (fewer than 64 wait)
        if (first > top.border) all_words[atomicAdd(&taken, 1)] = first;
        if (lane < a.top && top.list > top.border) all_words[atomicAdd(&taken, 1)] = top.list;
        __syncthreads();
        if (wave == 0 && taken > 0) {
            list = sco_sort(lane < taken ? all_words[lane] : SCO_NONE);
            for (int k = 64; k < taken; k += 64) list = sco_merge(list, sco_sort(k + lane < taken ? all_words[k + lane] : SCO_NONE));
        }
    }
    if (wave != 0) return;
    if (a.parts == 1) {
        sco_answer<T>(a, row, of, list);
    } else {
        const long long k = row * a.parts + part;
        if (lane == 0) *reinterpret_cast<f32x4 *>(a.part + 4 * k) = f32x4{of.m, of.z, of.t, 0.f};
        if (TOP) reinterpret_cast<uint64_t *>(a.part + 4ll * a.n_rows * a.parts)[k * SCO_TOP + lane] = list;
    }
}

// The parts of a row; a wave per row.
template <typename T, bool TOP> __global__ __launch_bounds__(256) void k_score_join(ScoreArgs a)
{
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= a.n_rows) return;
    ScoRow s = {-INFINITY, 0.f, 0.f};
    if (lane < a.parts) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + 4 * (row * a.parts + lane));
        s = {x[0], x[1], x[2]};
    }
    const float m = sco_max(s.m);
    const float d = s.m == m ? 0.f : fmaxf((s.m - m) * SCO_LOG2_E, SCO_FAR), c = __builtin_amdgcn_exp2f(d);
    s.t = sco_sum(c * fmaf(d, s.z, s.t));
    s.z = sco_sum(c * s.z);
    s.m = m;
    uint64_t list = SCO_NONE;
    if (TOP) {
        const uint64_t *at = reinterpret_cast<const uint64_t *>(a.part + 4ll * a.n_rows * a.parts) + row * a.parts * SCO_TOP + lane;
        for (int k = 0; k < a.parts; ++k) list = sco_merge(list, at[k * SCO_TOP]);
    }
    sco_answer<T>(a, row, s, list);
}

// ---- gradient ---------------------------------------------------------------------------------------

constexpr int SCO_BACK_THREADS = 256, SCO_BACK_PIECES = 2;

template <typename T, bool ONCE> __global__ __launch_bounds__(SCO_BACK_THREADS) void k_score_back(ScoreArgs a)
{
    constexpr int E = 16 / (int)sizeof(T), U = SCO_BACK_PIECES, NT = SCO_BACK_THREADS;
    typedef ScoAny<T> Any;
    const int tid = threadIdx.x;
    const long long row = a.first + blockIdx.x / a.parts;
    const int part = blockIdx.x - (int)(blockIdx.x / a.parts) * a.parts;
    const int begin = part * (NT * U * E), n = min(NT * U * E, a.vocab - begin);
    const T *const x = static_cast<const T *>(a.logits) + row * a.row + begin;
    T *const out = static_cast<T *>(a.d_logits) + row * a.d_row + begin;
    const int word = a.word ? a.word[row] : -1;
    const float m = a.stats[row], z = a.stats[a.n_rows + row], h = a.stats[2ll * a.n_rows + row];
    const bool some = m > -INFINITY, there = word >= 0 && word < a.vocab && some;
    const float dl = there && a.d_logprob ? a.d_logprob[row] : 0.f, dh = a.d_entropy && some ? a.d_entropy[row] : 0.f;
    const int pieces = n / E;
    if (dl == 0.f && dh == 0.f) {                               // (a row without a word costs no reads)
        for (int i = tid; i < pieces; i += NT) stream_store<ONCE>(out + i * E, Any{});
        if (pieces * E + tid < n) out[pieces * E + tid] = (T)0.f;
        return;
    }
    // d_j = [j = w] dl - p_j (dl + dh (log p_j + H)) with p_j = 2^d / z, d = x log2(e) - r less what rounding r = m log2(e) left
    const bool far = !(fabsf(m) <= SCO_LARGE);
    const float r = m * SCO_LOG2_E, lag = far ? 0.f : fmaf(m, SCO_LOG2_E, -r), per_z = __builtin_amdgcn_exp2f(-lag) / z;
    const float step = -dh * SCO_LN_2 * per_z, base = -fmaf(dh, h - logf(z) - lag * SCO_LN_2, dl) * per_z;
    auto gradient = [&](float v) {
        const float d = fmaxf(fmaf(v, SCO_LOG2_E, -r), SCO_FAR);
        return __builtin_amdgcn_exp2f(d) * fmaf(step, d, base);
    };
    auto gradient_far = [&](float v) {
        const float d = v == m ? 0.f : fmaxf((v - m) * SCO_LOG2_E, SCO_FAR);
        return __builtin_amdgcn_exp2f(d) * fmaf(step, d, base);
    };
    const int w = word - begin;                                 // (the word's own part is added to its one value)
    if (far) {
        for (int j = tid; j < n; j += NT) out[j] = (T)(gradient_far((float)x[j]) + (there && j == w ? dl : 0.f));
        return;
    }
    Any v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (tid + u * NT < pieces) stream_load<ONCE>(v[u], x + (tid + u * NT) * E);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * NT;
        if (i < pieces) {
            Any o;
#pragma unroll
            for (int e = 0; e < E; ++e) o.v[e] = (T)gradient((float)v[u].v[e]);
            if (there && (unsigned)(w - i * E) < (unsigned)E)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (w == i * E + e) o.v[e] = (T)(gradient((float)v[u].v[e]) + dl);
            stream_store<ONCE>(out + i * E, o);
        }
    }
    const int j = pieces * E + tid;
    if (j < n) out[j] = (T)(gradient((float)x[j]) + (there && j == w ? dl : 0.f));
}

}  // namespace tl
