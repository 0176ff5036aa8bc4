// Log probabilities of given words, entropies and the most probable words of rows of logits; the gradient of the first two.
//
//   m = max x,  z = sum_j exp(x_j - m),  log p_j = x_j - m - log z,  H = log z - sum_j exp(x_j - m) (x_j - m) / z
//   d_j = dl ([j = w] - p_j) - dH p_j (log p_j + H)
//
// One pass over a row: every lane keeps the largest value so far and the sums of e and e d for e = 2^d, d = (x - m) log2(e), and scales them
// when a larger value comes.  The most probable words are kept in the same pass: words as 64-bit numbers (the value's bits in the order
// of values, then the complement of the word's index, so that no two are equal and equal values go by index), a sorted list of 64 per wave, a lane each, and
// a border below which a word cannot be among the first.  What lies above the border is put into LDS; when 64 are there they are sorted and
// joined to the list, so that a row in ascending order costs a sort per 64 words and not a step per word.
#pragma once

#include "attend.hpp"
#include "sample.hpp"

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

__device__ inline uint64_t sco_swap(uint64_t x, int with) { return __shfl_xor((unsigned long long)x, with, 64); }

__device__ inline uint64_t sco_step(uint64_t x, int distance, bool largest)
{
    const uint64_t y = sco_swap(x, distance);
    return (x > y) == largest ? x : y;
}

__device__ inline uint64_t sco_sort(uint64_t x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 2; n <= 64; n *= 2)
#pragma unroll
        for (int d = n / 2; d > 0; d /= 2) x = sco_step(x, d, ((lane & d) == 0) == ((lane & n) == 0 || n == 64));
    return x;
}

// The largest 64 of two sorted lists.
__device__ inline uint64_t sco_merge(uint64_t x, uint64_t y)
{
    const int lane = threadIdx.x & 63;
    const uint64_t r = __shfl((unsigned long long)y, 63 - lane, 64);
    x = x > r ? x : r;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x = sco_step(x, d, (lane & d) == 0);
    return x;
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
    // Every lane's largest value so far: the first `top` lanes, in order of these, hold `top` words that are not below the last one's.
    __device__ void prime(float largest)
    {
        const uint64_t x = sco_sort((uint64_t)smp_key(fmaxf(largest, -INFINITY)) << 32);
        const uint64_t at = __shfl((unsigned long long)x, top - 1, 64);
        raise(at - 1);                          // (any word of that very value may still be one of them)
    }
    __device__ void join()
    {
        list = sco_join(list, wait, waiting);
        waiting = max(waiting - 64, 0);
        raise(__shfl((unsigned long long)list, top - 1, 64));
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

struct ScoSums {
    float m, z, t;                              // largest value, sum of e, sum of e d
    __device__ void scale(float to)
    {
        const float d = fmaxf((m - to) * SCO_LOG2_E, SCO_FAR), c = __builtin_amdgcn_exp2f(d);
        t = c * fmaf(d, z, t);
        z *= c;
        m = to;
    }
    __device__ void add(const ScoSums &o, float to)
    {
        ScoSums p = o;
        scale(to);
        p.scale(to);
        z += p.z;
        t += p.t;
    }
};

// Lanes' sums, in every lane.
__device__ inline ScoSums sco_wave(ScoSums s)
{
    float m = s.m;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d, 64));
    s.scale(m);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        s.z += __shfl_xor(s.z, d, 64);
        s.t += __shfl_xor(s.t, d, 64);
    }
    return s;
}

template <typename T> __device__ inline float sco_logit(const ScoreArgs &a, long long row, int j) { return (float)static_cast<const T *>(a.logits)[row * a.row + j]; }

// What is said of a row, from its sums and its list; one wave.
template <typename T> __device__ inline void sco_answer(const ScoreArgs &a, long long row, const ScoSums &s, uint64_t list)
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

template <typename T> struct __attribute__((packed, aligned(16))) ScoPiece {
    T v[16 / sizeof(T)];
};

template <typename T, int NT, bool TOP> __global__ __launch_bounds__(NT) void k_score(ScoreArgs a)
{
    constexpr int E = 16 / (int)sizeof(T), U = 16 / E, WAVES = NT / 64;
    __shared__ uint64_t wait[TOP ? WAVES : 1][128];
    __shared__ ScoSums sums[WAVES];
    __shared__ uint64_t borders[WAVES];
    __shared__ int taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long row = a.first + blockIdx.x / a.parts;
    const int part = blockIdx.x - (int)(blockIdx.x / a.parts) * a.parts;
    // parts are of whole pieces
    const int size = (((a.vocab + a.parts - 1) / a.parts) + E - 1) / E * E;
    const int begin = (int)min((long long)part * size, (long long)a.vocab), n = min(size, a.vocab - begin);
    const T *const p = static_cast<const T *>(a.logits) + row * a.row + begin;
    const int head = min(n, (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T));
    const int pieces = (n - head) / E, edge = n - pieces * E;       // words in front of the first whole piece and behind the last one
    const ScoPiece<T> *const q = reinterpret_cast<const ScoPiece<T> *>(p + head);
    ScoSums s = {-INFINITY, 0.f, 0.f};
    ScoList top;
    if (TOP) top.init(wait[TOP ? wave : 0], a.top);
    auto take = [&](const float (&v)[U][E], const int (&at)[U]) {   // at: index of each piece's first word
        float most[U], all;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            most[u] = v[u][0];
#pragma unroll
            for (int e = 1; e < E; ++e) most[u] = fmaxf(most[u], v[u][e]);
        }
        all = most[0];
#pragma unroll
        for (int u = 1; u < U; ++u) all = fmaxf(all, most[u]);
        s.scale(fmaxf(s.m, all));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = fmaxf((v[u][e] - s.m) * SCO_LOG2_E, SCO_FAR), x = __builtin_amdgcn_exp2f(d);
                s.z += x;
                s.t = fmaf(x, d, s.t);
            }
        if constexpr (TOP) {
            if (top.border == SCO_LEAST) top.prime(all);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (__any(most[u] >= top.least))
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (__any(v[u][e] >= top.least)) top.push(v[u][e], at[u] + e);
        }
    };
    float v[U][E];
    int at[U];
    if (wave == 0 && edge > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) v[u][e] = -INFINITY;
        at[0] = tid < head ? tid : tid + pieces * E;
#pragma unroll
        for (int u = 1; u < U; ++u) at[u] = 0;
        if (tid < edge) v[0][0] = (float)p[at[0]];
        at[0] += begin;
        take(v, at);
    }
    ScoPiece<T> next[U];
    auto load = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < pieces) next[u] = q[i + u * NT];
    };
    load(tid);
    for (int g = wave * 64; g < pieces; g += U * NT) {          // (the same in all lanes of a wave)
        const int i = g + lane;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[u][e] = i + u * NT < pieces ? (float)next[u].v[e] : -INFINITY;
            at[u] = begin + head + (i + u * NT) * E;
        }
        load(i + U * NT);
        take(v, at);
    }
    s = sco_wave(s);
    if (lane == 0) sums[wave] = s;
    if (TOP) {
        while (top.waiting > 0) top.join();
        if (lane == a.top - 1) borders[wave] = top.list;
    }
    if (tid == 0) taken = 0;
    __syncthreads();
    float m = sums[0].m;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sums[w].m);
    ScoSums r = {m, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) r.add(sums[w], m);
    if (m == INFINITY) {                                        // the words at infinity share the mass: they are counted
        float c = 0.f;
        for (int j = tid; j < n; j += NT) c += (float)p[j] == INFINITY ? 1.f : 0.f;
#pragma unroll
        for (int d = 32; d > 0; d /= 2) c += __shfl_xor(c, d, 64);
        __syncthreads();
        if (lane == 0) sums[wave].z = c;
        __syncthreads();
        r.z = r.t = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) r.z += sums[w].z;
    }
    uint64_t list = SCO_NONE;
    if (TOP) {
        // words that are not below any wave's last one, and wave 0 sorts them
        uint64_t border = SCO_LEAST;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) border = borders[w] > border ? borders[w] : border;
        uint64_t *const all = &wait[0][0];
        if (lane < a.top && top.list >= border && top.list > SCO_LEAST) all[atomicAdd(&taken, 1)] = top.list;
        __syncthreads();
        if (wave == 0)
            for (int k = 0; k < taken; k += 64) list = sco_merge(list, sco_sort(k + lane < taken ? all[k + lane] : SCO_NONE));
    }
    if (wave != 0) return;
    if (a.parts == 1) {
        sco_answer<T>(a, row, r, list);
    } else {
        const long long k = row * a.parts + part;
        if (lane == 0) *reinterpret_cast<f32x4 *>(a.part + 4 * k) = f32x4{r.m, r.z, r.t, 0.f};
        if (TOP) reinterpret_cast<uint64_t *>(a.part + 4ll * a.n_rows * a.parts)[k * SCO_TOP + lane] = list;
    }
}

// The parts of a row; a wave per row.
template <typename T, bool TOP> __global__ __launch_bounds__(256) void k_score_join(ScoreArgs a)
{
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= a.n_rows) return;
    ScoSums s = {-INFINITY, 0.f, 0.f};
    if (lane < a.parts) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + 4 * (row * a.parts + lane));
        s = {x[0], x[1], x[2]};
    }
    float m = s.m;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d, 64));
    if (m == INFINITY) {                                        // (an infinity less itself is no number)
        if (s.m < m) s.z = 0.f;
        s.t = 0.f;
        s.m = m;
    } else {
        s.scale(m);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        s.z += __shfl_xor(s.z, d, 64);
        s.t += __shfl_xor(s.t, d, 64);
    }
    uint64_t list = SCO_NONE;
    if (TOP) {
        const uint64_t *at = reinterpret_cast<const uint64_t *>(a.part + 4ll * a.n_rows * a.parts) + row * a.parts * SCO_TOP + lane;
        for (int k = 0; k < a.parts; ++k) list = sco_merge(list, at[k * SCO_TOP]);
    }
    sco_answer<T>(a, row, s, list);
}

// ---- gradient ---------------------------------------------------------------------------------------

constexpr int SCO_BACK_THREADS = 256, SCO_BACK_PIECES = 4;

template <typename T> __global__ __launch_bounds__(SCO_BACK_THREADS) void k_score_back(ScoreArgs a)
{
    constexpr int E = 16 / (int)sizeof(T), U = SCO_BACK_PIECES, NT = SCO_BACK_THREADS;
    struct __attribute__((packed, aligned(sizeof(T)))) Any {
        T v[E];
    };
    const int tid = threadIdx.x;
    const long long row = a.first + blockIdx.x / a.parts;
    const int part = blockIdx.x - (int)(blockIdx.x / a.parts) * a.parts;
    const int begin = part * (NT * U * E), n = min(NT * U * E, a.vocab - begin);
    const T *const x = static_cast<const T *>(a.logits) + row * a.row + begin;
    T *const out = static_cast<T *>(a.d_logits) + row * a.d_row + begin;
    const int word = a.word ? a.word[row] : -1;
    const bool some = a.stats[row] > -INFINITY;
    const bool there = word >= 0 && word < a.vocab && some;
    const float dl = there && a.d_logprob ? a.d_logprob[row] : 0.f, dh = a.d_entropy && some ? a.d_entropy[row] : 0.f;
    const float m = a.stats[row], z = a.stats[a.n_rows + row], h = a.stats[2ll * a.n_rows + row];
    // d_j = [j = w] dl - p_j (dl + dh (log p_j + H)) with p_j = 2^d / z
    const float per_z = 1.f / z, step = dh * SCO_LN_2 * per_z, base = fmaf(dh, h - logf(z), dl) * per_z;
    const bool zero = dl == 0.f && dh == 0.f;                   // a row without a word costs no reads
    auto gradient = [&](float v, int j) {
        const float d = v == m ? 0.f : fmaxf((v - m) * SCO_LOG2_E, SCO_FAR);
        const float g = -__builtin_amdgcn_exp2f(d) * fmaf(step, d, base);
        return j == word - begin ? g + dl : g;
    };
    const int pieces = n / E;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = tid + u * NT;
        if (i < pieces) {
            Any r = {};
            if (!zero) {
                r = *reinterpret_cast<const Any *>(x + i * E);
#pragma unroll
                for (int e = 0; e < E; ++e) r.v[e] = (T)gradient((float)r.v[e], i * E + e);
            }
            *reinterpret_cast<Any *>(out + i * E) = r;
        }
    }
    const int j = pieces * E + tid;
    if (j < n) out[j] = zero ? (T)0.f : (T)gradient((float)x[j], j);
}

}  // namespace tl
