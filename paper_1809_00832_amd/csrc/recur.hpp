// A gated linear recurrence along the words of ragged sentences, and its gradients.
//
//   h_t = f_t h_(t-1) + i_t x_t            per channel; f = sigmoid(g), i = sigmoid(-g), or f = g, i = 1
//   mu_t = f_t (dh_t + mu_(t+1))           what goes back to word t - 1; lambda_t = dh_t + mu_(t+1)
//   dx_t = i_t lambda_t,   dg_t = lambda_t (h_(t-1) - x_t) f_t i_t   (f = g: lambda_t h_(t-1)),   dh0 = mu of the first word
//
// Both are linear maps of a state, so that a run of words is one pair (A, B), state -> A state + B, and pairs of runs side by side join
// to one.  A lane owns V channels; a wave takes R words, a workgroup W R words at a time: a wave forms the pair of its words from registers, the
// pairs are exchanged through LDS, and each wave then steps through its words once more, from the state that is its own.  A workgroup walks a
// whole sentence so.  Sentences that are few and long are cut into parts of W R words, a workgroup each, which holds its words in registers: it publishes
// its pair, takes the pairs of the parts before it, and goes on from the state that they give, so that every tensor is read once.
//
// The backward pass needs h_(t-1) in fp32 for every word.  It reads no h: the forward keeps the state of every 64th word (the tape, 1/64 of the
// states in fp32), and a block of 64 words is stepped through again from there.  So five tensors move instead of six, and a 16-bit h's
// rounding is in no gradient.
//
// A pair can overflow, vanish or multiply an infinity by a zero where the words one after the other do not, and words can overflow where the pair does
// not.  So a pair is made such that it says what may be taken from it (below), and where that is too little the words in question are walked one by one
// for that channel: infinities and NaN come out as the loop has them.
#pragma once

#include "attend.hpp"
#include "recur_rows.hpp"

namespace tl {

constexpr int REC_TAPE = 64;                    // words between two states of the tape
constexpr int REC_WHOLE = 31;                   // shift of a part's words that leaves every sentence whole

struct RecurArgs {
    const void *g, *x, *d_h;
    void *h, *d_g, *d_x;
    long long g_row, x_row, h_row, d_h_row, d_g_row, d_x_row;
    const int32_t *off;
    const float *h0, *d_last;
    float *h_last, *d_h0, *tape;
    uint64_t *pairs;                            // of every part (see RecPart), a number per channel: A and B, all ones until it is published
    uint32_t *states;                           // behind every 32nd part of a sentence
    uint32_t *taken;                            // of every slice, a cache line each: how many of its parts have been started, less one
    int4 *parts;                                // of every part: its sentence, that one's words, the slot of its first part
    float *copy;                                // of h0, which h_last may be written over
    uint32_t *broken;                           // not 0 once a wait has run out: no other waits as long again; behind it the polls of a wait (read with them: a scalar register less)
    int n_trees, n_rows, C, slices, slots, shift, polls;
};

// ---- channels of a lane ----------------------------------------------------------------------

template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) RecRaw {
    T v[V];
};

// Channels base .. base + V - 1, moved back by `back` where they would pass the last one: such a lane reads what its neighbour reads too, and
// writes only what is its own.  Lanes behind the last channel do the same as the lane that has it.  A row's address is the same in all lanes, a lane's
// place in it a 32-bit number of its own.
template <int V> struct RecLane {
    uint32_t base;
    int back;
    bool even;                                  // no lane is moved back
    __device__ RecLane(int slice, int lane, int C)
    {
        const int want = min((slice * 64 + lane) * V, (C - 1) / V * V);
        back = max(want + V - C, 0);
        base = want - back;
        even = V == 1 || C % V == 0;
    }
    template <typename T> __device__ RecRaw<T, V> raw(const T *row) const
    {
        return *reinterpret_cast<const RecRaw<T, V> *>(reinterpret_cast<const char *>(row) + base * (uint32_t)sizeof(T));
    }
    template <typename T> __device__ void load(const T *row, float (&v)[V]) const
    {
        const RecRaw<T, V> r = raw(row);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)r.v[j];
    }
    template <typename T> __device__ void store(T *row, const float (&v)[V]) const
    {
        char *const at = reinterpret_cast<char *>(row) + base * (uint32_t)sizeof(T);
        RecRaw<T, V> r;
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = (T)v[j];
        if (even) {
            *reinterpret_cast<RecRaw<T, V> *>(at) = r;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j >= back) reinterpret_cast<T *>(at)[j] = r.v[j];
        }
    }
};

// (A gate's exponent is a rounded product, so that the gate is off by 2 |g| 2^-24 of itself, and the exponential gives no subnormal numbers: a gate below 2^-126 is zero.  More of either
// would take instructions for every gate, which are made twice in parts.)
template <int GATE> __device__ inline void rec_gates(float g, float &f, float &i)
{
    if constexpr (GATE == TL_GATE_SIGMOID) {
        const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g));     // sigmoid of |g| and of -|g|, neither by a difference
        const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
        f = g >= 0.f ? big : small;
        i = g >= 0.f ? small : big;
    } else {
        f = g;
        i = 1.f;
    }
}

// ---- what pairs may be trusted with --------------------------------------------------------------
//
// A state s goes through a run of n words as A s + B.  That is the loop's result, but for last bits, if nothing overflows between and the product A has its bits.  A product that
// vanishes, or is subnormal, is off by n 2^-149, and the state by that times s: 2^-120 of it at most, for n up to 2^13 and products of the runs before up to
// REC_PREFIX.  That much is let go (what is lost goes on through the same gates) of states up to REC_LARGE.  Larger ones: sigmoid gates enlarge nothing, so that it is
// in a result's last bits unless the result is 2^-116 of the state; gates of the caller's may, and such a state's words are walked.  A pair says what else it cannot be trusted with:
//   A is NaN        gates above one enlarge something by more than REC_GROW or REC_PREFIX on the way, or what had vanished (the product is taken in one order, gradients pass in the other)
//   B is NaN        inputs above REC_INPUT or sums above REC_LARGE
// and then the words are walked whatever the state.  So no state overflows between unless it is told: 2^60 2^16 2^32 at most, and 2^80 2^32 n from the inputs.
// Chains of runs are joined first and asked about once, by the largest state on the way, and again run by run where that fails.  (Asked about at every joining, two
// sentences of 26 000 words in all took 101 us; 91 so, and 90 without any of this.)

constexpr float REC_LEAST = 0x1p-126f, REC_GROW = 0x1p32f, REC_PREFIX = 0x1p16f, REC_LARGE = 0x1p60f, REC_INPUT = 0x1p80f, REC_RATIO = 0x1p116f;

// The larger of m and |x|, and of m, |x| and |y|, NaN left out (of which products and sums tell).  By hand: a number as it was read would first be made quiet, an instruction more.
__device__ inline void rec_largest(float &m, float x) { asm("v_max_f32 %0, |%1|, %0" : "+v"(m) : "v"(x)); }
__device__ inline void rec_largest(float &m, float x, float y) { asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(m) : "v"(x), "v"(y)); }

// Whether t, which came from states up to `most`, may be something else than what the loop has.
template <int GATE> __device__ inline bool rec_doubt(float most, float t)
{
    return !(fabsf(t) < INFINITY && most <= (GATE == TL_GATE_SIGMOID ? fmaxf(fabsf(t) * REC_RATIO, REC_LARGE) : REC_LARGE));
}

// A chain of runs, a channel: a state B on its way, or the pair A, B of all.
template <int GATE> struct RecChain {
    float A = 1.f, B = 0.f, most = 0.f, above = 0.f;            // the largest state before a run, the largest product so far
    __device__ void state(float P, float Q)
    {
        rec_largest(most, B);
        B = fmaf(P, B, Q);
    }
    __device__ void pair(float P, float Q)
    {
        state(P, Q);
        A *= P;
        if constexpr (GATE == TL_GATE_GIVEN) rec_largest(above, A);
    }
    __device__ bool doubt() const { return rec_doubt<GATE>(most, B); }
    __device__ void settle()
    {
        if (doubt()) B = NAN;
        if (GATE == TL_GATE_GIVEN && above > REC_PREFIX) A = NAN;
    }
};

// The pair of a run that a wave has in registers, once A and B are the products and sums, and D (D_TOO) the sum that comes back: what it says for itself.  f_most, u_most, d_most: the
// largest gate, input and gradient (0 where they do not matter).  gate(k, f): gates of word k; grad(k, j): what comes back to it.
template <int GATE, int V, int R, bool D_TOO, typename F, typename E>
__device__ __forceinline__ void rec_sound(int words, const float (&f_most)[V], const float (&u_most)[V], const float (&d_most)[V], float (&A)[V], float (&B)[V], float (&D)[V], F gate, E grad)
{
    if constexpr (GATE == TL_GATE_GIVEN) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < V; ++j) any = any || f_most[j] > 1.f;
        if (__any(any)) {
            float p[V], least[V], grow[V], m[V], f[V];
            bool closed[V];
#pragma unroll
            for (int j = 0; j < V; ++j) p[j] = least[j] = grow[j] = 1.f, m[j] = 0.f, closed[j] = false;
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (k < words) {
                    gate(k, f);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        closed[j] = closed[j] || f[j] == 0.f;
                        p[j] *= f[j];
                        least[j] = closed[j] ? least[j] : fminf(least[j], fabsf(p[j]));
                        grow[j] *= fmaxf(1.f, fabsf(f[j]));
                    }
                }
            // what comes back in its own order, as the loop takes it
            if constexpr (D_TOO) {
#pragma unroll
                for (int k = R - 1; k >= 0; --k)
                    if (k < words) {
                        gate(k, f);
#pragma unroll
                        for (int j = 0; j < V; ++j) m[j] = f[j] * (grad(k, j) + m[j]);
                    }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (f_most[j] > 1.f && (!(grow[j] <= REC_GROW) || least[j] < REC_LEAST)) A[j] = NAN;
                if constexpr (D_TOO) D[j] = f_most[j] > 1.f ? m[j] : D[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (GATE == TL_GATE_GIVEN && u_most[j] > REC_INPUT) B[j] = NAN;
        if (D_TOO && (rec_doubt<GATE>(d_most[j], D[j]) || d_most[j] > REC_INPUT)) D[j] = NAN;
    }
}

// The state behind words [from, to), whose pair is A, B.
template <typename T, int GATE, int V, bool BACK>
__device__ inline void rec_join(const RecurArgs &a, const RecLane<V> &l, int from, int to, const float (&A)[V], const float (&B)[V], float (&s)[V], bool all = false)
{
    float t[V];
    bool walk[V], any = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        t[j] = fmaf(A[j], s[j], B[j]);
        walk[j] = all || (rec_doubt<GATE>(fabsf(s[j]), t[j]) && s[j] == s[j]);      // (a NaN stays one)
        any = any || walk[j];
    }
    if (__any(any)) {
        float w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = s[j];
#pragma unroll 1
        for (int n = 0; n < to - from; ++n) {
            const long long r = BACK ? to - 1 - n : from + n;
            float g[V], u[V] = {};
            l.load(static_cast<const T *>(a.g) + r * a.g_row, g);
            if (!BACK) l.load(static_cast<const T *>(a.x) + r * a.x_row, u);
            else if (a.d_h) l.load(static_cast<const T *>(a.d_h) + r * a.d_h_row, u);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float f, i;
                rec_gates<GATE>(g[j], f, i);
                w[j] = BACK ? f * (w[j] + u[j]) : fmaf(f, w[j], i * u[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = walk[j] ? w[j] : t[j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = t[j];
}

// c through the runs of the waves from `first` on, of R words from `block` on each (BACK: of those before it), as far as `wave`, in front of whose run it is s; unless that ends
// it, on behind the last one.  pair(w, 0, j), pair(w, 1, j): what wave w found.  Whether a channel has to be joined run by run, from where it began.
template <int GATE, int V, int W, int R, bool BACK, typename F>
__device__ __forceinline__ bool rec_steps(int block, int end, int first, int wave, bool ends, float (&c)[V], float (&s)[V], bool (&bad)[V], F pair)
{
    RecChain<GATE> t[V];
    bool any = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        t[j].B = c[j];
        bad[j] = false;
    }
#pragma unroll 1
    for (int w = first; BACK ? w >= 0 : w < W; w += BACK ? -1 : 1) {
        if (w == wave) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] = t[j].B;
                bad[j] = t[j].doubt();
            }
            if (ends) break;
        }
        if (block + w * R >= end) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) t[j].state(pair(w, 0, j), pair(w, 1, j));
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        c[j] = t[j].B;
        bad[j] = bad[j] || (!ends && t[j].doubt());
        any = any || bad[j];
    }
    return any;
}
// The same run by run from `from` on, for channels that have to be.
template <typename T, int GATE, int V, int W, int R, bool BACK, typename F>
__device__ __forceinline__ void rec_steps_again(const RecurArgs &a, const RecLane<V> &l, int block, int end, int first, int wave, bool ends, const float (&from)[V], const bool (&bad)[V],
                                                float (&c)[V], float (&s)[V], F pair)
{
    float r[V], A[V], B[V];
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = from[j];
#pragma unroll 1
    for (int w = first; BACK ? w >= 0 : w < W; w += BACK ? -1 : 1) {
        if (w == wave) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = bad[j] ? r[j] : s[j];
            if (ends) break;
        }
        const int begin = block + w * R;
        if (begin >= end) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = pair(w, 0, j), B[j] = pair(w, 1, j);
        rec_join<T, GATE, V, BACK>(a, l, begin, min(begin + R, end), A, B, r);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = bad[j] ? r[j] : c[j];
}

// ---- which words a workgroup has -------------------------------------------------------------

// A sentence has a slot for every part, and at most one more: slot off / words + sentence on.  (Offsets are kept inside the batch, whatever they hold.)
struct RecPart {
    int tree, slot0;                            // the sentence, and the slot of its first part
    int lo, hi;                                 // its words
    int part, parts;
    int first, end;                             // the words of this part
    bool there;
    __device__ void take(int n, int size)
    {
        part = n;
        first = (int)min(lo + (long long)n * size, (long long)hi);
        end = (int)min((long long)first + size, (long long)hi);
    }
    template <bool CUT> __device__ static RecPart of(const RecurArgs &a, int slot)
    {
        RecPart p;
        if constexpr (CUT) {
            const int4 r = a.parts[slot];
            p.tree = __builtin_amdgcn_readfirstlane(r.x);
            p.lo = __builtin_amdgcn_readfirstlane(r.y);
            p.hi = __builtin_amdgcn_readfirstlane(r.z);
            p.slot0 = __builtin_amdgcn_readfirstlane(r.w);
            const int size = 1 << a.shift;
            p.parts = max((int)(((long long)p.hi - p.lo + size - 1) >> a.shift), 1);
            p.there = slot - p.slot0 >= 0 && slot - p.slot0 < p.parts;
            p.take(slot - p.slot0, size);
        } else {
            p.tree = p.slot0 = slot;
            tree_range(a.off, slot, a.n_rows, &p.lo, &p.hi);
            p.part = 0;
            p.parts = 1;
            p.first = p.lo;
            p.end = p.hi;
            p.there = true;
        }
        return p;
    }
};

// R words from `row` on (as far as `end`; beyond it the last one again) of one tensor, as they lie in memory; zeros where there is none.
template <typename T, int V, int R> struct RecRows {
    static constexpr int WORDS = V * (int)sizeof(T) / 4;        // registers of a row; 0: a single 16-bit value
    struct Row {
        uint32_t w[WORDS > 0 ? WORDS : 1];
    };
    Row r[R];
    __device__ void clear()
    {
#pragma unroll
        for (int k = 0; k < R; ++k) r[k] = {};
    }
    // ONCE: nothing reads the rows again, so they need no place in the caches.
    template <bool ONCE = false> __device__ void load(const void *p, long long stride, const RecLane<V> &l, int row, int end)
    {
        typedef uint32_t Vec __attribute__((ext_vector_type(WORDS > 1 ? WORDS : 2)));
        typedef Vec __attribute__((aligned(2))) Many;
        typedef uint32_t __attribute__((aligned(2))) One;
        const T *at = static_cast<const T *>(p) + row * stride;
        const int more = end - 1 - row;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const char *const here = reinterpret_cast<const char *>(at) + l.base * (uint32_t)sizeof(T);
            if constexpr (ONCE && WORDS == 1) {
                r[k].w[0] = __builtin_nontemporal_load(reinterpret_cast<const One *>(here));
            } else if constexpr (ONCE && WORDS > 1) {
                const Vec v = __builtin_nontemporal_load(reinterpret_cast<const Many *>(here));
                __builtin_memcpy(&r[k], &v, sizeof(v));
            } else {
                const RecRaw<T, V> v = l.raw(at);
                __builtin_memcpy(&r[k], &v, sizeof(v));
            }
            at += k < more ? stride : 0;
        }
    }
    __device__ float get(int k, int j) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(r[k].w[j]);
        const uint32_t w = r[k].w[j / 2];
        if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float(j % 2 ? w & 0xffff0000u : w << 16);
        const uint16_t half = (uint16_t)(j % 2 ? w >> 16 : w);
        f16_t v;
        __builtin_memcpy(&v, &half, 2);
        return (float)v;
    }
    // What is computed from the rows after this is computed anew: registers hold the rows, not the results.
    __device__ void forget()
    {
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int n = 0; n < (WORDS > 0 ? WORDS : 1); ++n) asm volatile("" : "+v"(r[k].w[n]));
    }
};

// The gates of R words: held (KEEP), or made again from the words wherever they are needed.
template <typename T, int V, int R, int GATE, bool KEEP> struct RecGates {
    RecRows<T, V, R> g;
    float f[KEEP ? R : 1][V], i[KEEP ? R : 1][V];
    __device__ explicit RecGates(const RecRows<T, V, R> &rows) : g(rows)
    {
        if constexpr (KEEP)
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) rec_gates<GATE>(g.get(k, j), f[k][j], i[k][j]);
    }
    __device__ __forceinline__ void at(int k, float (&F)[V], float (&I)[V]) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (KEEP) F[j] = f[k][j], I[j] = i[k][j];
            else rec_gates<GATE>(g.get(k, j), F[j], I[j]);
        }
    }
    __device__ void forget()
    {
        if constexpr (!KEEP) g.forget();
    }
};

// ---- parts of a sentence -------------------------------------------------------------------------
//
// A part's pair needs nothing but the part's own words, so a workgroup that waits for pairs waits for workgroups that wait for nothing.  A state is
// published behind every 32nd part: a part needs the state behind the last such part before it, and the pairs from there on, 31 at most.  Values are
// published as they are, in words that were filled with ones before: a word that is no longer all ones is complete, and no fence is needed.
// Parts are numbered in the order in which a state passes them.  A workgroup takes the next number of its slice when it starts: the hardware starts them in order within an XCD only, and two
// launches side by side could else fill one another's units with workgroups that wait for such as find no place.  So what is waited for has been started (a lane that is moved back
// waits for its own channels alone).  It costs an atomic add's way a workgroup: two sentences of 26 000 words in all 94 us, 91 without.  Every wait ends all the same: after REC_POLLS polls (tenths of a second), or as
// many as the caller allows, the words in question are walked, from the start of the sentence.

constexpr int REC_GROUP = 32, REC_POLLS = 1 << 16, REC_LINE = 32;
constexpr uint32_t REC_NAN = 0x7fc00000u;       // published for a NaN that is all ones

__device__ inline uint32_t rec_bits(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b == ~0u ? REC_NAN : b;
}

template <int V> __device__ inline void rec_publish(uint64_t *at, const RecLane<V> &l, const float (&A)[V], const float (&B)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= l.back) __hip_atomic_store(at + l.base + j, (uint64_t)rec_bits(A[j]) << 32 | rec_bits(B[j]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int V> __device__ inline void rec_publish(uint32_t *at, const RecLane<V> &l, const float (&s)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= l.back) __hip_atomic_store(at + l.base + j, rec_bits(s[j]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Whether the words came.
template <int V, int N, typename W> __device__ inline bool rec_wait(const RecurArgs &a, W *const (&at)[N], int n, const RecLane<V> &l, W (&v)[N][V])
{
#pragma unroll 1
    for (int poll = 1;; ++poll) {
        bool there = true;
        const uint64_t how = __hip_atomic_load(reinterpret_cast<uint64_t *>(a.broken), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < n)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v[k][j] = __hip_atomic_load(at[k] + l.base + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    if (V > 1 && j < l.back) v[k][j] = 0;
                    there = there && v[k][j] != (W)~(W)0;
                }
        const int polls = __builtin_amdgcn_readfirstlane((int)(how >> 32));
        if (__all(there) && polls > 0) return true;
        if (poll >= polls) break;
        if ((poll & 255) == 0 && __builtin_amdgcn_readfirstlane((uint32_t)how) != 0) return false;
        __builtin_amdgcn_s_sleep(1);
    }
    __hip_atomic_store(a.broken, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return false;
}

// A pair that is there.
template <int V> __device__ inline void rec_taken(const RecurArgs &a, int slot, const RecLane<V> &l, float (&A)[V], float (&B)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint64_t v = V > 1 && j < l.back ? 0 : __hip_atomic_load(a.pairs + (long long)slot * a.C + l.base + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        A[j] = __uint_as_float((uint32_t)(v >> 32));
        B[j] = __uint_as_float((uint32_t)v);
    }
}

template <int V, int W> struct RecEnter {
    float pair[W][2][V][64], state[V][64];
    int late;
};

// s becomes the state in front of a part's first word, or (BACK) what comes back to its last one; in wave 0 it is the one at the sentence's own end before.  Every
// wave joins an even share of the pairs to one, all join these.  (e.late was set to zero in front of a barrier.)
template <typename T, int GATE, int V, int W, bool BACK>
__device__ inline void rec_enter(const RecurArgs &a, const RecPart &p, const RecLane<V> &l, int wave, RecEnter<V, W> &e, float (&s)[V])
{
    constexpr int SHARE = (REC_GROUP - 1 + W - 1) / W;
    const int lane = threadIdx.x & 63, size = 1 << a.shift;
    const int nth = BACK ? p.parts - 1 - p.part : p.part, group = nth & ~(REC_GROUP - 1), many = nth - group;
    auto slot = [&](int n) { return p.slot0 + (BACK ? p.parts - 1 - n : n); };
    bool fine = true;
    if (wave == 0) {
        if (group > 0) {
            uint32_t *const at[1] = {a.states + (long long)(slot(group - 1) / REC_GROUP) * a.C};
            uint32_t v[1][V];
            fine = rec_wait<V, 1>(a, at, 1, l, v);
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = __uint_as_float(v[0][j]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) e.state[j][lane] = s[j];
    }
    const int first = wave * SHARE, n = min(SHARE, many - first);
    if (n > 0) {
        constexpr int N = SHARE < 4 ? SHARE : 4;
        RecChain<GATE> c[V];
#pragma unroll 1
        for (int i = 0; i < n; i += N) {
            uint64_t *at[N], v[N][V];
#pragma unroll
            for (int k = 0; k < N; ++k) at[k] = a.pairs + (long long)slot(group + first + min(i + k, n - 1)) * a.C;
            fine = rec_wait<V, N>(a, at, n - i, l, v) && fine;
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (i + k < n)
#pragma unroll
                    for (int j = 0; j < V; ++j) c[j].pair(__uint_as_float((uint32_t)(v[k][j] >> 32)), __uint_as_float((uint32_t)v[k][j]));
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            c[j].settle();
            e.pair[wave][0][j][lane] = c[j].A, e.pair[wave][1][j][lane] = c[j].B;
        }
    }
    if (!fine) e.late = 1;
    __syncthreads();
    const bool late = e.late != 0;
    float t[V];
    bool bad[V], any = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        RecChain<GATE> c;
        c.B = s[j] = e.state[j][lane];
        for (int w = 0; w * SHARE < many; ++w) c.state(e.pair[w][0][j][lane], e.pair[w][1][j][lane]);
        t[j] = c.B;
        bad[j] = late || c.doubt();
        any = any || bad[j];
    }
    if (__any(any)) {
        // part by part from the published state, of pairs that are all there; or from the sentence's own end, every word
        float w[V];
        const float *const from = BACK ? a.d_last : a.copy;
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = late ? 0.f : s[j];
        if (late && from) l.load(from + (long long)p.tree * a.C, w);
#pragma unroll 1
        for (int n = late ? 0 : group; n < nth; ++n) {
            const int at = slot(n) - p.slot0;
            float A[V], B[V];
            rec_taken<V>(a, slot(n), l, A, B);                          // (whatever it is, where all words are walked)
            rec_join<T, GATE, V, BACK>(a, l, p.lo + at * size, (int)min(p.lo + (at + 1ll) * size, (long long)p.hi), A, B, w, late);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = bad[j] ? w[j] : t[j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = t[j];
}

// What the parts need before they start: what each of them is, words of ones, and a copy of h0.
__global__ __launch_bounds__(256) void k_recur_prepare(RecurArgs a, long long n_words, long long n_copy)
{
    const long long at = blockIdx.x * 256ll + threadIdx.x, step = (long long)gridDim.x * 256;
    for (long long slot = at; slot < a.slots; slot += step) {
        auto place = [&](int t) { return min(max(a.off[t], 0), a.n_rows); };
        int t = 0, n = a.n_trees;               // the last sentence whose slots do not begin behind this one
        while (n > 1) {
            const int half = n >> 1, base = (place(t + half) >> a.shift) + t + half;
            t = base <= slot ? t + half : t;
            n -= half;
        }
        const int lo = place(t);
        a.parts[slot] = int4{t, lo, max(place(t + 1), lo), (lo >> a.shift) + t};
    }
    if (at < 2) a.broken[at] = at ? (uint32_t)a.polls : 0;
    for (long long i = at; i < n_words; i += step) a.pairs[i] = ~0ull;      // (pairs, and behind them states and numbers of parts)
    if (a.copy)
        for (long long i = at; i < n_copy; i += step) a.copy[i] = a.h0[i];
}

// Which part a workgroup takes: as many as workgroups of its slice have started before it.
__device__ inline int rec_take(const RecurArgs &a, int slice)
{
    __shared__ uint32_t number;
    if (threadIdx.x == 0) number = __hip_atomic_fetch_add(a.taken + slice * REC_LINE, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(number);
}

// Where a sentence's words begin: its row of h0, or (BACK) of what comes back from behind them.
template <int V> __device__ inline void rec_start(const float *from, const RecPart &p, const RecLane<V> &l, int C, float (&s)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    if (from) l.load(from + (long long)p.tree * C, s);
}

__device__ inline float *rec_tape(const RecurArgs &a, const RecPart &p, int row)
{
    return a.tape + ((long long)(p.lo / REC_TAPE) + p.tree + (row - p.lo) / REC_TAPE) * a.C;
}

// ---- forward -----------------------------------------------------------------------------------

// f(k) for the first `words` of R words, in order.
template <int R, typename F> __device__ __forceinline__ void rec_each(int words, F f)
{
    if (words >= R) {
#pragma unroll
        for (int k = 0; k < R; ++k) f(k);
    } else {
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < words) f(k);
    }
}
template <int R, typename F> __device__ __forceinline__ void rec_each_back(int words, F f)
{
    if (words >= R) {
#pragma unroll
        for (int k = R - 1; k >= 0; --k) f(k);
    } else {
#pragma unroll
        for (int k = R - 1; k >= 0; --k)
            if (k < words) f(k);
    }
}

// CUT: a part of W R words, else a whole sentence, W R words at a time; AHEAD: the next block's rows are on their way while one is worked on.  Memory bounds long batches
// (256 sentences of 750 words x 512 bf16: 139 us, 4.2 TB/s; two of 13 000 x 2048: 92, 3.5, the vector unit 52 % busy), a block's chain of offsets, rows, pairs and
// states short ones (256 of 33 x 512 bf16: 10, of which bytes are 5).  A row is read in 4 bytes a lane: 8 take twice the registers and were slower (13 for 11).  In a part the registers hold the words as they were read, which are put through
// their gates twice, for the pair and for the states: that costs less than the registers of the results, which would halve the waves of a compute unit.
// ONCE: nothing reads g and x again (there is no tape); a branch on the tape in the kernel would cost what the other loads gain.  Measured (us, two sentences of
// 26 000 words in all, bf16 x 2048): 100 with ordinary loads, 94 so; a training step of eight of 1 800 words x 1024: 81.6 and 83.0.
template <typename T, int V, int W, int R, int GATE, bool CUT, bool ONCE, bool AHEAD> __global__ __launch_bounds__(64 * W) void k_recur(RecurArgs a)
{
    static_assert(REC_TAPE % R == 0, "states of the tape lie where a wave's words begin");
    static_assert(!(CUT && AHEAD), "a part is one block");
    constexpr bool KEEP = AHEAD && W > 1, WIDE = sizeof(T) == 4 || std::is_same<T, bf16_t>::value;      // (no fp16 number is above REC_INPUT)
    __shared__ float lds[W > 1 && !CUT ? 2 : 1][W][2][V][64];
    __shared__ RecEnter<V, W> enter[1];                         // (CUT only)
    __shared__ float begin_state[V][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int nth = blockIdx.x / a.slices, slice = blockIdx.x - nth * a.slices, slot = CUT ? rec_take(a, slice) : nth;
    const RecPart p = RecPart::of<CUT>(a, slot);
    if (!p.there) return;
    const RecLane<V> l(slice, lane, a.C);
    RecRows<T, V, R> g, x;
    auto load = [&](int row) {
        g.clear();                                              // (so that what was there ends here)
        x.clear();
        if (row >= p.end) return;
        g.template load<ONCE>(a.g, a.g_row, l, row, p.end);
        x.template load<ONCE>(a.x, a.x_row, l, row, p.end);
    };
    load(p.first + wave * R);
    // (one wave reads h0 and hands it on: h_last may lie in the same place, and must not be written before it has been read)
    float c[V] = {};
    if (wave == 0) {
        rec_start(CUT ? a.copy : a.h0, p, l, a.C, c);
#pragma unroll
        for (int j = 0; j < V; ++j) begin_state[j][lane] = c[j];
    }
    if (p.lo == p.hi) {                                         // no words
        if (a.h_last && wave == 0) l.store(a.h_last + (long long)p.tree * a.C, c);
        return;
    }
    if constexpr (CUT)
        if (threadIdx.x == 0) enter[0].late = 0;
    int buf = 0;
#pragma unroll 1
    for (int block = p.first;; block += W * R) {
        const int row = block + wave * R, words = p.end - row;
        RecGates<T, V, R, GATE, KEEP> G(g);
        RecRows<T, V, R> X = x;
        const bool more = !CUT && block + W * R < p.end;
        if (AHEAD && more) load(row + W * R);
        float f[V], i[V], s[V];
        if constexpr (W > 1) {
            float A[V], B[V], D[V], f_most[V], u_most[V], d_most[V];
#pragma unroll
            for (int j = 0; j < V; ++j) A[j] = 1.f, B[j] = D[j] = f_most[j] = u_most[j] = d_most[j] = 0.f;
            rec_each<R>(words, [&](int k) __attribute__((always_inline)) {
                G.at(k, f, i);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    A[j] *= f[j];
                    B[j] = fmaf(f[j], B[j], i[j] * X.get(k, j));
                    if constexpr (GATE == TL_GATE_GIVEN) {
                        if (k % 2 == 0) {                       // (behind the last word it is there again)
                            rec_largest(f_most[j], G.g.get(k, j), G.g.get(k + 1, j));
                            if constexpr (WIDE) rec_largest(u_most[j], X.get(k, j), X.get(k + 1, j));
                        }
                    }
                }
            });
            rec_sound<GATE, V, R, false>(words, f_most, u_most, d_most, A, B, D, [&](int k, float (&F)[V]) __attribute__((always_inline)) { float I[V]; G.at(k, F, I); },
                                         [](int, int) { return 0.f; });
            G.forget();
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds[buf][wave][0][j][lane] = A[j];
                lds[buf][wave][1][j][lane] = B[j];
            }
            __syncthreads();                                    // (the other buffer is written only after the next one)
            if (block == p.first)
#pragma unroll
                for (int j = 0; j < V; ++j) c[j] = begin_state[j][lane];
            if constexpr (CUT)
                if (p.parts > 1) {
                    if (wave == 0 && p.part < p.parts - 1) {
                        RecChain<GATE> t[V];
#pragma unroll
                        for (int w = 0; w < W; ++w)
#pragma unroll
                            for (int j = 0; j < V; ++j) t[j].pair(lds[0][w][0][j][lane], lds[0][w][1][j][lane]);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            t[j].settle();
                            A[j] = t[j].A, B[j] = t[j].B;
                        }
                        rec_publish(a.pairs + (long long)slot * a.C, l, A, B);
                    }
                    rec_enter<T, GATE, V, W, false>(a, p, l, wave, enter[0], c);
                }
            float from[V];
            bool bad[V];
            auto pair = [&](int w, int n, int j) __attribute__((always_inline)) { return lds[buf][w][n][j][lane]; };
#pragma unroll
            for (int j = 0; j < V; ++j) from[j] = c[j];
            if (__any(rec_steps<GATE, V, W, R, false>(block, p.end, 0, wave, CUT, c, s, bad, pair)))
                rec_steps_again<T, GATE, V, W, R, false>(a, l, block, p.end, 0, wave, CUT, from, bad, c, s, pair);
            if (!CUT) buf ^= 1;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = c[j];
        }
        if (a.tape && words > 0 && ((row - p.lo) & (REC_TAPE - 1)) == 0) l.store(rec_tape(a, p, row), s);
        T *h = static_cast<T *>(a.h) + row * a.h_row;
        rec_each<R>(words, [&](int k) __attribute__((always_inline)) {
            G.at(k, f, i);
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = fmaf(f[j], s[j], i[j] * X.get(k, j));
            l.store(h, s);
            h += a.h_row;
        });
        if (a.h_last && words > 0 && row + R >= p.hi) l.store(a.h_last + (long long)p.tree * a.C, s);
        if constexpr (CUT)
            if (wave == W - 1 && p.part < p.parts - 1 && p.part % REC_GROUP == REC_GROUP - 1) rec_publish(a.states + (long long)(slot / REC_GROUP) * a.C, l, s);
        if constexpr (W == 1)
#pragma unroll
            for (int j = 0; j < V; ++j) c[j] = s[j];
        if (!more) break;
        if (!AHEAD) load(row + W * R);
    }
}

// ---- gradients -----------------------------------------------------------------------------------

// Blocks from the last one to the first.  A block's words are stepped through from the tape's state first, for what each gate's gradient needs, then backwards.  Bound by memory:
// 256 sentences of 33 words x 512 fp32 21 to 22 us for 85 MB, eight of 1 800 x 1024 bf16 43 for 146 MB (one and a half rounds of workgroups).
// Registers: as many as leave a SIMD the waves that it would have without the code for words that are walked, which would take one wave's (fp32 256 x 33 x 512, with states: 39 us for 34).
template <typename T, int V, int W, int R, int GATE, bool CUT, bool AHEAD>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(!AHEAD ? 4 : V == 1 ? 3 : 2))) void k_recur_back(RecurArgs a)
{
    static_assert((W * R) % REC_TAPE == 0, "a block starts from a state of the tape");
    static_assert(!(CUT && AHEAD), "a part is one block");
    constexpr bool KEEP = AHEAD, WIDE = sizeof(T) == 4 || std::is_same<T, bf16_t>::value;
    __shared__ float lds[CUT ? 1 : 2][W][3][V][64];
    __shared__ RecEnter<V, W> enter[1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    // (from behind, as gradients pass them)
    const int nth = blockIdx.x / a.slices, slice = blockIdx.x - nth * a.slices, slot = a.slots - 1 - (CUT ? rec_take(a, slice) : nth);
    const RecLane<V> l(slice, lane, a.C);
    {   // rows behind the last sentence
        const int tail = min(max(__builtin_amdgcn_readfirstlane(a.off[a.n_trees]), 0), a.n_rows);
        const float none[V] = {};
        for (long long r = rec_behind(tail, slot, wave, a.slots); r < a.n_rows; r += (long long)W * a.slots) {
            l.store(static_cast<T *>(a.d_g) + r * a.d_g_row, none);
            l.store(static_cast<T *>(a.d_x) + r * a.d_x_row, none);
        }
    }
    const RecPart p = RecPart::of<CUT>(a, slot);
    if (!p.there) return;
    float c[V];
    rec_start(a.d_last, p, l, a.C, c);
    if (p.lo == p.hi) {
        if (a.d_h0 && wave == 0) l.store(a.d_h0 + (long long)p.tree * a.C, c);
        return;
    }
    RecRows<T, V, R> g, x, d;
    float s0[V];
    auto load = [&](int block) {
        const int row = block + wave * R;
        l.load(rec_tape(a, p, block), s0);
        g.clear();
        x.clear();
        d.clear();
        if (row >= p.end) return;
        g.load(a.g, a.g_row, l, row, p.end);
        x.load(a.x, a.x_row, l, row, p.end);
        if (a.d_h) d.load(a.d_h, a.d_h_row, l, row, p.end);     // (zeros else)
    };
    const int blocks = (p.end - p.first + W * R - 1) / (W * R);
    load(p.first + (blocks - 1) * (W * R));
    if constexpr (CUT)
        if (threadIdx.x == 0) enter[0].late = 0;
    int buf = 0;
#pragma unroll 1
    for (int n = blocks - 1;; --n) {
        const int block = p.first + n * (W * R), row = block + wave * R, words = p.end - row;
        RecGates<T, V, R, GATE, KEEP> G(g);
        RecRows<T, V, R> X = x, E = d;
        float f[V], i[V], s[V], m[V], A[V], B[V], D[V], f_most[V], u_most[V], d_most[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s[j] = s0[j];
            A[j] = 1.f, B[j] = D[j] = f_most[j] = u_most[j] = d_most[j] = 0.f;
        }
        const bool more = !CUT && n > 0;
        if (AHEAD && more) load(block - W * R);
        rec_each<R>(words, [&](int k) __attribute__((always_inline)) {
            G.at(k, f, i);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                A[j] *= f[j];
                B[j] = fmaf(f[j], B[j], i[j] * X.get(k, j));
                D[j] = fmaf(A[j], E.get(k, j), D[j]);           // (what comes back from word k passes the gates of words 0 .. k)
                if (k % 2 == 0) {                               // (behind the last word it is there again)
                    if constexpr (GATE == TL_GATE_GIVEN) {
                        rec_largest(f_most[j], G.g.get(k, j), G.g.get(k + 1, j));
                        if constexpr (WIDE) rec_largest(u_most[j], X.get(k, j), X.get(k + 1, j));
                    }
                    if constexpr (WIDE) rec_largest(d_most[j], E.get(k, j), E.get(k + 1, j));
                }
            }
        });
        rec_sound<GATE, V, R, true>(words, f_most, u_most, d_most, A, B, D, [&](int k, float (&F)[V]) __attribute__((always_inline)) { float I[V]; G.at(k, F, I); },
                                    [&](int k, int j) __attribute__((always_inline)) { return E.get(k, j); });
        G.forget();
#pragma unroll
        for (int j = 0; j < V; ++j) {
            lds[buf][wave][0][j][lane] = A[j];
            lds[buf][wave][1][j][lane] = B[j];
            lds[buf][wave][2][j][lane] = D[j];
        }
        __syncthreads();
        if constexpr (CUT)
            if (p.parts > 1) {
                if (wave == W - 1 && p.part > 0) {
                    RecChain<GATE> t[V];
#pragma unroll 4
                    for (int w = W - 1; w >= 0; --w)
#pragma unroll
                        for (int j = 0; j < V; ++j) t[j].pair(lds[0][w][0][j][lane], lds[0][w][2][j][lane]);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        t[j].settle();
                        A[j] = t[j].A, D[j] = t[j].B;
                    }
                    rec_publish(a.pairs + (long long)slot * a.C, l, A, D);
                }
                rec_enter<T, GATE, V, W, true>(a, p, l, wave, enter[0], c);
            }
        {
            float from[V], from_back[V], here[V];
            bool bad[V], bad_back[V];
            auto pair = [&](int w, int n, int j) __attribute__((always_inline)) { return lds[buf][w][n][j][lane]; };
            auto pair_back = [&](int w, int n, int j) __attribute__((always_inline)) { return lds[buf][w][2 * n][j][lane]; };
#pragma unroll
            for (int j = 0; j < V; ++j) from[j] = s[j], from_back[j] = c[j];
            const bool any = rec_steps<GATE, V, W, R, false>(block, p.end, 0, wave, true, s, here, bad, pair);
            const bool any_back = rec_steps<GATE, V, W, R, true>(block, p.end, W - 1, wave, CUT, c, m, bad_back, pair_back);
            if (__any(any || any_back)) {
                rec_steps_again<T, GATE, V, W, R, false>(a, l, block, p.end, 0, wave, true, from, bad, s, here, pair);
                rec_steps_again<T, GATE, V, W, R, true>(a, l, block, p.end, W - 1, wave, CUT, from_back, bad_back, c, m, pair_back);
            }
        }
        if (!CUT) buf ^= 1;
        // forwards: what a word's own lambda is multiplied by in the gradient of its gate, but for f i
        float q[R][V];
        rec_each<R>(words, [&](int k) __attribute__((always_inline)) {
            G.at(k, f, i);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = X.get(k, j);
                q[k][j] = GATE == TL_GATE_SIGMOID ? s[j] - v : s[j];
                s[j] = fmaf(f[j], s[j], i[j] * v);
            }
        });
        G.forget();
        const int top = min(words, R) - 1;
        T *at_g = static_cast<T *>(a.d_g) + (row + top) * a.d_g_row, *at_x = static_cast<T *>(a.d_x) + (row + top) * a.d_x_row;
        rec_each_back<R>(words, [&](int k) __attribute__((always_inline)) {
            G.at(k, f, i);
            float dg[V], dx[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float lambda = E.get(k, j) + m[j];
                dx[j] = lambda * i[j];
                m[j] = lambda * f[j];
                dg[j] = (GATE == TL_GATE_SIGMOID ? m[j] * i[j] : lambda) * q[k][j];
            }
            l.store(at_g, dg);
            l.store(at_x, dx);
            at_g -= a.d_g_row;
            at_x -= a.d_x_row;
        });
        if (wave == 0) {
            if (a.d_h0 && block == p.lo) l.store(a.d_h0 + (long long)p.tree * a.C, m);
            if (CUT && p.part > 0 && (p.parts - 1 - p.part) % REC_GROUP == REC_GROUP - 1) rec_publish(a.states + (long long)(slot / REC_GROUP) * a.C, l, m);
        }
        if (!more) break;
        if (!AHEAD) load(block - W * R);
    }
}

}  // namespace tl
