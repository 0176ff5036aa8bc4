// A gated linear recurrence along the words of ragged sentences, and its gradients.
//
//   h_t = f_t h_(t-1) + i_t x_t            per channel; f = sigmoid(g), i = sigmoid(-g), or f = g, i = 1
//   mu_t = f_t (dh_t + mu_(t+1))           what goes back to word t - 1; lambda_t = dh_t + mu_(t+1)
//   dx_t = i_t lambda_t,   dg_t = lambda_t (h_(t-1) - x_t) f_t i_t   (f = g: lambda_t h_(t-1)),   dh0 = mu of the first word
//
// Both are linear maps of a state, so that a run of words is one pair (A, B), state -> A state + B, and pairs of runs side by side join
// to one.  A lane owns V channels; a wave takes R words, a workgroup W R words at a time: a wave forms the pair of its words from registers, the
// pairs are exchanged through LDS, and each wave then steps through its words once more, from the state that is its own.  Sentences that are few
// and long are cut into parts: a first launch writes the pair of every part, the second one starts each part from the pairs before it.
//
// The backward pass needs h_(t-1) in fp32 for every word.  It reads no h: the forward keeps the state of every 64th word (the tape, 1/64 of the
// states in fp32), and a block of 64 words is stepped through again from there.  So five tensors move instead of six, and a 16-bit h's
// rounding is in no gradient.
//
// A pair can overflow, or multiply an infinity by a zero, where the words one after the other do neither.  So where joining gives
// something that is not finite, the words in question are walked one by one for that channel: infinities and NaN come out as the formula has them.
#pragma once

#include "attend.hpp"

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
    float *pairs;                               // of every part (see find_slot): A [channels], then B; a cut sentence's last part holds a copy of h0 instead
    int n_trees, n_rows, C, slices, slots, shift;
};

// ---- channels of a lane ----------------------------------------------------------------------

template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) RecRaw {
    T v[V];
};

// Channels base .. base + V - 1, moved back by `back` where they would pass the last one: such a lane reads what its neighbour reads too, and
// writes only what is its own.
template <int V> struct RecLane {
    int base, back;
    bool on;
    __device__ RecLane(int slice, int lane, int C)
    {
        const int want = (slice * 64 + lane) * V;
        on = want < C;
        back = on ? max(want + V - C, 0) : 0;
        base = on ? want - back : 0;
    }
    template <typename T> __device__ void load(const T *p, float (&v)[V]) const
    {
        const RecRaw<T, V> r = *reinterpret_cast<const RecRaw<T, V> *>(p + base);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)r.v[j];
    }
    template <typename T> __device__ void store(T *p, const float (&v)[V]) const
    {
        if (!on) return;
        if (back == 0) {
            RecRaw<T, V> r;
#pragma unroll
            for (int j = 0; j < V; ++j) r.v[j] = (T)v[j];
            *reinterpret_cast<RecRaw<T, V> *>(p + base) = r;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j >= back) p[base + j] = (T)v[j];
        }
    }
};

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

__device__ inline bool rec_finite(float x) { return fabsf(x) < INFINITY; }

// Words [from, to) of one channel, one by one.
template <typename T, int GATE> __device__ __noinline__ float rec_walk(const RecurArgs &a, int from, int to, int c, float s)
{
    for (int r = from; r < to && s == s; ++r) {
        float f, i;
        rec_gates<GATE>((float)static_cast<const T *>(a.g)[r * a.g_row + c], f, i);
        s = f * s + i * (float)static_cast<const T *>(a.x)[r * a.x_row + c];
    }
    return s;
}
template <typename T, int GATE> __device__ __noinline__ float rec_walk_back(const RecurArgs &a, int from, int to, int c, float m)
{
    for (int r = to - 1; r >= from && m == m; --r) {
        float f, i;
        rec_gates<GATE>((float)static_cast<const T *>(a.g)[r * a.g_row + c], f, i);
        m = f * (m + (a.d_h ? (float)static_cast<const T *>(a.d_h)[r * a.d_h_row + c] : 0.f));
    }
    return m;
}

// The state behind words [from, to), whose pair is A, B.
template <typename T, int GATE, int V, bool BACK>
__device__ inline void rec_join(const RecurArgs &a, const RecLane<V> &l, int from, int to, const float (&A)[V], const float (&B)[V], float (&s)[V])
{
    float t[V];
    bool fine = true;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        t[j] = fmaf(A[j], s[j], B[j]);
        fine = fine && rec_finite(t[j]);
    }
    if (!fine && l.on) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (!rec_finite(t[j])) t[j] = BACK ? rec_walk_back<T, GATE>(a, from, to, l.base + j, s[j]) : rec_walk<T, GATE>(a, from, to, l.base + j, s[j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = t[j];
}

// ---- which words a workgroup has -------------------------------------------------------------

struct RecPart {
    int tree, slot0;                            // the sentence, and the slot of its first part
    int lo, hi;                                 // its words
    int part, parts;
    int first, end;                             // the words of this part
    bool there;
    __device__ RecPart(const RecurArgs &a, int slot)
    {
        // (places as in find_slot, of offsets kept inside the batch: pairs are looked up by them)
        auto base = [&](int t) { return (min(max(a.off[t], 0), a.n_rows) >> a.shift) + t; };
        tree = a.shift == REC_WHOLE ? slot : find_last(a.n_trees, slot, base);
        slot0 = a.shift == REC_WHOLE ? slot : __builtin_amdgcn_readfirstlane(base(tree));
        tree_range(a.off, tree, a.n_rows, &lo, &hi);
        const long long n = hi - lo, size = 1ll << a.shift;
        parts = max((int)((n + size - 1) >> a.shift), 1);
        part = slot - slot0;
        there = part >= 0 && part < parts;
        if (!there) part = 0;
        first = (int)min(lo + part * size, (long long)hi);
        end = (int)min(first + size, (long long)hi);
    }
};

// R words from `row` on (as far as `end`; beyond it the last one again) of one tensor.
template <typename T, int V, int R> struct RecRows {
    RecRaw<T, V> r[R];
    __device__ void load(const void *p, long long stride, const RecLane<V> &l, int row, int end)
    {
        const T *at = static_cast<const T *>(p) + l.base;
#pragma unroll
        for (int k = 0; k < R; ++k) r[k] = *reinterpret_cast<const RecRaw<T, V> *>(at + min(row + k, end - 1) * stride);
    }
    __device__ float get(int k, int j) const { return (float)r[k].v[j]; }
};

// ---- pairs of parts ----------------------------------------------------------------------------

// A part's waves take an even share of its words each, one after the other.
template <typename T, int V, int W, int R, int GATE, bool BACK> __global__ __launch_bounds__(64 * W) void k_recur_pairs(RecurArgs a)
{
    __shared__ float lds[W][2][V][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int slot = blockIdx.x / a.slices, slice = blockIdx.x - slot * a.slices;
    const RecPart p(a, slot);
    if (!p.there || p.parts == 1) return;
    const RecLane<V> l(slice, lane, a.C);
    float *const out = a.pairs + 2ll * slot * a.C;
    if (!BACK && p.part == p.parts - 1) {
        float s[V] = {};
        if (wave == 0 && a.h0) l.load(a.h0 + (long long)p.tree * a.C, s);
        if (wave == 0) l.store(out, s);
        return;
    }
    if (BACK && p.part == 0) return;
    const int share = (1 << a.shift) / W;
    const int from = min(p.first + wave * share, p.end), to = min(from + share, p.end);
    float A[V], B[V];
#pragma unroll
    for (int j = 0; j < V; ++j) A[j] = 1.f, B[j] = 0.f;
    const void *const second = BACK ? a.d_h : a.x;
    const long long second_row = BACK ? a.d_h_row : a.x_row;
    RecRows<T, V, R> g, u;
    // (backwards: words are taken from the last run of R on)
    const int runs = (to - from + R - 1) / R;
    auto at = [&](int n) { return from + (BACK ? runs - 1 - n : n) * R; };
    if (runs > 0) {
        g.load(a.g, a.g_row, l, at(0), to);
        if (second) u.load(second, second_row, l, at(0), to);
    }
    for (int n = 0; n < runs; ++n) {
        const RecRows<T, V, R> G = g, U = u;
        if (n + 1 < runs) {
            g.load(a.g, a.g_row, l, at(n + 1), to);
            if (second) u.load(second, second_row, l, at(n + 1), to);
        }
        const int row = at(n);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int k = BACK ? R - 1 - q : q;
            if (row + k < to) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, i;
                    rec_gates<GATE>(G.get(k, j), f, i);
                    A[j] *= f;
                    B[j] = BACK ? f * (B[j] + (second ? U.get(k, j) : 0.f)) : fmaf(f, B[j], i * U.get(k, j));
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) lds[wave][0][j][lane] = A[j], lds[wave][1][j][lane] = B[j];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int j = 0; j < V; ++j) A[j] = 1.f, B[j] = 0.f;
    for (int q = 0; q < W; ++q) {
        const int w = BACK ? W - 1 - q : q;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float c = lds[w][0][j][lane];
            A[j] *= c;
            B[j] = fmaf(c, B[j], lds[w][1][j][lane]);
        }
    }
    l.store(out, A);
    l.store(out + a.C, B);
}

// The state at the start of a part, or (BACK) what comes back to its last word: pairs of the parts in between, joined one by one.
template <typename T, int GATE, int V, bool BACK> __device__ inline void rec_enter(const RecurArgs &a, const RecPart &p, const RecLane<V> &l, float (&s)[V])
{
    const float *const from = BACK ? a.d_last : a.h0;
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    if (!BACK && p.parts > 1) {
        l.load(a.pairs + 2ll * (p.slot0 + p.parts - 1) * a.C, s);
    } else if (from) {
        l.load(from + (long long)p.tree * a.C, s);
    }
    const int size = 1 << (a.shift & 31);
    const int many = BACK ? p.parts - 1 - p.part : p.part;
    for (int n = 0; n < many; ++n) {
        const int k = BACK ? p.parts - 1 - n : n;
        const float *const at = a.pairs + 2ll * (p.slot0 + k) * a.C;
        float A[V], B[V];
        l.load(at, A);
        l.load(at + a.C, B);
        const int begin = p.lo + k * size;
        rec_join<T, GATE, V, BACK>(a, l, begin, (int)min((long long)begin + size, (long long)p.hi), A, B, s);
    }
}

// ---- forward -----------------------------------------------------------------------------------

template <typename T, int V, int W, int R, int GATE> __global__ __launch_bounds__(64 * W) void k_recur(RecurArgs a)
{
    static_assert(REC_TAPE % (W * R) == 0, "states of the tape lie at starts of blocks");
    __shared__ float lds[W > 1 ? 2 : 1][W][2][V][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int slot = blockIdx.x / a.slices, slice = blockIdx.x - slot * a.slices;
    const RecPart p(a, slot);
    if (!p.there) return;
    const RecLane<V> l(slice, lane, a.C);
    float c[V];
    rec_enter<T, GATE, V, false>(a, p, l, c);
    if (p.lo == p.hi) {                                         // no words
        if (a.h_last && wave == 0) l.store(a.h_last + (long long)p.tree * a.C, c);
        return;
    }
    RecRows<T, V, R> g, x;
    auto load = [&](int row) {
        if (row >= p.end) return;
        g.load(a.g, a.g_row, l, row, p.end);
        x.load(a.x, a.x_row, l, row, p.end);
    };
    load(p.first + wave * R);
    int buf = 0;
    for (int block = p.first; block < p.end; block += W * R, buf ^= 1) {
        const int row = block + wave * R;
        float f[R][V], u[R][V], s[V];
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float i;
                rec_gates<GATE>(g.get(k, j), f[k][j], i);
                u[k][j] = i * x.get(k, j);
                if (row + k >= p.end) f[k][j] = 1.f, u[k][j] = 0.f;         // leaves a state as it is
            }
        if (block + W * R < p.end) load(row + W * R);
        if (a.tape && wave == 0 && ((block - p.lo) & (REC_TAPE - 1)) == 0)
            l.store(a.tape + (((long long)p.lo / REC_TAPE) + p.tree + (block - p.lo) / REC_TAPE) * a.C, c);
        if constexpr (W > 1) {
            float A[V], B[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                A[j] = 1.f, B[j] = 0.f;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    A[j] *= f[k][j];
                    B[j] = fmaf(f[k][j], B[j], u[k][j]);
                }
                lds[buf][wave][0][j][lane] = A[j];
                lds[buf][wave][1][j][lane] = B[j];
            }
            __syncthreads();                                    // (the other buffer is written only after the next one)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w == wave)
#pragma unroll
                    for (int j = 0; j < V; ++j) s[j] = c[j];
                const int begin = block + w * R;
                if (begin >= p.end) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) A[j] = lds[buf][w][0][j][lane], B[j] = lds[buf][w][1][j][lane];
                rec_join<T, GATE, V, false>(a, l, begin, min(begin + R, p.end), A, B, c);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = c[j];
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = fmaf(f[k][j], s[j], u[k][j]);
            if (row + k < p.end) {
                l.store(static_cast<T *>(a.h) + (row + k) * a.h_row, s);
                if (a.h_last && row + k == p.hi - 1) l.store(a.h_last + (long long)p.tree * a.C, s);
            }
        }
        if constexpr (W == 1)
#pragma unroll
            for (int j = 0; j < V; ++j) c[j] = s[j];
    }
}

// ---- gradients -----------------------------------------------------------------------------------

template <typename T, int V, int W, int R, int GATE> __global__ __launch_bounds__(64 * W) void k_recur_back(RecurArgs a)
{
    static_assert(REC_TAPE == W * R, "a block starts from a state of the tape");
    __shared__ float lds[2][W][3][V][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int slot = blockIdx.x / a.slices, slice = blockIdx.x - slot * a.slices;
    const RecLane<V> l(slice, lane, a.C);
    {   // rows behind the last sentence
        const int tail = min(max(__builtin_amdgcn_readfirstlane(a.off[a.n_trees]), 0), a.n_rows);
        const float none[V] = {};
        for (long long r = tail + slot + (long long)wave * a.slots; r < a.n_rows; r += (long long)W * a.slots) {
            l.store(static_cast<T *>(a.d_g) + r * a.d_g_row, none);
            l.store(static_cast<T *>(a.d_x) + r * a.d_x_row, none);
        }
    }
    const RecPart p(a, slot);
    if (!p.there) return;
    float c[V];
    rec_enter<T, GATE, V, true>(a, p, l, c);
    if (p.lo == p.hi) {
        if (a.d_h0 && wave == 0) l.store(a.d_h0 + (long long)p.tree * a.C, c);
        return;
    }
    RecRows<T, V, R> g, x, d;
    float s0[V];
    auto load = [&](int block) {
        const int row = block + wave * R;
        l.load(a.tape + (((long long)p.lo / REC_TAPE) + p.tree + (block - p.lo) / REC_TAPE) * a.C, s0);
        if (row >= p.end) return;
        g.load(a.g, a.g_row, l, row, p.end);
        x.load(a.x, a.x_row, l, row, p.end);
        if (a.d_h) d.load(a.d_h, a.d_h_row, l, row, p.end);
    };
    const int blocks = (p.end - p.first + W * R - 1) / (W * R);
    load(p.first + (blocks - 1) * (W * R));
    int buf = 0;
    for (int n = blocks - 1; n >= 0; --n, buf ^= 1) {
        const int block = p.first + n * (W * R), row = block + wave * R;
        float f[R][V], i[R][V], q[R][V], e[R][V], s[V], m[V];
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = s0[j];
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                rec_gates<GATE>(g.get(k, j), f[k][j], i[k][j]);
                q[k][j] = x.get(k, j);
                e[k][j] = a.d_h ? d.get(k, j) : 0.f;
                if (row + k >= p.end) f[k][j] = 1.f, i[k][j] = q[k][j] = e[k][j] = 0.f;
            }
        if (n > 0) load(block - W * R);
        {
            float A[V], B[V], D[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                A[j] = 1.f, B[j] = D[j] = 0.f;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    A[j] *= f[k][j];
                    B[j] = fmaf(f[k][j], B[j], i[k][j] * q[k][j]);
                }
#pragma unroll
                for (int k = R - 1; k >= 0; --k) D[j] = f[k][j] * (D[j] + e[k][j]);
                lds[buf][wave][0][j][lane] = A[j];
                lds[buf][wave][1][j][lane] = B[j];
                lds[buf][wave][2][j][lane] = D[j];
            }
            __syncthreads();
            for (int w = 0; w < wave; ++w) {
                const int begin = block + w * R;
#pragma unroll
                for (int j = 0; j < V; ++j) A[j] = lds[buf][w][0][j][lane], B[j] = lds[buf][w][1][j][lane];
                if (begin < p.end) rec_join<T, GATE, V, false>(a, l, begin, min(begin + R, p.end), A, B, s);
            }
#pragma unroll
            for (int w = W - 1; w >= 0; --w) {
                if (w == wave)
#pragma unroll
                    for (int j = 0; j < V; ++j) m[j] = c[j];
                const int begin = block + w * R;
                if (begin >= p.end) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) A[j] = lds[buf][w][0][j][lane], D[j] = lds[buf][w][2][j][lane];
                rec_join<T, GATE, V, true>(a, l, begin, min(begin + R, p.end), A, D, c);
            }
        }
        // forwards: what a word's own lambda is multiplied by in the gradient of its gate
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float before = s[j];
                s[j] = fmaf(f[k][j], before, i[k][j] * q[k][j]);
                q[k][j] = GATE == TL_GATE_SIGMOID ? (before - q[k][j]) * (f[k][j] * i[k][j]) : before;
            }
#pragma unroll
        for (int k = R - 1; k >= 0; --k) {
            float dg[V], dx[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float lambda = e[k][j] + m[j];
                dg[j] = lambda * q[k][j];
                dx[j] = lambda * i[k][j];
                m[j] = f[k][j] * lambda;
            }
            if (row + k < p.end) {
                l.store(static_cast<T *>(a.d_g) + (row + k) * a.d_g_row, dg);
                l.store(static_cast<T *>(a.d_x) + (row + k) * a.d_x_row, dx);
            }
        }
        if (a.d_h0 && wave == 0 && block == p.lo) l.store(a.d_h0 + (long long)p.tree * a.C, m);
    }
}

}  // namespace tl
