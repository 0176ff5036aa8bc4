// Cross attention of a decoder's queries to the node states of their trees, and its gradients.
//
//   s_ij = scale q_i . k_j  over the nodes j of i's tree that may be read,   P_ij = exp(s_ij - lse_i),   o_i = sum_j P_ij v_j
//   dV_j = sum_i P_ij dO_i,  dS_ij = P_ij (dO_i . v_j - dO_i . o_i),  dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i
//
// Batches are ragged: tree t owns rows q_off[t] .. q_off[t+1]-1 of the queries and kv_off[t] .. kv_off[t+1]-1 of the nodes.
// The G query heads that share a head of keys and values are rows of one product: packed row m of a tree is its query m / G,
// head m % G of the group, so that a node's row is read once for the whole group, and one query of G heads fills G rows of a tile.
//
// Every product runs on 32 x 32 tiles of the matrix unit: lane l holds column l % 32 of a result and, with half = l / 32, its
// rows 8 (r / 4) + 4 half + r % 4 in registers r = 0 .. 15.  The score tile is taken transposed (rows: nodes, columns: queries): a
// lane then owns one query, so that maxima, sums and scales are the lane's own numbers, and the registers that hold its
// probabilities are, as they stand, an operand of the product with the values: the operand's k-th element only has to be
// the same node on both sides, and the values are read from LDS in that order (16-bit types by the transposing LDS read).
//
// LDS rows are not padded: 16-byte granules are exchanged within 256 bytes by exclusive or with bits of the row, so that reads along a
// row by 16 lanes of 16 rows, reads down columns and the staging writes all spread over the 64 banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "treelstm.h"

namespace tl {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int ATT_THREADS = 256;
constexpr int ATT_WAVES = 4;

// A tensor of rows x heads x D; strides in elements, the last dimension contiguous.
struct AttTensor {
    void *p;
    long long row, head;
};

struct AttArgs {
    AttTensor q, k, v, o, d_o, d_q, d_k, d_v;
    const int32_t *q_off, *kv_off;
    const uint8_t *mask;
    float *lse;             // [n_q x n_heads], natural logarithm
    float *delta;           // backward: sum over d of d_o * o, [n_q x n_heads]
    float *part_o;          // splits > 1: outputs of each part, [splits][n_q x n_heads][D]
    float *part_lse;        // ... and their logarithms, [splits][n_q x n_heads]
    float scale, scale_log2;
    int n_trees, n_q, n_kv, Hq, Hk, G, D;
    int slots;              // row tiles (see find_slot)
    int splits;             // parts that a tree's nodes are cut into
    int vec;                // rows of q, k, v (and of what a backward pass reads) may be read in 16-byte pieces
    int vec_out;            // ... and the outputs written so
};

template <typename T> struct Elem;
template <> struct Elem<float> {
    typedef f32x4 frag;
};
template <> struct Elem<bf16_t> {
    typedef bf16x8 frag;
};
template <> struct Elem<f16_t> {
    typedef f16x8 frag;
};

// The last t in [0, n) with f(t) <= x, for an f that does not descend (0 where there is none).  All 64 lanes probe at once.
template <typename F> __device__ inline int find_last(int n, long long x, F f)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, len = n;
    for (;;) {
        const int step = (len + 63) >> 6;
        const bool in = lane * step < len;
        const unsigned long long le = __ballot(in && f(lo + (in ? lane * step : 0)) <= x);
        const int c = max((int)__popcll(le) - 1, 0);
        const int at = __builtin_amdgcn_readfirstlane(lo + c * step);
        if (step == 1) return at;
        len = min(step, lo + len - at);
        lo = at;
    }
}

// Which tree, and which of its tiles, slot `slot` stands for.  With n_t packed rows in tree t and tiles of 2^shift rows, slots
// mul off[t] / 2^shift + t .. are as many as tree t has tiles or one more: the host needs no lengths, and a slot beyond its
// tree's rows has nothing to do.  Offsets that do not ascend give a wrong tree, never one outside the batch.
__device__ inline int find_slot(const int32_t *__restrict__ off, int n, int mul, int shift, int slot, long long *tile)
{
    auto base = [&](int t) { return (((long long)off[t] * mul) >> shift) + t; };
    const int t = find_last(n, slot, base);
    *tile = slot - base(t);
    return t;
}

// Offsets as the batch should have them: kept inside the arrays whatever they hold.
__device__ inline void tree_range(const int32_t *__restrict__ off, int t, int n, int *lo, int *hi)
{
    const int a = __builtin_amdgcn_readfirstlane(off[t]), b = __builtin_amdgcn_readfirstlane(off[t + 1]);
    *lo = min(max(a, 0), n);
    *hi = min(max(b, *lo), n);
}

// Workgroups that read the same nodes follow one another in `logical`; the chip deals workgroups to its eight L2 domains in turn,
// so consecutive logical numbers are given to one domain.
__device__ inline long long xcd_order(long long id, long long n)
{
    const long long per = n >> 3, rest = n & 7, x = id & 7, y = id >> 3;
    return x * per + min(x, rest) + y;
}

// ---- LDS tiles --------------------------------------------------------------------------

template <typename T, int DP> struct Rows {
    static constexpr int EPG = 16 / (int)sizeof(T);      // elements of a granule
    static constexpr int GPR = DP / EPG;                 // granules of a row (a power of two)
    static constexpr int STEPS = GPR / 2;                // k-steps of a product over D: two granules, one per half of the wave
    static constexpr int BYTES = DP * (int)sizeof(T);

    __device__ static int turn(int r)
    {
        if constexpr (sizeof(T) == 2) {
            // column reads: rows r .. r+3 (r a multiple of 4), four granules from a multiple of four on
            if constexpr (GPR >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
            if constexpr (GPR == 8) return ((r & 2) << 1) | ((r >> 2) & 3);
            return (r >> 2) & 3;
        } else {
            // column reads: rows r and r+4, eight granules each
            if constexpr (GPR >= 16) return ((r & 4) << 1) | (r & 3) | ((r & 8) >> 1);
            return ((r & 4) << 1) | ((r & 2) >> 1) | ((r & 4) >> 1) | ((r & 8) >> 1);
        }
    }
    __device__ static int at(int r, int g) { return ((r * GPR + g) ^ turn(r)) << 4; }
};

// Operand of a product over D: row r of a tile, k-step s.
template <typename T, int DP> __device__ inline typename Elem<T>::frag row_frag(const unsigned char *tile, int r, int s, int half)
{
    return *reinterpret_cast<const typename Elem<T>::frag *>(tile + Rows<T, DP>::at(r, 2 * s + half));
}

__device__ inline void mma(floatx16 &c, f32x4 a, f32x4 b)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}
__device__ inline void mma(floatx16 &c, bf16x8 a, bf16x8 b) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline void mma(floatx16 &c, f16x8 a, f16x8 b) { c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

// Four rows of a 16-bit tile, row0 + 4 half .. + 3 of column d0 + l % 32 in lane l.
template <typename T, int DP> __device__ inline s16x4 column4(const unsigned char *tile, int row0, int d0, int lane)
{
    const int i = lane & 15;
    const int r = row0 + 4 * (lane >> 5) + (i >> 2);
    const int g = d0 / 8 + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    const unsigned char *p = tile + Rows<T, DP>::at(r, g) + 8 * (i & 1);
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
}

// c[t] += sum over 32 rows of tile^T (columns d_first + 32 t ..) times w, whose register r belongs to row row0 + 8 (r / 4) + 4 half + r % 4.
// 16-bit types: w is rounded to the type, as an operand of the matrix unit has to be (relative 2^-9 or 2^-12 of a probability or of a
// score's gradient, the size of the inputs' own roundings); sums stay in fp32.
template <typename T, int DP, int NT> __device__ inline void mma_columns(floatx16 (&c)[NT], const unsigned char *tile, int row0, const floatx16 &w,
                                                                         int d_first, int lane)
{
    if constexpr (sizeof(T) == 2) {
        typedef typename Elem<T>::frag frag;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            frag b;
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = (T)w[8 * s + j];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const s16x4 lo = column4<T, DP>(tile, row0 + 16 * s, d_first + 32 * t, lane);
                const s16x4 hi = column4<T, DP>(tile, row0 + 16 * s + 8, d_first + 32 * t, lane);
                frag a = __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                mma(c[t], a, b);
            }
        }
    } else {
        const int half = lane >> 5, col = d_first + (lane & 31);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = row0 + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int d = col + 32 * t;
                const float a = *reinterpret_cast<const float *>(tile + Rows<T, DP>::at(row, d >> 2) + 4 * (d & 3));
                c[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w[r], c[t], 0, 0, 0);
            }
        }
    }
}

// ---- global memory ----------------------------------------------------------------------

// Granule g of a row of D elements (zeros beyond D).
template <typename T> __device__ inline u32x4 load_granule(const T *__restrict__ row, int g, int D, bool vec)
{
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 x = {0u, 0u, 0u, 0u};
    const int d = g * E;
    if (vec) {
        if (d < D) x = *reinterpret_cast<const u32x4 *>(row + d);
    } else {
        T e[E];
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = d + j < D ? row[d + j] : (T)0.f;
        __builtin_memcpy(&x, e, 16);
    }
    return x;
}

// Four consecutive elements from d on.
template <typename T> __device__ inline void store4(T *__restrict__ row, int d, int D, bool vec, float a, float b, float c, float e)
{
    T x[4] = {(T)a, (T)b, (T)c, (T)e};
    if (vec) {
        if (d < D) __builtin_memcpy(__builtin_assume_aligned(row + d, 4 * sizeof(T)), x, 4 * sizeof(T));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) row[d + j] = x[j];
    }
}

template <typename T> __device__ inline T *row_of(const AttTensor &a, long long row, int head)
{
    return static_cast<T *>(a.p) + row * a.row + (long long)head * a.head;
}

__device__ inline float other_half(float x)
{
    return __shfl_xor(x, 32);
}

// ---- staging of node rows -----------------------------------------------------------------

// A workgroup's share of a tile of N node rows of K and of V: requested into registers (request), put into LDS later (put).  Rows
// that may not be read become zeros where a product would sum over them (zero_k, zero_v): whatever they hold, a NaN among it, times a
// probability of zero must not reach a sum.  Rows beyond the tree are read from its last row.
template <typename T, int DP, int N> struct NodeTile {
    typedef Rows<T, DP> R;
    static constexpr int GRANULES = N * R::GPR;
    static constexpr int EACH = (GRANULES + ATT_THREADS - 1) / ATT_THREADS;
    u32x4 k[EACH], v[EACH];
    unsigned live;

    __device__ void request(const T *__restrict__ kp, const T *__restrict__ vp, const AttArgs &a, int first, int lo, int hi)
    {
        live = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = threadIdx.x + i * ATT_THREADS;
            if (GRANULES % ATT_THREADS == 0 || e < GRANULES) {
                const int r = e / R::GPR, g = e % R::GPR;
                const int node = min(first + r, hi - 1);
                const bool in = first + r < hi && (!a.mask || a.mask[node] != 0);
                live |= in ? 1u << i : 0u;
                k[i] = load_granule<T>(kp + (long long)node * a.k.row, g, a.D, a.vec);
                v[i] = load_granule<T>(vp + (long long)node * a.v.row, g, a.D, a.vec);
            }
        }
    }
    template <bool ZERO_K, bool ZERO_V> __device__ void put(unsigned char *kt, unsigned char *vt)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = threadIdx.x + i * ATT_THREADS;
            if (GRANULES % ATT_THREADS == 0 || e < GRANULES) {
                const int at = R::at(e / R::GPR, e % R::GPR);
                const bool in = live >> i & 1;
                const u32x4 zero = {0u, 0u, 0u, 0u};
                *reinterpret_cast<u32x4 *>(kt + at) = ZERO_K && !in ? zero : k[i];
                *reinterpret_cast<u32x4 *>(vt + at) = ZERO_V && !in ? zero : v[i];
            }
        }
    }
};

// Which of 64 nodes from `first` on may be read (the same word in every lane).
__device__ inline unsigned long long live_nodes(const AttArgs &a, int first, int hi)
{
    const int node = first + (threadIdx.x & 63);
    return __ballot(node < hi && (!a.mask || a.mask[min(node, hi - 1)] != 0));
}

// ---- forward ------------------------------------------------------------------------------

// WM waves side by side along the rows (32 packed rows each), WK waves along the nodes; NT node tiles of 32 per wave and stage.
// Rows of trees with many queries: WM = 4, every wave reads all nodes of a stage.  Few queries (a single token): WM = 1, the four waves
// share one tile of rows, each takes a quarter of the nodes, and their sums are joined at the end.
template <typename T, int DP, int WM> struct AttFwd {
    static constexpr int WK = ATT_WAVES / WM;
    static constexpr int NT = WM > 1 && DP * (int)sizeof(T) <= 256 ? 2 : 1;
    static constexpr int BM = 32 * WM;
    static constexpr int BN = 32 * WK * NT;
    static constexpr int STAGE = 2 * BN * Rows<T, DP>::BYTES;
    static constexpr int BUFS = STAGE <= 32768 ? 2 : 1;
    static constexpr int JOIN = WK > 1 ? WK * 32 * (DP + 4) * 4 + WK * 64 * 4 : 0;
    static constexpr int LDS = STAGE * BUFS > JOIN ? STAGE * BUFS : JOIN;
    static constexpr int MIN_BLOCKS = DP * (int)sizeof(T) > 256 ? 1 : 2;
};

template <typename T, int DP, int WM>
__global__ __launch_bounds__(ATT_THREADS, (AttFwd<T, DP, WM>::MIN_BLOCKS)) void k_attend(const AttArgs a)
{
    typedef AttFwd<T, DP, WM> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int WK = C::WK, NT = C::NT, DT = DP / 32;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wk = wave / WM;
    const long long id = xcd_order(blockIdx.x, gridDim.x);
    const int slot = (int)(id % a.slots), part = (int)(id / a.slots % a.splits), hk = (int)(id / a.slots / a.splits);
    long long tile;
    const int tree = find_slot(a.q_off, a.n_trees, a.G, C::BM == 32 ? 5 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G, m0 = tile * C::BM;
    if (tile < 0 || m0 >= n_rows) return;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    const int n_stage = (hi - lo + C::BN - 1) / C::BN;
    int s_lo = 0, s_hi = n_stage;
    if (a.splits > 1) {
        const int per = (n_stage + a.splits - 1) / a.splits;
        s_lo = min(part * per, n_stage);
        s_hi = min(s_lo + per, n_stage);
        if (s_lo >= s_hi) return;
    }

    const long long m = m0 + 32 * wm + col;
    const bool mine = m < n_rows;
    const int qi = q_lo + (int)((mine ? m : m0) / a.G), head = hk * a.G + (int)((mine ? m : m0) % a.G);
    frag qf[R::STEPS];
    {
        const T *qr = row_of<T>(a.q, qi, head);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) qf[s] = __builtin_bit_cast(frag, load_granule<T>(qr, 2 * s + half, a.D, a.vec));
    }

    floatx16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = floatx16{};
    float top = -INFINITY, sum = 0.f;          // largest raw score so far (of the lane's query), sum of the lane's half of its nodes

    const T *kp = row_of<T>(a.k, 0, hk), *vp = row_of<T>(a.v, 0, hk);
    NodeTile<T, DP, C::BN> st;
    if (s_lo < s_hi) {
        st.request(kp, vp, a, lo + s_lo * C::BN, lo, hi);
        st.template put<false, true>(att_lds, att_lds + C::STAGE / 2);
    }
    for (int s = s_lo; s < s_hi; ++s) {
        const int first = lo + s * C::BN;
        const unsigned char *kt = att_lds + (C::BUFS == 2 ? ((s - s_lo) & 1) * C::STAGE : 0), *vt = kt + C::STAGE / 2;
        __syncthreads();
        if (s + 1 < s_hi) st.request(kp, vp, a, first + C::BN, lo, hi);
        const int w_first = first + 32 * NT * wk;
        const unsigned long long live = live_nodes(a, w_first, hi);
        if (w_first < hi) {
            floatx16 p[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                p[t] = floatx16{};
#pragma unroll
                for (int d = 0; d < R::STEPS; ++d) mma(p[t], row_frag<T, DP>(kt, 32 * (NT * wk + t) + col, d, half), qf[d]);
            }
            const unsigned long long all = NT == 2 ? ~0ull : 0xffffffffull;
            if ((live & all) != all) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const unsigned w = (unsigned)(live >> (32 * t)) >> (4 * half);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!(w >> (8 * (r >> 2) + (r & 3)) & 1)) p[t][r] = -INFINITY;
                }
            }
            float high = top;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) high = fmaxf(high, p[t][r]);
            high = fmaxf(high, other_half(high));
            const float ref = high == -INFINITY ? 0.f : high * a.scale_log2;
            if (__any(high > top)) {
                const float f = __builtin_amdgcn_exp2f(top == high ? 0.f : top * a.scale_log2 - ref);
                sum *= f;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[t][r] *= f;
                top = high;
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[t][r] = __builtin_amdgcn_exp2f(fmaf(p[t][r], a.scale_log2, -ref));
                    sum += p[t][r];
                }
                mma_columns<T, DP, DT>(acc, vt, 32 * (NT * wk + t), p[t], 0, lane);
            }
        }
        if (C::BUFS == 1) __syncthreads();
        if (s + 1 < s_hi) {
            unsigned char *nk = att_lds + (C::BUFS == 2 ? ((s + 1 - s_lo) & 1) * C::STAGE : 0);
            st.template put<false, true>(nk, nk + C::STAGE / 2);
        }
    }
    sum += other_half(sum);

    const long long row_head = (long long)qi * a.Hq + head;
    const bool partial = a.splits > 1;
    if constexpr (WK == 1) {
        if (!mine) return;
        const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
        const float lse = sum > 0.f || sum != sum ? (top * a.scale_log2 + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
        if (half == 0) {
            if (partial) a.part_lse[(long long)part * a.n_q * a.Hq + row_head] = lse;
            else if (a.lse) a.lse[row_head] = lse;
        }
        float *po = partial ? a.part_o + ((long long)part * a.n_q * a.Hq + row_head) * a.D : nullptr;
        T *o = row_of<T>(a.o, qi, head);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d = 32 * t + 2 * r + 4 * half;
                if (partial) store4<float>(po, d, a.D, (a.D & 3) == 0, acc[t][r] * inv, acc[t][r + 1] * inv, acc[t][r + 2] * inv, acc[t][r + 3] * inv);
                else store4<T>(o, d, a.D, a.vec_out, acc[t][r] * inv, acc[t][r + 1] * inv, acc[t][r + 2] * inv, acc[t][r + 3] * inv);
            }
    } else {
        // the waves' sums over their nodes, brought to one maximum
        float *jo = reinterpret_cast<float *>(att_lds), *jt = jo + WK * 32 * (DP + 4), *js = jt + WK * 32;
        __syncthreads();
        if (half == 0) {
            jt[wk * 32 + col] = top;
            js[wk * 32 + col] = sum;
        }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4 *>(jo + (wk * 32 + col) * (DP + 4) + 32 * t + 2 * r + 4 * half) =
                    f32x4{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
        __syncthreads();
        constexpr int G4 = DP / 4;
        const int n_here = (int)min((long long)32, n_rows - m0);
        for (int e = threadIdx.x; e < n_here * G4; e += ATT_THREADS) {
            const int r = e / G4, d = 4 * (e % G4);
            float tt = -INFINITY;
#pragma unroll
            for (int w = 0; w < WK; ++w) tt = fmaxf(tt, jt[w * 32 + r]);
            float total = 0.f;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float tw = jt[w * 32 + r];
                const float f = tw == tt ? 1.f : __builtin_amdgcn_exp2f((tw - tt) * a.scale_log2);
                total += f * js[w * 32 + r];
                const f32x4 y = *reinterpret_cast<const f32x4 *>(jo + (w * 32 + r) * (DP + 4) + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += f * y[j];
            }
            const bool any = total > 0.f || total != total;
            const float inv = any ? 1.f / total : 0.f;
            const int i = q_lo + (int)((m0 + r) / a.G), hd = hk * a.G + (int)((m0 + r) % a.G);
            const long long rh = (long long)i * a.Hq + hd;
            if (d == 0) {
                const float lse = any ? (tt * a.scale_log2 + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
                if (partial) a.part_lse[(long long)part * a.n_q * a.Hq + rh] = lse;
                else if (a.lse) a.lse[rh] = lse;
            }
            if (partial)
                store4<float>(a.part_o + ((long long)part * a.n_q * a.Hq + rh) * a.D, d, a.D, (a.D & 3) == 0, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            else
                store4<T>(row_of<T>(a.o, i, hd), d, a.D, a.vec_out, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
        }
    }
}

// Joins the parts of a split forward: one wave per query and head.  BN: nodes per stage of the kernel that made them.
template <typename T> __global__ __launch_bounds__(ATT_THREADS) void k_attend_join(const AttArgs a, int bn)
{
    const int lane = threadIdx.x & 63;
    const long long rh = (long long)blockIdx.x * ATT_WAVES + (threadIdx.x >> 6), n = (long long)a.n_q * a.Hq;
    if (rh >= n) return;
    const int qi = (int)(rh / a.Hq), head = (int)(rh % a.Hq);
    int lo, hi;
    const int tree = find_last(a.n_trees, qi, [&](int t) { return (long long)a.q_off[t]; });
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    const int n_stage = (hi - lo + bn - 1) / bn, per = (n_stage + a.splits - 1) / a.splits;
    const int parts = per ? (n_stage + per - 1) / per : 0;
    float top = -INFINITY;
    for (int j = lane; j < parts; j += 64) top = fmaxf(top, a.part_lse[j * n + rh]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    float total = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < parts; ++j) {
        const float l = a.part_lse[j * n + rh];
        const float f = l == -INFINITY ? 0.f : __expf(l - top);
        total += f;
        const float *po = a.part_o + (j * n + rh) * a.D;
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (lane + 64 * t < a.D) x[t] += f * po[lane + 64 * t];
    }
    const bool any = total > 0.f || total != total;
    const float inv = any ? 1.f / total : 0.f;
    T *o = row_of<T>(a.o, qi, head);
#pragma unroll
    for (int t = 0; t < 4; ++t)
        if (lane + 64 * t < a.D) o[lane + 64 * t] = (T)(x[t] * inv);
    if (a.lse && lane == 0) a.lse[rh] = any ? top + __logf(total) : -INFINITY;
}

// ---- backward -----------------------------------------------------------------------------

// delta[i] = d_o[i] . o[i]: 16 lanes per query and head.
template <typename T> __global__ __launch_bounds__(ATT_THREADS) void k_attend_delta(const AttArgs a)
{
    const int l16 = threadIdx.x & 15;
    const long long rh = ((long long)blockIdx.x * ATT_THREADS + threadIdx.x) >> 4, n = (long long)a.n_q * a.Hq;
    float x = 0.f;
    if (rh < n) {
        const int qi = (int)(rh / a.Hq), head = (int)(rh % a.Hq);
        const T *o = row_of<T>(a.o, qi, head), *g = row_of<T>(a.d_o, qi, head);
        constexpr int E = 16 / (int)sizeof(T);
        for (int c = l16; c * E < a.D; c += 16) {
            T y[E], z[E];
            const u32x4 yo = load_granule<T>(o, c, a.D, a.vec), zo = load_granule<T>(g, c, a.D, a.vec);
            __builtin_memcpy(y, &yo, 16);
            __builtin_memcpy(z, &zo, 16);
#pragma unroll
            for (int j = 0; j < E; ++j) x = fmaf((float)y[j], (float)z[j], x);
        }
    }
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    if (rh < n && l16 == 0) a.delta[rh] = x;
}

// What exp2 subtracts: a row without nodes (lse = -inf) has no probabilities.
__device__ inline float lse_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// dQ: like the forward, rows (queries) on the lanes' columns.  Waves side by side along the rows (WM) and, for wide heads, along the
// columns of dQ (WD), where every wave of a row tile works out the tile's scores itself.
template <typename T, int DP> struct AttDq {
    static constexpr int WD = DP > 128 ? 2 : 1;
    static constexpr int WM = ATT_WAVES / WD;
    static constexpr int BM = 32 * WM;
    static constexpr int BN = 32;
    static constexpr int DT = DP / 32 / WD;
    static constexpr int STAGE = 2 * BN * Rows<T, DP>::BYTES;
    static constexpr int BUFS = 2;
    static constexpr int LDS = STAGE * BUFS;
    static constexpr int MIN_BLOCKS = DP * (int)sizeof(T) > 256 ? 1 : 2;
};

template <typename T, int DP>
__global__ __launch_bounds__(ATT_THREADS, (AttDq<T, DP>::MIN_BLOCKS)) void k_attend_dq(const AttArgs a)
{
    typedef AttDq<T, DP> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int DT = C::DT;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / C::WD, wd = wave % C::WD;
    const long long id = xcd_order(blockIdx.x, gridDim.x);
    const int slot = (int)(id % a.slots), hk = (int)(id / a.slots);
    long long tile;
    const int tree = find_slot(a.q_off, a.n_trees, a.G, C::BM == 64 ? 6 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G, m0 = tile * C::BM;
    if (tile < 0 || m0 >= n_rows) return;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    const int n_stage = (hi - lo + C::BN - 1) / C::BN;

    const long long m = m0 + 32 * wm + col;
    const bool mine = m < n_rows;
    const int qi = q_lo + (int)((mine ? m : m0) / a.G), head = hk * a.G + (int)((mine ? m : m0) % a.G);
    const long long row_head = (long long)qi * a.Hq + head;
    frag qf[R::STEPS], gf[R::STEPS];
    {
        const T *qr = row_of<T>(a.q, qi, head), *gr = row_of<T>(a.d_o, qi, head);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) {
            qf[s] = __builtin_bit_cast(frag, load_granule<T>(qr, 2 * s + half, a.D, a.vec));
            gf[s] = __builtin_bit_cast(frag, load_granule<T>(gr, 2 * s + half, a.D, a.vec));
        }
    }
    const float ref = lse_log2(a.lse[row_head]), delta = a.delta[row_head];
    floatx16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = floatx16{};

    const T *kp = row_of<T>(a.k, 0, hk), *vp = row_of<T>(a.v, 0, hk);
    NodeTile<T, DP, C::BN> st;
    if (n_stage) {
        st.request(kp, vp, a, lo, lo, hi);
        st.template put<true, false>(att_lds, att_lds + C::STAGE / 2);
    }
    for (int s = 0; s < n_stage; ++s) {
        const int first = lo + s * C::BN;
        const unsigned char *kt = att_lds + (s & 1) * C::STAGE, *vt = kt + C::STAGE / 2;
        __syncthreads();
        if (s + 1 < n_stage) st.request(kp, vp, a, first + C::BN, lo, hi);
        const unsigned w = (unsigned)live_nodes(a, first, hi) >> (4 * half);
        floatx16 p = floatx16{}, dp = floatx16{};
#pragma unroll
        for (int d = 0; d < R::STEPS; ++d) {
            mma(p, row_frag<T, DP>(kt, col, d, half), qf[d]);
            mma(dp, row_frag<T, DP>(vt, col, d, half), gf[d]);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(p[r], a.scale_log2, -ref)) * (dp[r] - delta);
            p[r] = w >> (8 * (r >> 2) + (r & 3)) & 1 ? e : 0.f;
        }
        mma_columns<T, DP, DT>(acc, kt, 0, p, 32 * DT * wd, lane);
        if (s + 1 < n_stage) {
            unsigned char *nk = att_lds + ((s + 1) & 1) * C::STAGE;
            st.template put<true, false>(nk, nk + C::STAGE / 2);
        }
    }
    if (!mine) return;
    T *o = row_of<T>(a.d_q, qi, head);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            store4<T>(o, 32 * (DT * wd + t) + 2 * r + 4 * half, a.D, a.vec_out, acc[t][r] * a.scale, acc[t][r + 1] * a.scale, acc[t][r + 2] * a.scale,
                      acc[t][r + 3] * a.scale);
}

// dK and dV: nodes on the lanes' columns, packed query rows go by in LDS.  Every sum over queries and over the heads of a group is
// taken by one wave in one order: no atomics, the same bits every run.
template <typename T, int DP> struct AttDkv {
    static constexpr int WD = DP > 128 ? 2 : 1;
    static constexpr int WN = ATT_WAVES / WD;
    static constexpr int BN = 32 * WN;
    static constexpr int BQ = 32;
    static constexpr int DT = DP / 32 / WD;
    static constexpr int STAGE = 2 * BQ * Rows<T, DP>::BYTES + 2 * BQ * 4;
    static constexpr int LDS = 2 * STAGE;
    static constexpr int MIN_BLOCKS = DP * (int)sizeof(T) > 128 ? 1 : 2;
};

template <typename T, int DP>
__global__ __launch_bounds__(ATT_THREADS, (AttDkv<T, DP>::MIN_BLOCKS)) void k_attend_dkv(const AttArgs a)
{
    typedef AttDkv<T, DP> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int DT = C::DT, BQ = C::BQ;
    constexpr int GRANULES = BQ * R::GPR, EACH = (GRANULES + ATT_THREADS - 1) / ATT_THREADS;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = wave / C::WD, wd = wave % C::WD;
    const long long id = xcd_order(blockIdx.x, gridDim.x);
    const int slot = (int)(id % a.slots), hk = (int)(id / a.slots);
    long long tile;
    const int tree = find_slot(a.kv_off, a.n_trees, 1, C::BN == 64 ? 6 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    const long long n0 = lo + tile * C::BN;
    if (tile < 0 || n0 >= hi) return;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G;

    const long long node = n0 + 32 * wn + col;
    const bool mine = node < hi;
    const long long node_in = mine ? node : n0;
    const bool live = mine && (!a.mask || a.mask[node_in] != 0);
    frag kf[R::STEPS], vf[R::STEPS];
    {
        const T *kr = row_of<T>(a.k, node_in, hk), *vr = row_of<T>(a.v, node_in, hk);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) {
            kf[s] = __builtin_bit_cast(frag, load_granule<T>(kr, 2 * s + half, a.D, a.vec));
            vf[s] = __builtin_bit_cast(frag, load_granule<T>(vr, 2 * s + half, a.D, a.vec));
        }
    }
    floatx16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dk[t] = dv[t] = floatx16{};

    u32x4 rq[EACH], rg[EACH];
    float r_ref = 0.f, r_delta = 0.f;
    auto request = [&](long long first) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = threadIdx.x + i * ATT_THREADS;
            rq[i] = rg[i] = u32x4{0u, 0u, 0u, 0u};
            if (GRANULES % ATT_THREADS == 0 || e < GRANULES) {
                const long long m = first + e / R::GPR;
                if (m < n_rows) {
                    const int qi = q_lo + (int)(m / a.G), head = hk * a.G + (int)(m % a.G);
                    rq[i] = load_granule<T>(row_of<T>(a.q, qi, head), e % R::GPR, a.D, a.vec);
                    rg[i] = load_granule<T>(row_of<T>(a.d_o, qi, head), e % R::GPR, a.D, a.vec);
                }
            }
        }
        if (threadIdx.x < BQ) {
            const long long m = first + threadIdx.x;
            r_ref = INFINITY;
            r_delta = 0.f;
            if (m < n_rows) {
                const long long rh = (q_lo + m / a.G) * a.Hq + hk * a.G + m % a.G;
                r_ref = lse_log2(a.lse[rh]);
                r_delta = a.delta[rh];
            }
        }
    };
    auto put = [&](unsigned char *b) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = threadIdx.x + i * ATT_THREADS;
            if (GRANULES % ATT_THREADS == 0 || e < GRANULES) {
                const int at = R::at(e / R::GPR, e % R::GPR);
                *reinterpret_cast<u32x4 *>(b + at) = rq[i];
                *reinterpret_cast<u32x4 *>(b + BQ * R::BYTES + at) = rg[i];
            }
        }
        if (threadIdx.x < BQ) {
            float *x = reinterpret_cast<float *>(b + 2 * BQ * R::BYTES);
            x[threadIdx.x] = r_ref;
            x[BQ + threadIdx.x] = r_delta;
        }
    };
    const int n_stage = (int)((n_rows + BQ - 1) / BQ);
    if (n_stage) {
        request(0);
        put(att_lds);
    }
    for (int s = 0; s < n_stage; ++s) {
        const unsigned char *qt = att_lds + (s & 1) * C::STAGE, *gt = qt + BQ * R::BYTES;
        const float *ref = reinterpret_cast<const float *>(gt + BQ * R::BYTES), *delta = ref + BQ;
        __syncthreads();
        if (s + 1 < n_stage) request((long long)(s + 1) * BQ);
        floatx16 p = floatx16{}, dp = floatx16{};
#pragma unroll
        for (int d = 0; d < R::STEPS; ++d) {
            mma(p, row_frag<T, DP>(qt, col, d, half), kf[d]);
            mma(dp, row_frag<T, DP>(gt, col, d, half), vf[d]);
        }
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 rr = *reinterpret_cast<const f32x4 *>(ref + 8 * r4 + 4 * half);
            const f32x4 dd = *reinterpret_cast<const f32x4 *>(delta + 8 * r4 + 4 * half);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 4 * r4 + j;
                const float e = __builtin_amdgcn_exp2f(fmaf(p[r], a.scale_log2, -rr[j]));
                p[r] = live ? e : 0.f;
                dp[r] = live ? e * (dp[r] - dd[j]) : 0.f;
            }
        }
        mma_columns<T, DP, DT>(dv, gt, 0, p, 32 * DT * wd, lane);
        mma_columns<T, DP, DT>(dk, qt, 0, dp, 32 * DT * wd, lane);
        if (s + 1 < n_stage) put(att_lds + ((s + 1) & 1) * C::STAGE);
    }
    if (!mine) return;
    T *ok = row_of<T>(a.d_k, node, hk), *ov = row_of<T>(a.d_v, node, hk);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * (DT * wd + t) + 2 * r + 4 * half;
            store4<T>(ok, d, a.D, a.vec_out, dk[t][r] * a.scale, dk[t][r + 1] * a.scale, dk[t][r + 2] * a.scale, dk[t][r + 3] * a.scale);
            store4<T>(ov, d, a.D, a.vec_out, dv[t][r], dv[t][r + 1], dv[t][r + 2], dv[t][r + 3]);
        }
}

}  // namespace tl
