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

#include <type_traits>

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
    float *delta, *ref;     // backward: sum over d of d_o * o, and lse in base 2 (less ATT_LIFT), [n_q x n_heads]
    float *size;            // backward, fp16: power of two that brings a row of d_o, lifted, to a length of 2^10, [n_q x n_heads]
    int32_t *list, *live;   // backward, with a mask: the nodes that may be read, tree by tree from kv_off on, and how many a tree has
    float *part_o;          // splits > 1: outputs of each part, [splits][n_q x n_heads][D]
    float *part_lse;        // ... and their logarithms, [splits][n_q x n_heads]
    float *part_q, *part_kv; // backward, splits > 1: parts of dQ [splits][n_q x n_heads][D], of dK and dV [splits][n_kv x n_kv_heads][2][D]
    float scale, scale_log2;
    int n_trees, n_q, n_kv, Hq, Hk, G, D;
    int slots;              // row tiles (see find_slot)
    int splits;             // parts that a tree's nodes are cut into
    int bufs;               // stages that LDS holds: 2, the next one arriving while one is worked on, or 1
    int kv_slots, kv_splits, kv_bufs, kv_blocks;    // backward: the same of the gradients of keys and values, and their workgroups
    int near;               // 128 rows of any input span less than 2^31 bytes
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
__device__ inline uint32_t xcd_order(uint32_t id, uint32_t n)
{
    const uint32_t per = n >> 3, rest = n & 7, x = id & 7, y = id >> 3;
    return x * per + min(x, rest) + y;
}

// (Division in 64 bits takes some hundred instructions.)
__device__ inline long long divide(long long a, int b) { return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }

// Query and head of the group of packed rows m0 + r for r below 256, all of it in 32 bits.  (x + 1/2) / G lies 1 / (2 G) or more from a
// whole number, and x < 4096 + 256: far more than rounding moves it.
struct Packed {
    int G, q0, first;
    float per;
    __device__ Packed(int q_lo, long long m0, int group) : G(group), per(__builtin_amdgcn_rcpf((float)group))
    {
        const long long k = divide(m0, G);
        q0 = q_lo + (int)k;
        first = (int)(m0 - k * G);
    }
    __device__ void at(int r, int *query, int *head) const
    {
        const int k = (int)(((float)(first + r) + 0.5f) * per);
        *query = q0 + k;
        *head = first + r - k * G;
    }
};

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

#define ATT_LDS __attribute__((address_space(3)))
__device__ inline uint32_t lds_address(const unsigned char *p) { return (uint32_t)(uintptr_t)(const ATT_LDS unsigned char *)p; }

// Operands of products over D: row r0 + l % 32 of a tile, k-step s.  at[s] is the lane's place for r0 = 0; further rows are a constant away (r0 a
// multiple of 16, after which the exchange repeats), so that a read is one instruction.
template <typename T, int DP> struct RowReads {
    typedef typename Elem<T>::frag frag;
    typedef Rows<T, DP> R;
    uint32_t at[R::STEPS];
    __device__ explicit RowReads(const unsigned char *tile)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) at[s] = lds_address(tile) + R::at(lane & 31, 2 * s + (lane >> 5));
    }
    __device__ void move(int bytes)
    {
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) at[s] += bytes;
    }
    __device__ frag get(int r0, int s) const { return *(const ATT_LDS frag *)(uintptr_t)(at[s] + r0 * R::BYTES); }
};

__device__ inline void mma(floatx16 &c, f32x4 a, f32x4 b)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}
__device__ inline void mma(floatx16 &c, bf16x8 a, bf16x8 b) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline void mma(floatx16 &c, f16x8 a, f16x8 b) { c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

typedef ATT_LDS s16x4 *lds_s16x4;

// Operands of products over the rows of a tile: its columns.  16-bit types: four rows r0 + 4 half .. + 3 (and those 8 further) of column
// d0 + l % 32 by the transposing read; fp32: one element of row r0 + 8 (r / 4) + 4 half + r % 4.
template <typename T, int DP> struct ColumnReads {
    typedef Rows<T, DP> R;
    static constexpr int KINDS = sizeof(T) == 2 ? 2 : 8;                        // rows whose exchange differs
    static constexpr int WIDE = sizeof(T) == 2 ? 4 : 2;                         // column tiles until the exchange repeats
    static constexpr int TILES = DP / 32 < WIDE ? DP / 32 : WIDE;
    uint32_t at[KINDS][TILES];
    __device__ explicit ColumnReads(const unsigned char *tile, int d_first)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int k = 0; k < KINDS; ++k)
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                if constexpr (sizeof(T) == 2) {
                    const int i = lane & 15;
                    const int r = 8 * k + 4 * half + (i >> 2), g = (d_first + 32 * t) / 8 + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
                    at[k][t] = lds_address(tile) + R::at(r, g) + 8 * (i & 1);
                } else {
                    const int r = 8 * (k >> 2) + 4 * half + (k & 3), d = d_first + 32 * t + (lane & 31);
                    at[k][t] = lds_address(tile) + R::at(r, d >> 2) + 4 * (d & 3);
                }
            }
    }
    __device__ void move(int bytes)
    {
#pragma unroll
        for (int k = 0; k < KINDS; ++k)
#pragma unroll
            for (int t = 0; t < TILES; ++t) at[k][t] += bytes;
    }
    // rows from r0 (a multiple of 16) on, column tile t
    __device__ uint32_t place(int k, int t, int r0) const { return at[k][t % WIDE] + (t / WIDE) * WIDE * 32 * (int)sizeof(T) + r0 * R::BYTES; }
    __device__ s16x4 four(int k, int t, int r0) const { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)place(k, t, r0)); }
    __device__ float one(int r, int t, int r0) const { return *(const ATT_LDS float *)(uintptr_t)place(r & 7, t, r0 + (r & 8) * 2); }
};

// c[t] += sum over the 32 rows from r0 on of tile^T (column tile t) times w, whose register r belongs to row r0 + 8 (r / 4) + 4 half + r % 4.
// 16-bit types: an operand of the matrix unit has to be of the type.  With TERMS = 1 w is rounded to it once, which adds to a result as much error
// as its own rounding to the type does; with TERMS = 2 what the rounding left is a second operand (16 bits of w together, in fp16 22).
// fp16 holds these bits only from 2^-14 (2^-3) on: probabilities and score gradients come scaled (ATT_LIFT, fit_fp16).  Sums stay in fp32.
template <typename T, int DP, int TERMS, int NT>
__device__ inline void mma_columns(floatx16 (&c)[NT], const ColumnReads<T, DP> &tile, int r0, const floatx16 &w)
{
    if constexpr (sizeof(T) == 2) {
        typedef typename Elem<T>::frag frag;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            frag b[TERMS];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                b[0][j] = (T)w[8 * s + j];
                if (TERMS == 2) b[TERMS - 1][j] = (T)(w[8 * s + j] - (float)b[0][j]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const frag a = __builtin_bit_cast(frag, __builtin_shufflevector(tile.four(0, t, r0 + 16 * s), tile.four(1, t, r0 + 16 * s), 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int q = TERMS - 1; q >= 0; --q) mma(c[t], a, b[q]);
            }
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile.one(r, t, r0), w[r], c[t], 0, 0, 0);
    }
}

// What lane l ^ 32 holds, joined with the lane's own.
__device__ inline float max_of_halves(float x)
{
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ inline float sum_of_halves(float x)
{
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// fp16 probabilities are operands times 2^14, and so are the sums until the end: of thousands of nodes most have less than fp16's least normal value, 2^-14,
// and below it steps no longer shrink.  So scaled, all bits of one term are there from 2^-28 on, of two from 2^-17.  They do not exceed 1, so
// that 2^14 is far from the type's largest value.  exp2 adds the 14 for nothing, in what it subtracts.
template <typename T> constexpr float ATT_LIFT = std::is_same<T, f16_t>::value ? 14.f : 0.f;
template <typename T> constexpr float ATT_LIFTED = std::is_same<T, f16_t>::value ? 16384.f : 1.f;

// fp16 score gradients on their way into a product: neither may a scaled loss overflow them nor a small one let them vanish.  A lane's column of the
// sums c carries a power of two, `size`, which is lowered (and the sums with it) when a gradient would come near the type's largest value.
template <int NT> __device__ inline void fit_fp16(floatx16 &w, float &size, floatx16 (&c)[NT])
{
    float high = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) high = fmaxf(high, fabsf(w[r]));
    high = max_of_halves(high) * size;
    if (__any(high > 32768.f)) {
        const float f = high > 32768.f ? exp2f(-ceilf(log2f(high * 0x1p-10f))) : 1.f;
        size *= f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) c[t][r] *= f;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] *= size;
}

// ---- global memory ----------------------------------------------------------------------

// (Pointers out of the argument struct are cast to global memory: through generic ones loads and LDS reads would wait for each other.)
#define ATT_GLOBAL __attribute__((address_space(1)))

typedef u32x4 u32x4_any __attribute__((aligned(2)));          // at any address of an element

// Granule g of a row of D elements that does not divide into granules: 16 bytes at any address, those of the last granule ending with the row;
// shifted into place, with zeros beyond D, by granule_in_place, which waits for the load.
template <typename T> __device__ inline u32x4 granule_anywhere(const T *row, int g, int D)
{
    constexpr int E = 16 / (int)sizeof(T);
    const ATT_GLOBAL T *p = (const ATT_GLOBAL T *)row;
    if (D >= E) return *(const ATT_GLOBAL u32x4_any *)(p + min(g * E, D - E));
    T e[E];
    u32x4 x;
#pragma unroll
    for (int j = 0; j < E; ++j) e[j] = p[min(j, D - 1)];
    __builtin_memcpy(&x, e, 16);
    return x;
}
template <typename T> __device__ inline u32x4 granule_in_place(u32x4 x, int g, int D)
{
    constexpr int E = 16 / (int)sizeof(T), BITS = 8 * (int)sizeof(T);
    uint64_t lo = (uint64_t)x[1] << 32 | x[0], hi = (uint64_t)x[3] << 32 | x[2];
    if (D >= E) {
        const int bits = BITS * max(g * E - (D - E), 0);
        lo = bits < 64 ? lo >> bits | (bits ? hi << (64 - bits) : 0) : bits < 128 ? hi >> (bits - 64) : 0;
        hi = bits < 64 ? hi >> bits : 0;
    } else {
        const int bits = g ? 0 : BITS * D;                      // that belong to the row
        lo = bits < 64 ? lo & ~(~0ull << bits) : lo;
        hi = bits > 64 ? hi & ~(~0ull << (bits - 64)) : 0;
    }
    return u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

// Granule g of a row of D elements (zeros beyond D); vec: rows divide into granules and lie on 16-byte boundaries.
template <typename T> __device__ inline u32x4 load_granule(const T *row, int g, int D, bool vec)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (!vec) return granule_in_place<T>(granule_anywhere<T>(row, g, D), g, D);
    u32x4 x = {0u, 0u, 0u, 0u};
    if (g * E < D) x = *(const ATT_GLOBAL u32x4 *)((const ATT_GLOBAL T *)row + g * E);
    return x;
}

// Four consecutive elements from d on.
template <typename T> __device__ inline void store4(T *row, int d, int D, bool vec, float a, float b, float c, float e)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 x = {(T)a, (T)b, (T)c, (T)e};
    ATT_GLOBAL T *p = (ATT_GLOBAL T *)row;
    if (vec) {
        if (d < D) *(ATT_GLOBAL T4 *)(p + d) = x;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) p[d + j] = x[j];
    }
}

template <typename T> __device__ inline T *row_of(const AttTensor &a, long long row, int head)
{
    return static_cast<T *>(a.p) + row * a.row + (long long)head * a.head;
}

// ---- staging straight into LDS ------------------------------------------------------------

static __device__ const u32x4 att_zeros[1] = {};

// 16 bytes a lane from global memory to LDS, lane l's at lds + 16 l; nothing passes through registers.  The hardware counts it with the vector
// loads; stage_wait() waits for it.  (Written out because the compiler, given its builtin, waits in front of every LDS read that follows.  It has no
// output register that could be reused too early, and what the compiler counts itself only becomes stricter by it.)
// (m0 is named as written: it is reserved, so that the compiler keeps nothing of its own there and warns of the name, but where it sets m0 for an
// instruction of its own it may do so far ahead.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void stage_16(uint32_t lds, const void *p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
__device__ inline void stage_16(uint32_t lds, const void *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// 4 bytes a lane.
__device__ inline void stage_4(uint32_t lds, const void *p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop
// Makes the compiler wait for loads into x here.  Without it, it waits at their first use: inside a loop in every pass, and then for what is
// being staged as well.
template <typename F, int N> __device__ inline void arrived(F (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
__device__ inline void stage_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Which granule of a tile of N rows belongs at a thread's i-th place: the exchange is its own inverse within 256 bytes.
template <typename T, int DP> __device__ inline void place_of(int slot, int *row, int *granule)
{
    typedef Rows<T, DP> R;
    const int line = R::GPR >= 16 ? slot / R::GPR : (slot >> 4) * (16 / R::GPR);
    const int e = slot ^ R::turn(line);
    *row = e / R::GPR;
    *granule = e % R::GPR;
}

// Tiles of N rows that follow one another in memory at one distance, whole in D: a thread's places are the same in every tile, so that only the
// tile's base moves, in scalar registers.
template <typename T, int DP, int N, int THREADS> struct NearRows {
    static constexpr int GRANULES = N * Rows<T, DP>::GPR, EACH = (GRANULES + THREADS - 1) / THREADS;
    uint32_t offset[EACH];
    __device__ explicit NearRows(long long row)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            int r, g;
            place_of<T, DP>(i * THREADS + threadIdx.x, &r, &g);
            offset[i] = (uint32_t)r * (uint32_t)row * (uint32_t)sizeof(T) + g * 16;
        }
    }
    __device__ void stage(unsigned char *tile, const T *first) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t base = lds_address(tile) + wave * 1024;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (GRANULES % THREADS == 0 || i * THREADS + wave * 64 < GRANULES) stage_16(base + i * THREADS * 16, first, offset[i]);
    }
};

// Puts N rows into a tile; row(r) gives where row r lies, or nothing for a row of zeros.  VEC: straight into LDS (stage_wait and a barrier before
// it is read).  Else, rows that do not divide into granules: through registers, requested by request() and put into place by put().
template <typename T, int DP, int N, int THREADS, bool VEC> struct StageRows {
    typedef Rows<T, DP> R;
    static constexpr int GRANULES = N * R::GPR, EACH = (GRANULES + THREADS - 1) / THREADS;
    u32x4 held[VEC ? 1 : EACH];

    template <typename F> __device__ void request(unsigned char *tile, int D, F row)
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t base = lds_address(tile) + wave * 1024;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (GRANULES % THREADS != 0 && i * THREADS + wave * 64 >= GRANULES) continue;
            int r, g;
            place_of<T, DP>(i * THREADS + threadIdx.x, &r, &g);
            const T *p = row(r);
            if constexpr (VEC) {
                const void *from = p && g * R::EPG < D ? (const void *)(p + g * R::EPG) : (const void *)att_zeros;
                stage_16(base + i * THREADS * 16, from);
            } else {
                held[i] = p ? granule_anywhere<T>(p, g, D) : u32x4{0u, 0u, 0u, 0u};
            }
        }
    }
    __device__ void put(unsigned char *tile, int D) const
    {
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (GRANULES % THREADS != 0 && i * THREADS + (threadIdx.x & ~63) >= GRANULES) continue;
                int r, g;
                place_of<T, DP>(i * THREADS + threadIdx.x, &r, &g);
                *reinterpret_cast<u32x4 *>(tile + (i * THREADS + threadIdx.x) * 16) = granule_in_place<T>(held[i], g, D);
            }
        }
    }
};

// The nodes of a tree, or of a part of it, that may be read, up to BN at a time.  With a mask their numbers go through a ring in LDS, filled
// from 4 THREADS mask bytes at a time, so that masked nodes cost neither a place in a tile nor a read.
template <int BN, int THREADS> struct Nodes {
    static constexpr int RING = 2048;
    static constexpr int LDS = RING * 4 + 64;
    static_assert(BN + 4 * THREADS <= RING, "room for what is left and a filling");
    const ATT_GLOBAL uint8_t *mask;
    int at, hi;                 // the next node to look at, the end
    int first, n;               // the current stage: its first node, or place in the ring
    int tail;                   // end of the ring's filling
    int *ring, *counts;

    __device__ void begin(const AttArgs &a, int from, int to, unsigned char *lds)
    {
        mask = (const ATT_GLOBAL uint8_t *)a.mask;
        at = from;
        hi = to;
        first = n = tail = 0;
        ring = reinterpret_cast<int *>(lds);
        counts = ring + RING;
    }
    // The next stage; how many nodes it has.  Everyone must call it.
    __device__ int next()
    {
        if (!mask) {
            first = at;
            n = max(min(BN, hi - at), 0);
            at += n;
            return n;
        }
        first += n;
        while (tail - first < BN && at < hi) {
            const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            const int mine = at + 4 * threadIdx.x;
            unsigned bits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint8_t m = mask[min(mine + j, hi - 1)];
                bits |= mine + j < hi && m ? 1u << j : 0u;
            }
            int upto = __popc(bits);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(upto, o);
                upto += lane >= o ? y : 0;
            }
            __syncthreads();                                    // (the ring's last reads, and counts', are over)
            if (lane == 63) counts[wave] = upto;
            __syncthreads();
            int place = tail + upto - __popc(bits), all = 0;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) {
                place += w < wave ? counts[w] : 0;
                all += counts[w];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (bits >> j & 1) ring[place++ & (RING - 1)] = mine + j;
            tail += __builtin_amdgcn_readfirstlane(all);
            at += 4 * THREADS;
            __syncthreads();
        }
        n = min(BN, tail - first);
        return n;
    }
    // Number of the stage's r-th node.
    __device__ int node(int r) const { return mask ? ring[(first + r) & (RING - 1)] : first + r; }
};

// ---- forward ------------------------------------------------------------------------------

// Four waves: WM side by side along the rows, 32 packed rows each, and WK = 4 / WM along the nodes, whose sums are joined at the end; NT node tiles
// of 32 per wave and stage.
// One pass over a tree's nodes: scores of a stage, their maximum and sum joined with those so far (what is summed is scaled when the maximum moves),
// probabilities, their product with the values.  Bounds and measurements (us of the kernel): few rows, long trees: memory (4 documents of 40 000
// to 65 000 nodes, one token, bf16, 8 heads of 128: 177, 4.9 TB/s); many rows: LDS reads, exponentials and products of two waves per SIMD one after
// the other (8 documents, 768 tokens x 16 heads, bf16 x 128: 234 to 247 from machine to machine, 720 to 760 TFLOP/s); short trees: one chain of reads and products, and tiles that
// their rows and nodes fill to 40 % (256 trees of 54 nodes: one token 7.5, 33 words of bf16 x 64 20).
template <typename T, int DP, int WM_> struct AttFwd {
    static constexpr int THREADS = ATT_THREADS;
    static constexpr int WM = WM_, WK = ATT_WAVES / WM;
    static constexpr int NT = WM == 4 && DP * (int)sizeof(T) <= 256 ? 2 : 1;
    // Of a probability: the second one costs time only where there are many rows.  One term: o is off by 0.0023 of its size in bf16 where its own
    // rounding is 0.0017.
    static constexpr int TERMS = WM == 4 ? 1 : 2;
    static constexpr int BM = 32 * WM;
    static constexpr int BN = 32 * WK * NT;
    static constexpr int STAGE = 2 * BN * Rows<T, DP>::BYTES;
    static constexpr int MAX_BUFS = STAGE <= 32768 ? 2 : 1;
    static constexpr int JOIN_WAVES = WK == 4 ? 4 : WK - 1;
    static constexpr int JOIN = JOIN_WAVES * WM * 32 * (DP + 6) * 4;
    __host__ __device__ static constexpr int list(int bufs) { return STAGE * bufs > JOIN ? STAGE * bufs : JOIN; }    // place of the nodes' ring
    __host__ __device__ static constexpr int lds(int bufs, bool mask) { return list(bufs) + (mask ? Nodes<BN, THREADS>::LDS : 0); }
    static constexpr int MIN_WAVES = DP * (int)sizeof(T) > 256 ? 1 : 2;
};

template <typename T, int DP, int WM, bool VEC>
__global__ __launch_bounds__(ATT_THREADS, (VEC || DP < 128 ? AttFwd<T, DP, WM>::MIN_WAVES : 1)) void k_attend(const AttArgs a)
{
    typedef AttFwd<T, DP, WM> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int WK = C::WK, NT = C::NT, DT = DP / 32, THREADS = C::THREADS;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wk = wave / WM;
    const uint32_t id = xcd_order(blockIdx.x, gridDim.x), lists = id / (uint32_t)a.slots;
    const int slot = (int)(id - lists * a.slots), hk = (int)(lists / (uint32_t)a.splits), part = (int)(lists - hk * (uint32_t)a.splits);
    long long tile;
    const int tree = find_slot(a.q_off, a.n_trees, a.G, C::BM == 32 ? 5 : C::BM == 64 ? 6 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G, m0 = tile * C::BM;
    if (tile < 0 || m0 >= n_rows) return;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    if (a.splits > 1) {
        const int n_stage = (hi - lo + C::BN - 1) / C::BN, per = (n_stage + a.splits - 1) / a.splits;
        const int s_lo = min(part * per, n_stage), s_hi = min(s_lo + per, n_stage);
        if (s_lo >= s_hi) return;
        hi = min(hi, lo + s_hi * C::BN);
        lo += s_lo * C::BN;
    }

    // the lane's query (a row beyond the last one repeats the first: its results are not stored)
    const long long m = m0 + 32 * wm + col;
    const bool mine = m < n_rows;
    const Packed rows(q_lo, m0, a.G);
    int qi, head;
    rows.at(mine ? 32 * wm + col : 0, &qi, &head);
    head += hk * a.G;
    frag qf[R::STEPS];
    {
        const T *qr = row_of<T>(a.q, qi, head);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) qf[s] = __builtin_bit_cast(frag, load_granule<T>(qr, 2 * s + half, a.D, VEC));
    }
    floatx16 acc[DT];
    float top = -INFINITY, sum = 0.f;          // largest raw score so far (of the lane's query), sum of the lane's half of its nodes
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = floatx16{};

    const T *kp = row_of<T>(a.k, 0, hk), *vp = row_of<T>(a.v, 0, hk);
    Nodes<C::BN, THREADS> nodes;
    const bool two = C::MAX_BUFS == 2 && a.bufs == 2;
    nodes.begin(a, lo, hi, att_lds + C::list(two ? 2 : 1));
    const bool near = VEC && !a.mask && a.near && a.D == DP;
    const NearRows<T, DP, C::BN, THREADS> k_near(a.k.row), v_near(a.v.row);
    StageRows<T, DP, C::BN, THREADS, VEC> ks, vs;
    auto request = [&](unsigned char *b) {
        if (near && nodes.n == C::BN) {
            k_near.stage(b, kp + nodes.first * a.k.row);
            v_near.stage(b + C::STAGE / 2, vp + nodes.first * a.v.row);
            return;
        }
        ks.request(b, a.D, [&](int r) { return r < nodes.n ? kp + nodes.node(r) * a.k.row : (const T *)nullptr; });
        vs.request(b + C::STAGE / 2, a.D, [&](int r) { return r < nodes.n ? vp + nodes.node(r) * a.v.row : (const T *)nullptr; });
    };
    auto put = [&](unsigned char *b) {
        ks.put(b, a.D);
        vs.put(b + C::STAGE / 2, a.D);
    };
    RowReads<T, DP> kr(att_lds + 32 * NT * wk * R::BYTES);
    ColumnReads<T, DP> vc(att_lds + C::STAGE / 2 + 32 * NT * wk * R::BYTES, 0);
    // one stage of n nodes; the wave's own are those from 32 NT wk on.  TAIL: some of them may be missing.
    auto compute = [&](auto tail, int n) {
        constexpr bool TAIL = decltype(tail)::value;
        const int left = n - 32 * NT * wk;
        if (TAIL && left <= 0) return;
        floatx16 p[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) p[t] = floatx16{};
#pragma unroll
        for (int d = 0; d < R::STEPS; ++d)
#pragma unroll
            for (int t = 0; t < NT; ++t) mma(p[t], kr.get(32 * t, d), qf[d]);
        if (TAIL) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + 8 * (r >> 2) + 4 * half + (r & 3) >= left) p[t][r] = -INFINITY;
        }
        float high = top;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) high = fmaxf(high, p[t][r]);
        high = max_of_halves(high);
        const float ref = high == -INFINITY ? 0.f : high * a.scale_log2, less = ATT_LIFT<T> > 0.f ? ATT_LIFT<T> - ref : -ref;
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
                p[t][r] = __builtin_amdgcn_exp2f(fmaf(p[t][r], a.scale_log2, less));
                sum += p[t][r];
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (!TAIL || 32 * t < left) mma_columns<T, DP, C::TERMS, DT>(acc, vc, 32 * t, p[t]);
    };
    int n = nodes.next(), odd = 0;
    if (n) {
        request(att_lds);
        put(att_lds);
    }
    arrived(qf);
    while (n == C::BN) {                                        // (all stages but the last are full)
        unsigned char *next = att_lds + (two && !odd ? C::STAGE : 0);
        if (VEC) stage_wait();
        __syncthreads();
        n = nodes.next();
        if ((!VEC || two) && n) request(next);
        compute(std::false_type{}, C::BN);
        if (!two) {
            __syncthreads();
            if (VEC && n) request(next);
        } else {
            kr.move(odd ? -C::STAGE : C::STAGE);
            vc.move(odd ? -C::STAGE : C::STAGE);
        }
        if (n) put(next);
        odd ^= 1;
    }
    if (n) {
        if (VEC) stage_wait();
        __syncthreads();
        compute(std::true_type{}, n);
    }
    sum = sum_of_halves(sum);

    const bool partial = a.splits > 1;
    // one query's result: four of its columns, from d on
    auto store = [&](int i, int hd, int d, float inv, const f32x4 &x) {
        if (partial)
            store4<float>(a.part_o + ((long long)part * a.n_q * a.Hq + (long long)i * a.Hq + hd) * a.D, d, a.D, (a.D & 3) == 0, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
        else
            store4<T>(row_of<T>(a.o, i, hd), d, a.D, a.vec_out, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    };
    auto store_lse = [&](int i, int hd, bool any, float highest, float total) {
        const float lse = any ? (highest * a.scale_log2 + (__builtin_amdgcn_logf(total) - ATT_LIFT<T>)) * 0.6931471805599453f : -INFINITY;
        const long long rh = (long long)i * a.Hq + hd;
        if (partial) a.part_lse[(long long)part * a.n_q * a.Hq + rh] = lse;
        else if (a.lse) a.lse[rh] = lse;
    };
    if constexpr (WK <= 2) {
        if constexpr (WK == 2) {
            // the second wave's sums over its nodes, brought to one maximum with the first one's
            float *jo = reinterpret_cast<float *>(att_lds) + (32 * wm + col) * (DP + 4), *jt = reinterpret_cast<float *>(att_lds) + WM * 32 * (DP + 4) + (32 * wm + col) * 2;
            __syncthreads();
            if (wk == 1) {
                if (half == 0) {
                    jt[0] = top;
                    jt[1] = sum;
                }
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *reinterpret_cast<f32x4 *>(jo + 32 * t + 2 * r + 4 * half) = f32x4{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
            }
            __syncthreads();
            if (wk == 1) return;
            const float other = jt[0], highest = fmaxf(top, other);
            const float f = top == highest ? 1.f : __builtin_amdgcn_exp2f((top - highest) * a.scale_log2);
            const float g = other == highest ? 1.f : __builtin_amdgcn_exp2f((other - highest) * a.scale_log2);
            top = highest;
            sum = f * sum + g * jt[1];
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(jo + 32 * t + 2 * r + 4 * half);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[t][r + j] = f * acc[t][r + j] + g * y[j];
                }
        }
        if (!mine) return;
        const bool any = sum > 0.f || sum != sum;
        const float inv = any ? 1.f / sum : 0.f;
        if (half == 0) store_lse(qi, head, any, top, sum);
        if (!any) {                                             // (zero times an infinite value is a NaN)
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] = floatx16{};
        }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                store(qi, head, 32 * t + 2 * r + 4 * half, inv, f32x4{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]});
    } else {
        // the waves' sums over their nodes, brought to one maximum
        float *jo = reinterpret_cast<float *>(att_lds), *jt = jo + ATT_WAVES * 32 * (DP + 4), *js = jt + ATT_WAVES * 32;
        const int mine_at = (wk * WM + wm) * 32 + col;
        __syncthreads();
        if (half == 0) {
            jt[mine_at] = top;
            js[mine_at] = sum;
        }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4 *>(jo + mine_at * (DP + 4) + 32 * t + 2 * r + 4 * half) =
                    f32x4{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
        __syncthreads();
        constexpr int G4 = DP / 4;
        const int n_here = (int)min((long long)C::BM, n_rows - m0);
        for (int e = threadIdx.x; e < n_here * G4; e += THREADS) {
            const int r = e / G4, d = 4 * (e % G4);
            float tt = -INFINITY, total = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) tt = fmaxf(tt, jt[w * C::BM + r]);
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float tw = jt[w * C::BM + r];
                const float f = tw == tt ? 1.f : __builtin_amdgcn_exp2f((tw - tt) * a.scale_log2);
                total += f * js[w * C::BM + r];
                const f32x4 y = *reinterpret_cast<const f32x4 *>(jo + (w * C::BM + r) * (DP + 4) + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += f * y[j];
            }
            const bool any = total > 0.f || total != total;
            int i, hd;
            rows.at(r, &i, &hd);
            hd += hk * a.G;
            if (d == 0) store_lse(i, hd, any, tt, total);
            store(i, hd, d, any ? 1.f / total : 0.f, any ? x : f32x4{0.f, 0.f, 0.f, 0.f});
        }
    }
}

// Joins the parts of a split forward: one workgroup per query and head, waves along the parts, lanes along the columns, so that a chain of loads is
// a quarter of the parts long and its loads do not wait for each other.  BN: nodes per stage of the kernel that made them.
template <typename T> __global__ __launch_bounds__(ATT_THREADS) void k_attend_join(const AttArgs a, int bn)
{
    __shared__ float sums[ATT_WAVES][256], weights[256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long rh = blockIdx.x, n = (long long)a.n_q * a.Hq;
    const int qi = (int)divide(rh, a.Hq), head = (int)(rh - (long long)qi * a.Hq);
    int lo, hi;
    const int tree = find_last(a.n_trees, qi, [&](int t) { return (long long)a.q_off[t]; });
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    const int n_stage = (hi - lo + bn - 1) / bn, per = (n_stage + a.splits - 1) / a.splits;
    const int parts = per ? (n_stage + per - 1) / per : 0;
    // the parts' logarithms (at most 256 parts): every wave works out the largest and the total
    float l[4], top = -INFINITY, total = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        l[i] = lane + 64 * i < parts ? a.part_lse[(lane + 64 * i) * n + rh] : -INFINITY;
        top = fmaxf(top, l[i]);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        l[i] = l[i] == -INFINITY ? 0.f : __expf(l[i] - top);
        total += l[i];
        if (wave == 0) weights[lane + 64 * i] = l[i];
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o);
    __syncthreads();
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int j = wave; j < parts; j += ATT_WAVES) {
        const ATT_GLOBAL float *po = (const ATT_GLOBAL float *)a.part_o + (j * n + rh) * a.D;
        const float f = weights[j];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (lane + 64 * t < a.D) x[t] = fmaf(f, po[lane + 64 * t], x[t]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) sums[wave][lane + 64 * t] = x[t];
    __syncthreads();
    const bool any = total > 0.f || total != total;
    const float inv = any ? 1.f / total : 0.f;
    const int d = threadIdx.x;
    if (d < a.D) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < ATT_WAVES; ++w) y += sums[w][d];
        row_of<T>(a.o, qi, head)[d] = (T)(y * inv);
    }
    if (a.lse && d == 0) a.lse[rh] = any ? top + __logf(total) : -INFINITY;
}

// ---- backward -----------------------------------------------------------------------------

// What exp2 subtracts: a row without nodes (lse = -inf) has no probabilities.
__device__ inline float lse_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// P (dP - delta); zero where the probability is, also beside an infinite value: v_mul_legacy_f32, whose zero times anything is zero.  (The compiler's
// intrinsic by its name: there is no builtin for it, and written as assembly it would not be scheduled.)
extern "C" __device__ float mul_zero_wins(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ inline float score_gradient(float p, float gap) { return mul_zero_wins(p, gap); }

// What both kernels of the backward pass need first.  Workgroups below `row_blocks`: delta[i] = d_o[i] . o[i] (of the o that was stored, rounded to the type: an
// output of fp32 beside it would be twice its bytes to write and to read again) and the logarithms in base 2, 16 lanes per query and head (fp16: also the
// power of two that brings the row of d_o to a length of 2^10, see fit_fp16).  With a mask, one further workgroup per tree: the tree's nodes that may be
// read, one after the other in `list` from kv_off[tree] on, and their number in live[tree]; masked nodes then cost the others nothing.
template <typename T> __global__ __launch_bounds__(ATT_THREADS) void k_attend_prepare(const AttArgs a, int row_blocks)
{
    if ((int)blockIdx.x < row_blocks) {
        const int l16 = threadIdx.x & 15;
        const long long rh = ((long long)blockIdx.x * ATT_THREADS + threadIdx.x) >> 4, n = (long long)a.n_q * a.Hq;
        float x = 0.f, sq = 0.f;
        if (rh < n) {
            const int qi = (int)divide(rh, a.Hq), head = (int)(rh - (long long)qi * a.Hq);
            const T *o = row_of<T>(a.o, qi, head), *g = row_of<T>(a.d_o, qi, head);
            constexpr int E = 16 / (int)sizeof(T);
            for (int c = l16; c * E < a.D; c += 16) {
                T y[E], z[E];
                const u32x4 yo = load_granule<T>(o, c, a.D, a.vec), zo = load_granule<T>(g, c, a.D, a.vec);
                __builtin_memcpy(y, &yo, 16);
                __builtin_memcpy(z, &zo, 16);
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    x = fmaf((float)y[j], (float)z[j], x);
                    sq = fmaf((float)z[j], (float)z[j], sq);
                }
            }
        }
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) {
            x += __shfl_xor(x, o);
            sq += __shfl_xor(sq, o);
        }
        if (rh < n && l16 == 0) {
            a.delta[rh] = x;
            a.ref[rh] = lse_log2(a.lse[rh]) - ATT_LIFT<T>;
            // (of the lifted score gradients, so without the lift)
            if (std::is_same<T, f16_t>::value) a.size[rh] = sq > 0.f && sq < INFINITY ? exp2f(10.f - ATT_LIFT<T> - ceilf(0.5f * log2f(sq))) : 1.f / ATT_LIFTED<T>;
        }
        return;
    }
    __shared__ int counts[ATT_WAVES];
    constexpr int EACH = 16;
    const int tree = blockIdx.x - row_blocks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int lo, hi, n = 0;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    for (int at = lo; at < hi; at += EACH * ATT_THREADS) {
        const int mine = at + EACH * threadIdx.x;
        unsigned bits = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) bits |= a.mask[min(mine + j, hi - 1)] != 0 && mine + j < hi ? 1u << j : 0u;
        int upto = __popc(bits);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o);
            upto += lane >= o ? y : 0;
        }
        __syncthreads();
        if (lane == 63) counts[wave] = upto;
        __syncthreads();
        int place = lo + n + upto - __popc(bits);
#pragma unroll
        for (int w = 0; w < ATT_WAVES; ++w) {
            place += w < wave ? counts[w] : 0;
            n += counts[w];
        }
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (bits >> j & 1) a.list[place++] = mine + j;
    }
    if (threadIdx.x == 0) a.live[tree] = n;
}

// Both gradients take the scores and probabilities again from lse: five products a pair of tiles would do, seven are done, so that neither side needs
// the other's sums or atomics.  Scores, probabilities and d_o . v stay in a lane's registers and are operands of the second products as they stand.
// The launch of both (us): 8 documents of 1 700 nodes, 70 % of them read, 384 tokens x 16 heads, bf16 x 128: 243 (apart, and with two
// terms of the probabilities too: 314); 256 trees of 54 nodes, 33 words, fp32 x 64, 8 heads: 165 (matrix unit 31 % busy, 60 % of it on places that short trees leave
// empty; most of the rest is waiting, at two waves per SIMD, for what is not known: a shorter search for the tree changed nothing); 25 trees, x 30: 14.
//
// dQ: like the forward, rows (queries) on the lanes' columns.  Four waves: WM side by side along the rows, WK along the nodes (their sums are joined
// at the end) and, for wide heads, WD along the columns of dQ, where every wave of a row tile works out the tile's scores itself.
template <typename T, int DP, int WM_> struct AttDq {
    static constexpr int WD = DP > 128 ? 2 : 1;
    static constexpr int WM = DP > 128 ? 2 : WM_;
    static constexpr int WK = ATT_WAVES / WM / WD;
    static constexpr int BM = 32 * WM;
    static constexpr int NT = WK == 1 && DP * (int)sizeof(T) <= 256 ? 2 : 1;
    static constexpr int BN = 32 * WK * NT;
    static constexpr int DT = DP / 32 / WD;
    static constexpr int STAGE = 2 * BN * Rows<T, DP>::BYTES;
    static constexpr int JOIN = WK > 1 ? WM * 32 * (DP + 4) * 4 : 0;
    static constexpr int lds(int bufs) { return bufs * STAGE > JOIN ? bufs * STAGE : JOIN; }
};

template <typename T, int DP, int WM, bool VEC> __device__ __forceinline__ void attend_dq(const AttArgs &a, uint32_t block, uint32_t blocks)
{
    typedef AttDq<T, DP, WM> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int DT = C::DT, BN = C::BN;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wd = wave % C::WD, wm = wave / C::WD % C::WM, wk = wave / C::WD / C::WM;
    const bool two = a.bufs == 2;
    const uint32_t id = xcd_order(block, blocks), lists = id / (uint32_t)a.slots;
    const int slot = (int)(id - lists * a.slots), hk = (int)(lists / (uint32_t)a.splits), part = (int)(lists - hk * (uint32_t)a.splits);
    long long tile;
    const int tree = find_slot(a.q_off, a.n_trees, a.G, C::BM == 64 ? 6 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G, m0 = tile * C::BM;
    if (tile < 0 || m0 >= n_rows) return;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    int n_nodes = a.mask ? min(__builtin_amdgcn_readfirstlane(a.live[tree]), hi - lo) : hi - lo;
    int first = 0;                              // of the stage that is staged next
    if (a.splits > 1) {
        const int n_stage = (n_nodes + BN - 1) / BN, per = (n_stage + a.splits - 1) / a.splits;
        first = min(part * per * BN, n_nodes);
        n_nodes = min(first + per * BN, n_nodes);
    }

    const long long m = m0 + 32 * wm + col;
    const bool mine = m < n_rows;
    int qi, head;
    Packed(q_lo, m0, a.G).at(mine ? 32 * wm + col : 0, &qi, &head);
    head += hk * a.G;
    const long long row_head = (long long)qi * a.Hq + head;
    frag qf[R::STEPS], gf[R::STEPS];
    {
        const T *qr = row_of<T>(a.q, qi, head), *gr = row_of<T>(a.d_o, qi, head);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) {
            qf[s] = __builtin_bit_cast(frag, load_granule<T>(qr, 2 * s + half, a.D, VEC));
            gf[s] = __builtin_bit_cast(frag, load_granule<T>(gr, 2 * s + half, a.D, VEC));
        }
    }
    constexpr bool F16 = std::is_same<T, f16_t>::value;
    float row[3] = {a.ref[row_head], a.delta[row_head], F16 ? a.size[row_head] : 1.f};
    floatx16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = floatx16{};

    const T *kp = row_of<T>(a.k, 0, hk), *vp = row_of<T>(a.v, 0, hk);
    const ATT_GLOBAL int32_t *list = (const ATT_GLOBAL int32_t *)a.list + lo;
    const bool near = VEC && !a.mask && a.near && a.D == DP;
    const NearRows<T, DP, BN, ATT_THREADS> k_near(a.k.row), v_near(a.v.row);
    StageRows<T, DP, BN, ATT_THREADS, VEC> ks, vs;
    auto request = [&](unsigned char *b, int n) {
        if (near && n == BN) {
            k_near.stage(b, kp + (lo + first) * a.k.row);
            v_near.stage(b + C::STAGE / 2, vp + (lo + first) * a.v.row);
        } else {
            auto node = [&](int r) { return (long long)(a.mask ? list[first + r] : lo + first + r); };
            ks.request(b, a.D, [&](int r) { return r < n ? kp + node(r) * a.k.row : (const T *)nullptr; });
            vs.request(b + C::STAGE / 2, a.D, [&](int r) { return r < n ? vp + node(r) * a.v.row : (const T *)nullptr; });
        }
        first += BN;
    };
    auto put = [&](unsigned char *b) {
        ks.put(b, a.D);
        vs.put(b + C::STAGE / 2, a.D);
    };
    const int own = 32 * C::NT * wk * R::BYTES;
    RowReads<T, DP> kr(att_lds + own);          // (rows of v lie BN rows behind)
    ColumnReads<T, DP> kc(att_lds + own, 32 * DT * wd);
    // one stage of n nodes.  TAIL: some may be missing (rows of zeros, but exp2 of a large -lse would still be infinite).
    auto compute = [&](auto tail, int n) {
        n -= 32 * C::NT * wk;
#pragma unroll
        for (int j = 0; j < C::NT; ++j) {
            if (decltype(tail)::value && 32 * j >= n) break;
            floatx16 p = {}, dp = {};
#pragma unroll
            for (int d = 0; d < R::STEPS; ++d) {
                mma(p, kr.get(32 * j, d), qf[d]);
                mma(dp, kr.get(32 * j + BN, d), gf[d]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = score_gradient(__builtin_amdgcn_exp2f(fmaf(p[r], a.scale_log2, -row[0])), dp[r] - row[1]);
                p[r] = decltype(tail)::value && 32 * j + 8 * (r >> 2) + 4 * half + (r & 3) >= n ? 0.f : e;
            }
            if constexpr (F16) fit_fp16(p, row[2], acc);
            mma_columns<T, DP, 2, DT>(acc, kc, 32 * j, p);
        }
    };
    int left = n_nodes - first, odd = 0;
    if (left > 0) {
        request(att_lds, min(left, BN));
        put(att_lds);
    }
    arrived(qf);
    arrived(gf);
    arrived(row);
    for (; left > BN; left -= BN) {
        if (VEC) stage_wait();
        __syncthreads();
        unsigned char *next = att_lds + (!two || odd ? 0 : C::STAGE);
        if (!VEC || two) request(next, min(left - BN, BN));
        compute(std::false_type{}, BN);
        if (!two) {
            __syncthreads();
            if (VEC) request(next, min(left - BN, BN));
        }
        put(next);
        const int step = !two ? 0 : odd ? -C::STAGE : C::STAGE;
        kr.move(step);
        kc.move(step);
        odd ^= 1;
    }
    if (left > 0) {
        if (VEC) stage_wait();
        __syncthreads();
        compute(std::true_type{}, left);
    }
    // (a row whose scores are all -infinity: its zeros may have met infinite keys)
    const bool none = row[0] == INFINITY;
    const float out_scale = a.scale / (row[2] * ATT_LIFTED<T>);
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = none ? floatx16{} : acc[t] * out_scale;
    if constexpr (C::WK == 2) {
        float *join = reinterpret_cast<float *>(att_lds) + (wm * 32 + col) * (DP + 4);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                if (wk == 1) *reinterpret_cast<f32x4 *>(join + 32 * t + 2 * r + 4 * half) = f32x4{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
        __syncthreads();
        if (wk == 1) return;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 y = *reinterpret_cast<const f32x4 *>(join + 32 * t + 2 * r + 4 * half);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][r + j] += y[j];
            }
    }
    if (!mine) return;
    T *o = row_of<T>(a.d_q, qi, head);
    float *po = a.part_q + ((long long)part * a.n_q * a.Hq + row_head) * a.D;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * (DT * wd + t) + 2 * r + 4 * half;
            const f32x4 x = {acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
            if (a.splits > 1) store4<float>(po, d, a.D, (a.D & 3) == 0, x[0], x[1], x[2], x[3]);
            else store4<T>(o, d, a.D, a.vec_out, x[0], x[1], x[2], x[3]);
        }
}

// dK and dV: nodes on the lanes' columns, packed query rows go by in LDS.  Every sum over queries and over the heads of a group is
// taken by one wave in one order: no atomics, the same bits every run.
template <typename T, int DP, int WN_> struct AttDkv {
    static constexpr int WD = DP <= 128 ? 1 : sizeof(T) == 2 ? 2 : 4;       // wide heads: waves along the columns of dK and dV
    static constexpr int WN = DP <= 128 ? WN_ : ATT_WAVES / WD;
    static constexpr int WQ = ATT_WAVES / WN / WD;                          // waves along the rows; their sums are joined at the end
    static constexpr int BN = 32 * WN;
    static constexpr int QT = WQ == 1 && DP * (int)sizeof(T) <= 128 ? 2 : 1;
    static constexpr int BQ = 32 * WQ * QT;
    static constexpr int DT = DP / 32 / WD;
    static constexpr int STAGE = 2 * BQ * Rows<T, DP>::BYTES + 512;         // rows of q, of d_o, 64 logarithms, 64 deltas
    static constexpr int JOIN = WQ > 1 ? WN * 32 * 2 * (DP + 4) * 4 : 0;
    // Of a probability: the second one costs time only where there are many rows.  (Of a score gradient always two: it is a difference, and the error of d_k
    // from rounding it once is up to 1.6 times that of d_k's own rounding.)
    static constexpr int TERMS = DP <= 128 && WN == 4 && !std::is_same<T, f16_t>::value ? 1 : 2;
    static constexpr int lds(int bufs) { return bufs * STAGE > JOIN ? bufs * STAGE : JOIN; }
    static constexpr int MIN_WAVES = DP * (int)sizeof(T) > 256 ? 1 : 2;
};

static __device__ const float att_no_row[2] = {INFINITY, 0.f};              // logarithm and delta of a row that is not there

template <typename T, int DP, int WN, bool VEC> __device__ __forceinline__ void attend_dkv(const AttArgs &a, uint32_t block, uint32_t blocks)
{
    typedef AttDkv<T, DP, WN> C;
    typedef Rows<T, DP> R;
    typedef typename Elem<T>::frag frag;
    constexpr int DT = C::DT, BQ = C::BQ, BN = C::BN;
    extern __shared__ __align__(16) unsigned char att_lds[];

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wd = wave % C::WD, wn = wave / C::WD % C::WN, wq = wave / C::WD / C::WN;
    const bool two = a.kv_bufs == 2;
    const uint32_t id = xcd_order(block, blocks), lists = id / (uint32_t)a.kv_slots;
    const int slot = (int)(id - lists * a.kv_slots), hk = (int)(lists / (uint32_t)a.kv_splits), part = (int)(lists - hk * (uint32_t)a.kv_splits);
    if (hk >= a.Hk) return;                     // (the launch rounds up)
    long long tile;
    const int tree = find_slot(a.kv_off, a.n_trees, 1, BN == 32 ? 5 : BN == 64 ? 6 : 7, slot, &tile);
    int q_lo, q_hi, lo, hi;
    tree_range(a.kv_off, tree, a.n_kv, &lo, &hi);
    if (tile < 0 || tile * BN >= hi - lo) return;
    const int t0 = (int)tile * BN;
    tree_range(a.q_off, tree, a.n_q, &q_lo, &q_hi);
    const long long n_rows = (long long)(q_hi - q_lo) * a.G;
    int n_nodes = hi - lo;
    if (a.mask) {
        // masked nodes among the tile's own: zeros
        n_nodes = min(__builtin_amdgcn_readfirstlane(a.live[tree]), n_nodes);
        const int end = part == 0 ? min(t0 + BN, hi - lo) : t0;
        for (int r = t0 + wave; r < end; r += ATT_WAVES) {
            if (a.mask[lo + r]) continue;
            T *ok = row_of<T>(a.d_k, lo + r, hk), *ov = row_of<T>(a.d_v, lo + r, hk);
            for (int d = lane; d < a.D; d += 64) ok[d] = ov[d] = (T)0.f;
        }
        if (t0 >= n_nodes) return;
    }

    const int place = t0 + 32 * wn + col;
    const bool mine = place < n_nodes;
    const int at = mine ? place : t0;
    const long long node = a.mask ? ((const ATT_GLOBAL int32_t *)a.list)[lo + at] : lo + at;
    frag kf[R::STEPS], vf[R::STEPS];
    {
        const T *kr = row_of<T>(a.k, node, hk), *vr = row_of<T>(a.v, node, hk);
#pragma unroll
        for (int s = 0; s < R::STEPS; ++s) {
            kf[s] = __builtin_bit_cast(frag, load_granule<T>(kr, 2 * s + half, a.D, VEC));
            vf[s] = __builtin_bit_cast(frag, load_granule<T>(vr, 2 * s + half, a.D, VEC));
        }
    }
    floatx16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dk[t] = dv[t] = floatx16{};

    // Groups that divide a stage: a thread's places are the same in every stage, BQ / G queries further on.
    const bool near = VEC && a.near && a.D == DP && BQ % a.G == 0;
    constexpr int GRANULES = BQ * R::GPR, EACH = (GRANULES + ATT_THREADS - 1) / ATT_THREADS;
    uint32_t q_offset[EACH], g_offset[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        int r, g;
        place_of<T, DP>(i * ATT_THREADS + threadIdx.x, &r, &g);
        const int qr = (uint32_t)r / (uint32_t)a.G, hr = r - qr * a.G;
        q_offset[i] = ((uint32_t)qr * (uint32_t)a.q.row + (uint32_t)hr * (uint32_t)a.q.head) * (uint32_t)sizeof(T) + g * 16;
        g_offset[i] = ((uint32_t)qr * (uint32_t)a.d_o.row + (uint32_t)hr * (uint32_t)a.d_o.head) * (uint32_t)sizeof(T) + g * 16;
    }
    int n_stage = (int)((n_rows + BQ - 1) / BQ), s_lo = 0;
    if (a.kv_splits > 1) {
        const int per = (n_stage + a.kv_splits - 1) / a.kv_splits;
        s_lo = min(part * per, n_stage);
        n_stage = min(s_lo + per, n_stage);
    }
    long long first = (long long)s_lo * BQ;     // packed row that is staged next
    StageRows<T, DP, BQ, ATT_THREADS, VEC> qs, gs;
    auto request = [&](unsigned char *b) {
        const Packed rows(q_lo, first, a.G);
        const int left = (int)min(n_rows - first, (long long)BQ);
        if (near && left == BQ) {
            const T *qp = row_of<T>(a.q, rows.q0, hk * a.G), *gp = row_of<T>(a.d_o, rows.q0, hk * a.G);
            const uint32_t base = lds_address(b) + wave * 1024;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (GRANULES % ATT_THREADS == 0 || i * ATT_THREADS + wave * 64 < GRANULES) {
                    stage_16(base + i * ATT_THREADS * 16, qp, q_offset[i]);
                    stage_16(base + BQ * R::BYTES + i * ATT_THREADS * 16, gp, g_offset[i]);
                }
        } else {
            auto row = [&](const AttTensor &x, int r) {
                int i, hd;
                rows.at(r, &i, &hd);
                return (const T *)row_of<T>(x, i, hk * a.G + hd);
            };
            // (a row that is not there is the tree's first query without a gradient: the score of a row of zeros would be a NaN beside an infinite key)
            const T *some = row_of<T>(a.q, q_lo, hk * a.G);
            qs.request(b, a.D, [&](int r) { return r < left ? row(a.q, r) : some; });
            gs.request(b + BQ * R::BYTES, a.D, [&](int r) { return r < left ? row(a.d_o, r) : (const T *)nullptr; });
        }
        if (wave < 2) {                         // (64 places; those beyond BQ are not read)
            int i, hd;
            rows.at(lane, &i, &hd);
            const float *from = wave == 0 ? a.ref : a.delta;
            from = lane < left ? from + (long long)i * a.Hq + hk * a.G + hd : att_no_row + wave;
            stage_4(lds_address(b) + 2 * BQ * R::BYTES + wave * 256, from);
        }
        first += BQ;
    };
    auto put = [&](unsigned char *b) {
        qs.put(b, a.D);
        gs.put(b + BQ * R::BYTES, a.D);
    };
    const int own = 32 * C::QT * wq;            // the wave's first row of a stage
    RowReads<T, DP> qr(att_lds + own * R::BYTES);               // (those of d_o lie BQ rows behind)
    ColumnReads<T, DP> qc(att_lds + own * R::BYTES, 32 * DT * wd);
    const unsigned char *numbers = att_lds + 2 * BQ * R::BYTES + 16 * half + 4 * own;
    if (s_lo < n_stage) {
        request(att_lds);
        put(att_lds);
    }
    // score gradients as fp16 operands: begin at the size of the tree's largest row of d_o
    constexpr bool F16 = std::is_same<T, f16_t>::value;
    float size = 1.f;
    if constexpr (F16) {
        float s = INFINITY;
        for (long long m = lane; m < n_rows; m += 64) {
            const long long i = divide(m, a.G);
            s = fminf(s, a.size[(q_lo + i) * a.Hq + hk * a.G + (m - i * a.G)]);
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) s = fminf(s, __shfl_xor(s, o));
        size = s < INFINITY ? s : 1.f / ATT_LIFTED<T>;
    }
    arrived(kf);
    arrived(vf);
    for (int s = s_lo, odd = 0; s < n_stage; ++s, odd ^= 1) {
        stage_wait();
        __syncthreads();
        unsigned char *next = att_lds + (!two || odd ? 0 : C::STAGE);
        if (two && s + 1 < n_stage) request(next);
#pragma unroll
        for (int q = 0; q < C::QT; ++q) {
            if ((long long)s * BQ + own + 32 * q >= n_rows) break;
            floatx16 p = {}, dp = {};
#pragma unroll
            for (int d = 0; d < R::STEPS; ++d) {
                mma(p, qr.get(32 * q, d), kf[d]);
                mma(dp, qr.get(32 * q + BQ, d), vf[d]);
            }
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 rr = *reinterpret_cast<const f32x4 *>(numbers + 128 * q + 32 * r4);
                const f32x4 dd = *reinterpret_cast<const f32x4 *>(numbers + 256 + 128 * q + 32 * r4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * r4 + j;
                    p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], a.scale_log2, -rr[j]));
                    dp[r] = score_gradient(p[r], dp[r] - dd[j]);
                }
            }
            mma_columns<T, DP, C::TERMS, DT>(dv, qc, 32 * q + BQ, p);
            if constexpr (F16) fit_fp16(dp, size, dk);
            mma_columns<T, DP, 2, DT>(dk, qc, 32 * q, dp);
        }
        if (!two && s + 1 < n_stage) {
            __syncthreads();
            request(next);
        }
        if (s + 1 < n_stage) put(next);
        const int step = !two ? 0 : odd ? -C::STAGE : C::STAGE;
        qr.move(step);
        qc.move(step);
        numbers += step;
    }
    const float k_scale = a.scale / (size * ATT_LIFTED<T>);
#pragma unroll
    for (int t = 0; t < DT; ++t) dk[t] *= k_scale;
    if constexpr (C::WQ == 2) {
        float *join = reinterpret_cast<float *>(att_lds) + (wn * 32 + col) * 2 * (DP + 4);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                if (wq == 1) {
                    *reinterpret_cast<f32x4 *>(join + 32 * t + 2 * r + 4 * half) = f32x4{dk[t][r], dk[t][r + 1], dk[t][r + 2], dk[t][r + 3]};
                    *reinterpret_cast<f32x4 *>(join + DP + 4 + 32 * t + 2 * r + 4 * half) = f32x4{dv[t][r], dv[t][r + 1], dv[t][r + 2], dv[t][r + 3]};
                }
        __syncthreads();
        if (wq == 1) return;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 y = *reinterpret_cast<const f32x4 *>(join + 32 * t + 2 * r + 4 * half), z = *reinterpret_cast<const f32x4 *>(join + DP + 4 + 32 * t + 2 * r + 4 * half);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dk[t][r + j] += y[j];
                    dv[t][r + j] += z[j];
                }
            }
    }
    if (!mine) return;
    T *ok = row_of<T>(a.d_k, node, hk), *ov = row_of<T>(a.d_v, node, hk);
    float *pk = a.part_kv + (((long long)part * a.n_kv + node) * a.Hk + hk) * 2 * a.D, *pv = pk + a.D;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * (DT * wd + t) + 2 * r + 4 * half;
            const f32x4 x = {dk[t][r], dk[t][r + 1], dk[t][r + 2], dk[t][r + 3]};
            const f32x4 y = f32x4{dv[t][r], dv[t][r + 1], dv[t][r + 2], dv[t][r + 3]} * (1.f / ATT_LIFTED<T>);
            if (a.kv_splits > 1) {
                store4<float>(pk, d, a.D, (a.D & 3) == 0, x[0], x[1], x[2], x[3]);
                store4<float>(pv, d, a.D, (a.D & 3) == 0, y[0], y[1], y[2], y[3]);
            } else {
                store4<T>(ok, d, a.D, a.vec_out, x[0], x[1], x[2], x[3]);
                store4<T>(ov, d, a.D, a.vec_out, y[0], y[1], y[2], y[3]);
            }
        }
}

// Both in one launch: neither needs the other's results, and the workgroups of one fill the compute units that those of the other leave idle at its end.  Keys
// and values first, whose workgroups take longer.
template <typename T, int DP, int WM, int WN, bool VEC> __global__ __launch_bounds__(ATT_THREADS, (AttDkv<T, DP, WN>::MIN_WAVES)) void k_attend_back(const AttArgs a)
{
    if ((int)blockIdx.x < a.kv_blocks) attend_dkv<T, DP, WN, VEC>(a, blockIdx.x, a.kv_blocks);
    else attend_dq<T, DP, WM, VEC>(a, blockIdx.x - a.kv_blocks, gridDim.x - a.kv_blocks);
}

// Adds up the parts of split gradients, part by part: workgroups below `q_blocks` those of dQ (q_splits parts), the others those of dK and dV.  A wave takes
// a row of D elements.
template <typename T> __global__ __launch_bounds__(ATT_THREADS) void k_attend_sum(const AttArgs a, int q_blocks, int q_splits, int kv_splits)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool of_q = (int)blockIdx.x < q_blocks;
    const long long i = (long long)((int)blockIdx.x - (of_q ? 0 : q_blocks)) * ATT_WAVES + wave, n = of_q ? (long long)a.n_q * a.Hq : 2ll * a.n_kv * a.Hk;
    if (i >= n) return;
    const float *from = (of_q ? a.part_q : a.part_kv) + i * a.D;
    T *to;
    bool dead = false;
    if (of_q) {
        const long long row = divide(i, a.Hq);
        to = row_of<T>(a.d_q, row, (int)(i - row * a.Hq));
    } else {
        const long long node = divide(i / 2, a.Hk);
        dead = a.mask && !a.mask[node];         // (its parts were not written)
        to = row_of<T>(i & 1 ? a.d_v : a.d_k, node, (int)(i / 2 - node * a.Hk));
    }
    const int parts = of_q ? q_splits : kv_splits;
    for (int d = lane; d < a.D; d += 64) {
        float x = 0.f;
        if (!dead)
            for (int p = 0; p < parts; ++p) x += from[p * n * a.D + d];
        to[d] = (T)x;
    }
}

}  // namespace tl
