// Launches of the attention kernels for one element type; attend_f32.hip, attend_bf16.hip and attend_f16.hip hold one type each.
#pragma once

#include "attend.hpp"

namespace tl {

// Head dimensions are padded to one of these (zeros in LDS and registers, never in memory).
constexpr int att_padded(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// What a forward call will do: decided from sizes alone, by the workspace query and by the call alike.
struct AttPlan {
    int wm;                 // waves along the rows (AttFwd)
    int bm, bn;             // packed rows and nodes of a workgroup's tile
    int slots, splits;
    int bufs;               // stages in LDS
};

// ... and a backward call: waves side by side along the rows (AttDq) and the nodes (AttDkv), parts that a tree's nodes and its rows are cut into.
struct AttBackPlan {
    int q_waves, kv_waves;
    int q_splits, kv_splits;
    int q_bufs, kv_bufs;
    int q_slots, kv_slots;          // row tiles and node tiles (see find_slot)
    int q_blocks, kv_blocks;        // workgroups of each kind, a multiple of eight of the latter
    int prepare_blocks, sum_blocks_q, sum_blocks_kv;
};

// A launch has fewer than 2^32 threads in all.
constexpr long long ATT_MOST_BLOCKS = (1ll << 32) / ATT_THREADS - 1;

// Packed rows of AttDq's tile and nodes of AttDkv's.
constexpr int att_dq_rows(int dp, int waves) { return 32 * (dp > 128 ? 2 : waves); }
constexpr int att_dkv_nodes(int dp, int size, int waves) { return 32 * (dp <= 128 ? waves : size == 2 ? 2 : 1); }

template <typename T> hipError_t attend_forward(const AttArgs &a, const AttPlan &p, hipStream_t st);
template <typename T> hipError_t attend_backward(const AttArgs &a, const AttBackPlan &p, hipStream_t st);

// Allows a kernel its dynamic LDS, once per kernel and device (the call takes about as long as a launch).
template <auto KERNEL> hipError_t att_allow(size_t lds)
{
    static unsigned long long allowed;                          // devices
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (__atomic_load_n(&allowed, __ATOMIC_RELAXED) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e == hipSuccess) __atomic_fetch_or(&allowed, bit, __ATOMIC_RELAXED);
    return e;
}

template <auto KERNEL> hipError_t att_launch(long long blocks, size_t lds, size_t most_lds, const AttArgs &a, hipStream_t st)
{
    const hipError_t e = att_allow<KERNEL>(most_lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(KERNEL, dim3((unsigned)blocks), dim3(ATT_THREADS), lds, st, a);
    return hipGetLastError();
}

template <typename T, int DP, int WM> hipError_t att_forward_of(const AttArgs &a, hipStream_t st)
{
    typedef AttFwd<T, DP, WM> C;
    const long long blocks = (long long)a.slots * a.splits * a.Hk;
    const size_t lds = C::lds(a.bufs < C::MAX_BUFS ? a.bufs : C::MAX_BUFS, a.mask), most = C::lds(C::MAX_BUFS, true);
    return a.vec ? att_launch<k_attend<T, DP, WM, true>>(blocks, lds, most, a, st) : att_launch<k_attend<T, DP, WM, false>>(blocks, lds, most, a, st);
}

template <typename T, int DP> hipError_t att_forward_at(const AttArgs &a, const AttPlan &p, hipStream_t st)
{
    if constexpr (DP * sizeof(T) <= 512)                        // (one stage of four waves' nodes has to fit the LDS)
        if (p.wm == 1) return att_forward_of<T, DP, 1>(a, st);
    if (p.wm == 2) return att_forward_of<T, DP, 2>(a, st);
    return att_forward_of<T, DP, 4>(a, st);
}

template <typename T, int DP, int WM, int WN, bool VEC> hipError_t att_both_of(AttArgs a, const AttBackPlan &p, hipStream_t st)
{
    typedef AttDq<T, DP, WM> Q;
    typedef AttDkv<T, DP, WN> KV;
    static_assert(Q::BM == att_dq_rows(DP, WM) && KV::BN == att_dkv_nodes(DP, sizeof(T), WN), "the plan's tiles");
    a.slots = p.q_slots;
    a.splits = p.q_splits;
    a.bufs = p.q_bufs;
    a.kv_slots = p.kv_slots;
    a.kv_splits = p.kv_splits;
    a.kv_bufs = p.kv_bufs;
    a.kv_blocks = p.kv_blocks;
    const size_t lds_q = Q::lds(a.bufs), lds_kv = KV::lds(a.kv_bufs), most_q = Q::lds(2), most_kv = KV::lds(2);
    return att_launch<k_attend_back<T, DP, Q::WM, KV::WN, VEC>>((long long)p.kv_blocks + p.q_blocks, lds_q > lds_kv ? lds_q : lds_kv, most_q > most_kv ? most_q : most_kv, a, st);
}

template <typename T, int DP, bool VEC> hipError_t att_backward_of(const AttArgs &a, const AttBackPlan &p, hipStream_t st)
{
    hipError_t e = hipSuccess;
    if (p.prepare_blocks > 0) {
        const int row_blocks = p.prepare_blocks - (a.mask ? a.n_trees : 0);
        hipLaunchKernelGGL(k_attend_prepare<T>, dim3(p.prepare_blocks), dim3(ATT_THREADS), 0, st, a, row_blocks);
        e = hipGetLastError();
    }
    if (e == hipSuccess && (a.n_q > 0 || a.n_kv > 0))
        e = p.q_waves == 2 ? (p.kv_waves == 2 ? att_both_of<T, DP, 2, 2, VEC>(a, p, st) : att_both_of<T, DP, 2, 4, VEC>(a, p, st))
                           : (p.kv_waves == 2 ? att_both_of<T, DP, 4, 2, VEC>(a, p, st) : att_both_of<T, DP, 4, 4, VEC>(a, p, st));
    if (e == hipSuccess && p.sum_blocks_q + p.sum_blocks_kv > 0) {
        hipLaunchKernelGGL(k_attend_sum<T>, dim3(p.sum_blocks_q + p.sum_blocks_kv), dim3(ATT_THREADS), 0, st, a, p.sum_blocks_q, p.q_splits, p.kv_splits);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, int DP> hipError_t att_backward_at(const AttArgs &a, const AttBackPlan &p, hipStream_t st)
{
    return a.vec ? att_backward_of<T, DP, true>(a, p, st) : att_backward_of<T, DP, false>(a, p, st);
}

#define ATT_INSTANCES(T)                                                                                                       \
    template <> hipError_t attend_forward<T>(const AttArgs &a, const AttPlan &p, hipStream_t st)                               \
    {                                                                                                                          \
        hipError_t e;                                                                                                          \
        switch (att_padded(a.D)) {                                                                                             \
        case 32: e = att_forward_at<T, 32>(a, p, st); break;                                                                   \
        case 64: e = att_forward_at<T, 64>(a, p, st); break;                                                                   \
        case 128: e = att_forward_at<T, 128>(a, p, st); break;                                                                 \
        default: e = att_forward_at<T, 256>(a, p, st);                                                                         \
        }                                                                                                                      \
        if (e != hipSuccess || a.splits == 1) return e;                                                                        \
        hipLaunchKernelGGL(k_attend_join<T>, dim3((unsigned)((long long)a.n_q * a.Hq)), dim3(ATT_THREADS), 0, st, a, p.bn);    \
        return hipGetLastError();                                                                                              \
    }                                                                                                                          \
    template <> hipError_t attend_backward<T>(const AttArgs &a, const AttBackPlan &p, hipStream_t st)                          \
    {                                                                                                                          \
        switch (att_padded(a.D)) {                                                                                             \
        case 32: return att_backward_at<T, 32>(a, p, st);                                                                      \
        case 64: return att_backward_at<T, 64>(a, p, st);                                                                      \
        case 128: return att_backward_at<T, 128>(a, p, st);                                                                    \
        default: return att_backward_at<T, 256>(a, p, st);                                                                     \
        }                                                                                                                      \
    }

}  // namespace tl
