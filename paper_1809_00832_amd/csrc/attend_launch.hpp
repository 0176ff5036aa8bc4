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
};

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
    a.slots = (int)((long long)a.n_q * a.G / Q::BM + a.n_trees);
    a.splits = p.q_splits;
    a.bufs = p.q_bufs;
    a.kv_slots = a.n_kv / KV::BN + a.n_trees;
    a.kv_splits = p.kv_splits;
    a.kv_bufs = p.kv_bufs;
    // (a multiple of eight, so that consecutive workgroups of both kinds lie in one L2 domain)
    a.kv_blocks = a.n_kv > 0 ? (int)(((long long)a.kv_slots * a.kv_splits * a.Hk + 7) & ~7ll) : 0;
    const long long q_blocks = a.n_q > 0 ? (long long)a.slots * a.splits * a.Hk : 0;
    const size_t lds_q = Q::lds(a.bufs), lds_kv = KV::lds(a.kv_bufs), most_q = Q::lds(2), most_kv = KV::lds(2);
    return att_launch<k_attend_back<T, DP, Q::WM, KV::WN, VEC>>(a.kv_blocks + q_blocks, lds_q > lds_kv ? lds_q : lds_kv, most_q > most_kv ? most_q : most_kv, a, st);
}

template <typename T, int DP, bool VEC> hipError_t att_backward_of(const AttArgs &a, const AttBackPlan &p, hipStream_t st)
{
    hipError_t e = hipSuccess;
    const long long row_blocks = ((long long)a.n_q * a.Hq + 15) / 16;
    if (row_blocks + (a.mask ? a.n_trees : 0) > 0) {
        hipLaunchKernelGGL(k_attend_prepare<T>, dim3((unsigned)(row_blocks + (a.mask ? a.n_trees : 0))), dim3(ATT_THREADS), 0, st, a, (int)row_blocks);
        e = hipGetLastError();
    }
    if (e == hipSuccess && (a.n_q > 0 || a.n_kv > 0))
        e = p.q_waves == 2 ? (p.kv_waves == 2 ? att_both_of<T, DP, 2, 2, VEC>(a, p, st) : att_both_of<T, DP, 2, 4, VEC>(a, p, st))
                           : (p.kv_waves == 2 ? att_both_of<T, DP, 4, 2, VEC>(a, p, st) : att_both_of<T, DP, 4, 4, VEC>(a, p, st));
    if (e == hipSuccess && (p.q_splits > 1 || p.kv_splits > 1)) {
        const long long q_blocks = p.q_splits > 1 ? ((long long)a.n_q * a.Hq + ATT_WAVES - 1) / ATT_WAVES : 0;
        const long long kv_blocks = p.kv_splits > 1 ? (2ll * a.n_kv * a.Hk + ATT_WAVES - 1) / ATT_WAVES : 0;
        hipLaunchKernelGGL(k_attend_sum<T>, dim3((unsigned)(q_blocks + kv_blocks)), dim3(ATT_THREADS), 0, st, a, (int)q_blocks, p.q_splits, p.kv_splits);
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
