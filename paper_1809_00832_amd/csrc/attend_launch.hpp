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
};

template <typename T> hipError_t attend_forward(const AttArgs &a, const AttPlan &p, hipStream_t st);
template <typename T> hipError_t attend_backward(const AttArgs &a, hipStream_t st);

template <typename K> hipError_t att_launch(K kernel, long long blocks, int threads, size_t lds, const AttArgs &a, hipStream_t st)
{
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), lds, st, a);
    return hipGetLastError();
}

template <typename T, int DP, int WM> hipError_t att_forward_of(const AttArgs &a, hipStream_t st)
{
    typedef AttFwd<T, DP, WM> C;
    const long long blocks = (long long)a.slots * a.splits * a.Hk;
    return a.vec ? att_launch(k_attend<T, DP, WM, true>, blocks, C::THREADS, C::LDS, a, st) : att_launch(k_attend<T, DP, WM, false>, blocks, C::THREADS, C::LDS, a, st);
}

template <typename T, int DP> hipError_t att_forward_at(const AttArgs &a, const AttPlan &p, hipStream_t st)
{
    if constexpr (DP * sizeof(T) <= 512)                        // (one stage of four waves' nodes has to fit the LDS)
        if (p.wm == 1) return att_forward_of<T, DP, 1>(a, st);
    if (p.wm == 2) return att_forward_of<T, DP, 2>(a, st);
    return att_forward_of<T, DP, 4>(a, st);
}

template <typename T, int DP, bool VEC> hipError_t att_backward_of(AttArgs a, hipStream_t st)
{
    const long long rows = (long long)a.n_q * a.G, row_blocks = ((long long)a.n_q * a.Hq + 15) / 16;
    if (row_blocks + (a.mask ? a.n_trees : 0) > 0) {
        hipLaunchKernelGGL(k_attend_prepare<T>, dim3((unsigned)(row_blocks + (a.mask ? a.n_trees : 0))), dim3(ATT_THREADS), 0, st, a, (int)row_blocks);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.n_q > 0) {
        a.slots = (int)(rows / AttDq<T, DP>::BM + a.n_trees);
        const hipError_t e = att_launch(k_attend_dq<T, DP, VEC>, (long long)a.slots * a.Hk, ATT_THREADS, AttDq<T, DP>::LDS, a, st);
        if (e != hipSuccess) return e;
    }
    if (a.n_kv > 0) {
        a.slots = a.n_kv / AttDkv<T, DP>::BN + a.n_trees;
        return att_launch(k_attend_dkv<T, DP, VEC>, (long long)a.slots * a.Hk, ATT_THREADS, AttDkv<T, DP>::LDS, a, st);
    }
    return hipSuccess;
}

template <typename T, int DP> hipError_t att_backward_at(const AttArgs &a, hipStream_t st)
{
    return a.vec ? att_backward_of<T, DP, true>(a, st) : att_backward_of<T, DP, false>(a, st);
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
        const long long rh = (long long)a.n_q * a.Hq;                                                                          \
        hipLaunchKernelGGL(k_attend_join<T>, dim3((unsigned)((rh + ATT_WAVES - 1) / ATT_WAVES)), dim3(ATT_THREADS), 0, st, a,  \
                           p.bn);                                                                                              \
        return hipGetLastError();                                                                                              \
    }                                                                                                                          \
    template <> hipError_t attend_backward<T>(const AttArgs &a, hipStream_t st)                                                \
    {                                                                                                                          \
        switch (att_padded(a.D)) {                                                                                             \
        case 32: return att_backward_at<T, 32>(a, st);                                                                         \
        case 64: return att_backward_at<T, 64>(a, st);                                                                         \
        case 128: return att_backward_at<T, 128>(a, st);                                                                       \
        default: return att_backward_at<T, 256>(a, st);                                                                        \
        }                                                                                                                      \
    }

}  // namespace tl
