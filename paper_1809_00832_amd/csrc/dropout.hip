// C entry point of dropout.
#include <math.h>

#include "dropout.hpp"
#include "entry.hpp"

using namespace tl;

namespace {

template <typename T, bool ONCE> void start(const DropArgs &a, dim3 grid, hipStream_t st)
{
    if (a.residual) hipLaunchKernelGGL((k_dropout<T, true, ONCE>), grid, dim3(DRO_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_dropout<T, false, ONCE>), grid, dim3(DRO_THREADS), 0, st, a);
}

template <typename T> hipError_t launch(DropArgs a, long long rows, hipStream_t st)
{
    // Inputs that are larger than the caches keep (256 MB hold them and what is written) are read past them.  Measured (us, kept / past, two calls, of which
    // one has a residual): 65536 x 1024 bf16 133 / 109, 32768 x 1024 fp32 130 / 120; 8192 x 1024 bf16 20 either way.
    const bool once = (double)rows * a.cols * sizeof(T) > 1e8;
    // whole rows per launch, of fewer than 2^32 threads
    const long long most = ((1ll << 32) - 2 * DRO_THREADS) / a.blocks;
    for (; a.first < rows; a.first = a.end) {
        a.end = a.first + most < rows ? a.first + most : rows;
        const dim3 grid((unsigned)(((a.end - a.first) * a.blocks + DRO_THREADS - 1) / DRO_THREADS));
        if (once) start<T, true>(a, grid, st);
        else start<T, false>(a, grid, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

extern "C" {

int tl_dropout(int dtype, int n_rows, int n_cols, const void *x, int64_t x_row, const void *residual, int64_t residual_row, void *y, int64_t y_row, float p,
               const uint64_t *numbers, void *hip_stream)
{
    if (!is_dtype(dtype) || n_rows < 0 || n_cols < 1 || n_cols > (1 << 30) || !(p >= 0.f && p <= 1.f)) return TL_EINVAL;
    if (n_rows == 0) return TL_OK;
    if (!check_matrix(x, x_row, dtype, n_rows, n_cols, false) || !check_matrix(y, y_row, dtype, n_rows, n_cols, true)) return TL_EINVAL;
    if (residual && !check_matrix(residual, residual_row, dtype, n_rows, n_cols, false)) return TL_EINVAL;
    if (!numbers || ((uintptr_t)numbers & 7)) return TL_EINVAL;
    if (n_rows > 1 && ((y == x && y_row != x_row) || (y == residual && y_row != residual_row))) return TL_EINVAL;
    DropArgs a = {};
    a.x = x;
    a.x_row = x_row;
    a.residual = residual;
    a.r_row = residual_row;
    a.y = y;
    a.y_row = y_row;
    a.numbers = numbers;
    a.cols = n_cols;
    a.blocks = (n_cols + 7) / 8;
    a.t = (uint32_t)rintf(p * 65536.f);
    a.scale = a.t < 65536 ? 65536.f / (float)(65536 - a.t) : 0.f;
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = dtype == TL_DT_F32 ? launch<float>(a, n_rows, st) : dtype == TL_DT_BF16 ? launch<bf16_t>(a, n_rows, st) : launch<f16_t>(a, n_rows, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

}  // extern "C"
