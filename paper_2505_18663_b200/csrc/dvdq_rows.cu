// C ABI (see include/dvdq.h) of the operators on rows that feed the 8-bit linear layer: RMS norm with the residual's addition,
// quantization of rows (rms_norm.cuh).  Argument validation, launches.
#include <math.h>

#include "rms_norm.cuh"

namespace dvdq {

template <bool NORM>
static dvdq_status rms_run(const RmsArgs& A, int32_t dtype, int access, cudaStream_t st) {
    return cuda_status(dtype == DVDQ_BF16  ? launch_rms_t<__nv_bfloat16, NORM>(A, access, st)
                       : dtype == DVDQ_F16 ? launch_rms_t<__half, NORM>(A, access, st)
                                           : launch_rms_t<float, NORM>(A, access, st));
}

}  // namespace dvdq

using namespace dvdq;

extern "C" {

dvdq_status dvdq_rms_norm(const void* X, int64_t x_outer, int64_t x_row, const void* R, int64_t r_outer, int64_t r_row, int64_t N, int64_t S,
                          int64_t C, const void* gamma, int32_t param_dtype, float eps, void* H, int64_t h_outer, int64_t h_row, void* Y,
                          int64_t y_outer, int64_t y_row, int8_t* codes, int64_t c_outer, int64_t c_row, float* scales, float* rstd_out,
                          int32_t dtype, void* stream) {
    if (!rows_sizes_ok(N, S, C) || !(eps >= 0.0f) || !isfinite(eps)) return DVDQ_ERR_SHAPE;
    if (!rows_dtype_ok(dtype) || (param_dtype != dtype && param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    if (N == 0 || S == 0) return DVDQ_OK;
    if (!X || (!H && !Y && !codes && !rstd_out) || (codes == nullptr) != (scales == nullptr)) return DVDQ_ERR_NULL;
    const int bytes = dtype_bytes(dtype), pb = dtype_bytes(param_dtype);
    RmsArgs A = {};
    A.x = RowsOf{const_cast<void*>(X), x_outer, x_row};
    A.r = RowsOf{const_cast<void*>(R), r_outer, r_row};
    A.h = RowsOf{H, h_outer, h_row};
    A.y = RowsOf{Y, y_outer, y_row};
    A.codes = RowsOf{codes, c_outer, c_row};
    dvdq_status s;
    if ((s = check_rows(&A.x, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.r, N, S, C, bytes, false)) != DVDQ_OK ||
        (s = check_rows(&A.h, N, S, C, bytes, true)) != DVDQ_OK || (s = check_rows(&A.y, N, S, C, bytes, true)) != DVDQ_OK ||
        (s = check_rows(&A.codes, N, S, C, 1, true)) != DVDQ_OK)
        return s;
    if (!in_place_ok(A.x, A.h) || !in_place_ok(A.r, A.h) || !in_place_ok(A.x, A.y) || !in_place_ok(A.r, A.y) || (H && H == Y)) return DVDQ_ERR_SHAPE;
    if ((gamma && !aligned_to(gamma, pb)) || (scales && !aligned_to(scales, 4)) || (rstd_out && !aligned_to(rstd_out, 4))) return DVDQ_ERR_ALIGN;
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    A.shape = rows_shape(N, S, C);
    A.gamma = gamma;
    A.scales = scales;
    A.rstd = rstd_out;
    A.params_f32 = param_dtype == DVDQ_F32;
    A.eps = eps;
    A.inv_c = 1.0f / (float)C;
    const RowsOf* all[] = {&A.x, &A.r, &A.h, &A.y};
    return rms_run<true>(A, dtype, rows_access(all, 4, &A.codes, gamma, bytes, pb), (cudaStream_t)stream);
}

dvdq_status dvdq_quantize_rows(const void* X, int64_t M, int64_t K, int64_t ldx, int8_t* codes, int64_t ldc, float* scales, int32_t dtype,
                               void* stream) {
    if (!rows_sizes_ok(1, M, K)) return DVDQ_ERR_SHAPE;
    if (!rows_dtype_ok(dtype)) return DVDQ_ERR_UNSUPPORTED;
    if (M == 0) return DVDQ_OK;
    if (!X || !codes || !scales) return DVDQ_ERR_NULL;
    const int bytes = dtype_bytes(dtype);
    RmsArgs A = {};
    A.x = RowsOf{const_cast<void*>(X), 0, ldx};
    A.codes = RowsOf{codes, 0, ldc};
    dvdq_status s;
    if ((s = check_rows(&A.x, 1, M, K, bytes, false)) != DVDQ_OK || (s = check_rows(&A.codes, 1, M, K, 1, true)) != DVDQ_OK) return s;
    if (!aligned_to(scales, 4)) return DVDQ_ERR_ALIGN;
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    A.shape = rows_shape(1, M, K);
    A.scales = scales;
    const RowsOf* all[] = {&A.x};
    return rms_run<false>(A, dtype, rows_access(all, 1, &A.codes, nullptr, bytes, 0), (cudaStream_t)stream);
}

}  // extern "C"
