// C ABI (see include/dvdq.h) of the operators on rows that feed the 8-bit linear layer: RMS norm with the residual's addition
// (rms_norm.cuh), its gradients (rms_norm_backward.cuh), quantization of rows.  Argument validation, size queries, launches.
#include <math.h>

#include "rms_norm.cuh"
#include "rms_norm_backward.cuh"

namespace dvdq {

// dvdq_rows_{bf16,f16,f32}.cu
cudaError_t launch_rms_norm_bf16(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_rms_norm_f16(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_rms_norm_f32(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_quantize_rows_bf16(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_quantize_rows_f16(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_quantize_rows_f32(const RmsArgs& A, int access, cudaStream_t st);
cudaError_t launch_rms_norm_backward_bf16(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st);
cudaError_t launch_rms_norm_backward_f16(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st);
cudaError_t launch_rms_norm_backward_f32(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st);

}  // namespace dvdq

using namespace dvdq;

extern "C" {

dvdq_status dvdq_rms_norm(const dvdq_rms_norm_args* args, void* stream) {
    if (!args) return DVDQ_ERR_NULL;
    const dvdq_rms_norm_args& a = *args;
    const int64_t N = a.N, S = a.S, C = a.C;
    if (!rows_sizes_ok(N, S, C) || !(a.eps >= 0.0f) || !isfinite(a.eps)) return DVDQ_ERR_SHAPE;
    if (!rows_dtype_ok(a.dtype) || (a.param_dtype != a.dtype && a.param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    if (N == 0 || S == 0) return DVDQ_OK;
    if (!a.X || (!a.H && !a.Y && !a.codes && !a.rstd_out) || (a.codes == nullptr) != (a.scales == nullptr)) return DVDQ_ERR_NULL;
    const int bytes = dtype_bytes(a.dtype), pb = dtype_bytes(a.param_dtype);
    RmsArgs A = {};
    A.x = RowsOf{const_cast<void*>(a.X), a.x_outer, a.x_row};
    A.r = RowsOf{const_cast<void*>(a.R), a.r_outer, a.r_row};
    A.h = RowsOf{a.H, a.h_outer, a.h_row};
    A.y = RowsOf{a.Y, a.y_outer, a.y_row};
    A.codes = RowsOf{a.codes, a.c_outer, a.c_row};
    dvdq_status s;
    if ((s = check_rows(&A.x, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.r, N, S, C, bytes, false)) != DVDQ_OK ||
        (s = check_rows(&A.h, N, S, C, bytes, true)) != DVDQ_OK || (s = check_rows(&A.y, N, S, C, bytes, true)) != DVDQ_OK ||
        (s = check_rows(&A.codes, N, S, C, 1, true)) != DVDQ_OK)
        return s;
    if (!in_place_ok(A.x, A.h) || !in_place_ok(A.r, A.h) || !in_place_ok(A.x, A.y) || !in_place_ok(A.r, A.y) || (a.H && a.H == a.Y)) return DVDQ_ERR_SHAPE;
    if ((a.gamma && !aligned_to(a.gamma, pb)) || (a.scales && !aligned_to(a.scales, 4)) || (a.rstd_out && !aligned_to(a.rstd_out, 4))) return DVDQ_ERR_ALIGN;
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    A.shape = rows_shape(N, S, C);
    A.gamma = a.gamma;
    A.scales = a.scales;
    A.rstd = a.rstd_out;
    A.params_f32 = a.param_dtype == DVDQ_F32;
    A.eps = a.eps;
    A.inv_c = 1.0f / (float)C;
    const RowsOf* all[] = {&A.x, &A.r, &A.h, &A.y};
    const int access = rows_access(all, 4, &A.codes, a.gamma, bytes, pb);
    const cudaStream_t st = (cudaStream_t)stream;
    return cuda_status(a.dtype == DVDQ_BF16  ? launch_rms_norm_bf16(A, access, st)
                       : a.dtype == DVDQ_F16 ? launch_rms_norm_f16(A, access, st)
                                             : launch_rms_norm_f32(A, access, st));
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
    const int access = rows_access(all, 1, &A.codes, nullptr, bytes, 0);
    const cudaStream_t st = (cudaStream_t)stream;
    return cuda_status(dtype == DVDQ_BF16  ? launch_quantize_rows_bf16(A, access, st)
                       : dtype == DVDQ_F16 ? launch_quantize_rows_f16(A, access, st)
                                           : launch_quantize_rows_f32(A, access, st));
}

size_t dvdq_rms_norm_backward_workspace_bytes(int64_t N, int64_t S, int64_t C) {
    if (!rows_sizes_ok(N, S, C) || N == 0 || S == 0) return 0;
    return (size_t)align_up(rms_parts(N * S, C) * C * 4, 256);
}

dvdq_status dvdq_rms_norm_backward(const dvdq_rms_norm_backward_args* args, void* stream) {
    if (!args) return DVDQ_ERR_NULL;
    const dvdq_rms_norm_backward_args& a = *args;
    const int64_t N = a.N, S = a.S, C = a.C;
    const int32_t dtype = a.dtype, param_dtype = a.param_dtype;
    const void* gamma = a.gamma;
    float* dgamma = a.dgamma;
    if (!rows_sizes_ok(N, S, C)) return DVDQ_ERR_SHAPE;
    if (!rows_dtype_ok(dtype) || (param_dtype != dtype && param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    const int bytes = dtype_bytes(dtype), pb = dtype_bytes(param_dtype);
    if ((gamma && !aligned_to(gamma, pb)) || (dgamma && !aligned_to(dgamma, 4)) || (a.rstd && !aligned_to(a.rstd, 4))) return DVDQ_ERR_ALIGN;
    dvdq_status s;
    const cudaStream_t st = (cudaStream_t)stream;
    if (N == 0 || S == 0) {  // sums over nothing
        if (!dgamma) return DVDQ_OK;
        if ((s = check_device_arch()) != DVDQ_OK) return s;
        return cuda_status(launch_after(rms_norm_no_rows_kernel, dim3((unsigned)ceil_div(C, 256)), dim3(256), 0, st, dgamma, (int)C));
    }
    if (!a.dY || !a.H || !a.rstd || (!a.dX && !dgamma)) return DVDQ_ERR_NULL;
    RmsBackwardArgs A = {};
    A.dy = RowsOf{const_cast<void*>(a.dY), a.dy_outer, a.dy_row};
    A.h = RowsOf{const_cast<void*>(a.H), a.h_outer, a.h_row};
    A.dh = RowsOf{const_cast<void*>(a.dH), a.dh_outer, a.dh_row};
    A.dx = RowsOf{a.dX, a.dx_outer, a.dx_row};
    if ((s = check_rows(&A.dy, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.h, N, S, C, bytes, false)) != DVDQ_OK ||
        (s = check_rows(&A.dh, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.dx, N, S, C, bytes, true)) != DVDQ_OK)
        return s;
    if (!in_place_ok(A.dy, A.dx) || !in_place_ok(A.h, A.dx) || !in_place_ok(A.dh, A.dx)) return DVDQ_ERR_SHAPE;
    const int64_t parts = rms_parts(N * S, C);
    if (dgamma) {
        if (!a.workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(a.workspace, 256)) return DVDQ_ERR_ALIGN;
        if (a.workspace_bytes < (uint64_t)(parts * C * 4)) return DVDQ_ERR_WORKSPACE;
    }
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    A.shape = rows_shape(N, S, C);
    A.gamma = gamma;
    A.rstd = a.rstd;
    A.part = dgamma ? static_cast<float*>(a.workspace) : nullptr;
    A.dgamma = dgamma;
    A.params_f32 = param_dtype == DVDQ_F32;
    A.inv_c = 1.0f / (float)C;
    const RowsOf* all[] = {&A.dy, &A.h, &A.dh, &A.dx};
    const int access = rows_access(all, 4, nullptr, gamma, bytes, pb);
    int ctas = 0;
    const cudaError_t e = dtype == DVDQ_BF16  ? launch_rms_norm_backward_bf16(A, access, parts, &ctas, st)
                          : dtype == DVDQ_F16 ? launch_rms_norm_backward_f16(A, access, parts, &ctas, st)
                                              : launch_rms_norm_backward_f32(A, access, parts, &ctas, st);
    if (e != cudaSuccess || !dgamma || ctas == 0) return cuda_status(e);  // no sums to add
    return cuda_status(launch_rms_join(A.part, ctas, (int)C, dgamma, st));
}

}  // extern "C"
