// C ABI (see include/dvdq.h) of the operators on rows that feed the 8-bit linear layer: RMS norm with the residual's addition and
// its gradients, quantization of rows (rms_norm.cuh).  Argument validation, size queries, launches.
#include <math.h>

#include "rms_norm.cuh"

namespace dvdq {

static bool rows_dtype_ok(int32_t t) { return t == DVDQ_BF16 || t == DVDQ_F16 || t == DVDQ_F32; }
static bool rows_sizes_ok(int64_t N, int64_t S, int64_t C) {
    const int64_t most = 0x7FFFFFFFll;
    return N >= 0 && S >= 0 && N <= most && S <= most && N * S <= most && C > 0 && C <= (1 << 20);
}

// A [N, S, C] tensor's pitches; those of an extent of one are not read.
static dvdq_status check_rows(RowsOf* t, int64_t N, int64_t S, int64_t C, int bytes, bool written) {
    if (!t->p) return DVDQ_OK;
    if (N == 1) t->outer = 0;
    if (S == 1) t->row = 0;
    if (t->outer < 0 || t->row < 0) return DVDQ_ERR_SHAPE;
    if (written && ((S > 1 && t->row < C) || (N > 1 && t->outer < C))) return DVDQ_ERR_SHAPE;  // outputs may not overlap
    return aligned_to(t->p, bytes) ? DVDQ_OK : DVDQ_ERR_ALIGN;
}
// An output over the tensor that it is made from lies exactly over it (after check_rows).
static bool in_place_ok(const RowsOf& from, const RowsOf& to) { return !to.p || from.p != to.p || (from.outer == to.outer && from.row == to.row); }

// The widest piece, in bytes of the tensors' type, that all of them and gamma allow.
static bool piece_ok(const RowsOf& t, int bytes, int piece) {
    return aligned_to(t.p, piece) && (t.outer * bytes) % piece == 0 && (t.row * bytes) % piece == 0;
}
static int rows_access(const RowsOf* const* tensors, int count, const RowsOf* codes, const void* gamma, int bytes, int param_bytes) {
    for (int piece = 16; piece > bytes; piece /= 4) {
        if (piece == 4 && bytes == 4) break;
        const int v = piece / bytes, of_gamma = v * param_bytes < 16 ? v * param_bytes : 16;
        bool ok = !gamma || aligned_to(gamma, of_gamma);
        for (int i = 0; i < count; ++i) ok = ok && (!tensors[i]->p || piece_ok(*tensors[i], bytes, piece));
        if (ok && (!codes || !codes->p || piece_ok(*codes, 1, v))) return piece;
    }
    return bytes;
}
static RowsShape rows_shape(int64_t N, int64_t S, int64_t C) {
    RowsShape r;
    r.rows = N * S;
    r.by_s = FastDiv((uint32_t)S);
    r.S = (int)S;
    r.C = (int)C;
    return r;
}

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

size_t dvdq_rms_norm_backward_workspace_bytes(int64_t N, int64_t S, int64_t C) {
    if (!rows_sizes_ok(N, S, C) || N == 0 || S == 0) return 0;
    return (size_t)align_up(rms_parts(N * S, C) * C * 4, 256);
}

dvdq_status dvdq_rms_norm_backward(const void* dY, int64_t dy_outer, int64_t dy_row, const void* H, int64_t h_outer, int64_t h_row,
                                   const float* rstd, const void* dH, int64_t dh_outer, int64_t dh_row, int64_t N, int64_t S, int64_t C,
                                   const void* gamma, int32_t param_dtype, void* dX, int64_t dx_outer, int64_t dx_row, float* dgamma,
                                   int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!rows_sizes_ok(N, S, C)) return DVDQ_ERR_SHAPE;
    if (!rows_dtype_ok(dtype) || (param_dtype != dtype && param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    const int bytes = dtype_bytes(dtype), pb = dtype_bytes(param_dtype);
    if ((gamma && !aligned_to(gamma, pb)) || (dgamma && !aligned_to(dgamma, 4)) || (rstd && !aligned_to(rstd, 4))) return DVDQ_ERR_ALIGN;
    dvdq_status s;
    const cudaStream_t st = (cudaStream_t)stream;
    if (N == 0 || S == 0) {  // sums over nothing
        if (!dgamma) return DVDQ_OK;
        if ((s = check_device_arch()) != DVDQ_OK) return s;
        return cuda_status(launch_after(rms_norm_no_rows_kernel, dim3((unsigned)ceil_div(C, 256)), dim3(256), 0, st, dgamma, (int)C));
    }
    if (!dY || !H || !rstd || (!dX && !dgamma)) return DVDQ_ERR_NULL;
    RmsBackwardArgs A = {};
    A.dy = RowsOf{const_cast<void*>(dY), dy_outer, dy_row};
    A.h = RowsOf{const_cast<void*>(H), h_outer, h_row};
    A.dh = RowsOf{const_cast<void*>(dH), dh_outer, dh_row};
    A.dx = RowsOf{dX, dx_outer, dx_row};
    if ((s = check_rows(&A.dy, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.h, N, S, C, bytes, false)) != DVDQ_OK ||
        (s = check_rows(&A.dh, N, S, C, bytes, false)) != DVDQ_OK || (s = check_rows(&A.dx, N, S, C, bytes, true)) != DVDQ_OK)
        return s;
    if (!in_place_ok(A.dy, A.dx) || !in_place_ok(A.h, A.dx) || !in_place_ok(A.dh, A.dx)) return DVDQ_ERR_SHAPE;
    const int64_t parts = rms_parts(N * S, C);
    if (dgamma) {
        if (!workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(workspace, 256)) return DVDQ_ERR_ALIGN;
        if (workspace_bytes < (size_t)(parts * C * 4)) return DVDQ_ERR_WORKSPACE;
    }
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    A.shape = rows_shape(N, S, C);
    A.gamma = gamma;
    A.rstd = rstd;
    A.part = dgamma ? static_cast<float*>(workspace) : nullptr;
    A.params_f32 = param_dtype == DVDQ_F32;
    A.inv_c = 1.0f / (float)C;
    const RowsOf* all[] = {&A.dy, &A.h, &A.dh, &A.dx};
    const int access = rows_access(all, 4, nullptr, gamma, bytes, pb);
    int ctas = 0;
    const cudaError_t e = dtype == DVDQ_BF16  ? launch_rms_backward_t<__nv_bfloat16>(A, access, parts, &ctas, st)
                          : dtype == DVDQ_F16 ? launch_rms_backward_t<__half>(A, access, parts, &ctas, st)
                                              : launch_rms_backward_t<float>(A, access, parts, &ctas, st);
    if (e != cudaSuccess || !dgamma) return cuda_status(e);
    return cuda_status(launch_after(rms_norm_join_kernel, dim3((unsigned)ceil_div(C, 32)), dim3(kRmsJoinWarps * 32), 0, st, A.part, ctas, (int)C, dgamma));
}

}  // extern "C"
