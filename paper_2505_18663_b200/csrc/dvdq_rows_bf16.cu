// The kernels on rows (rms_norm.cuh, rms_norm_backward.cuh) for one element type: a translation unit of its own, to be compiled beside the others.
#include "rms_norm.cuh"
#include "rms_norm_backward.cuh"

namespace dvdq {

cudaError_t launch_rms_norm_bf16(const RmsArgs& A, int access, cudaStream_t st) { return launch_rms_t<__nv_bfloat16, true>(A, access, st); }
cudaError_t launch_quantize_rows_bf16(const RmsArgs& A, int access, cudaStream_t st) { return launch_rms_t<__nv_bfloat16, false>(A, access, st); }
cudaError_t launch_rms_norm_backward_bf16(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st) {
    return launch_rms_backward_t<__nv_bfloat16>(A, access, parts, ctas, st);
}

}  // namespace dvdq
