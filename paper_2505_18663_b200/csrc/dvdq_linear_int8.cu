// C ABI (see include/dvdq.h) of the linear layer on 8-bit integers (linear_int8.cuh): argument validation, size query, launches.
#include "linear_int8.cuh"

namespace dvdq {

dvdq_status read_linear_int8_status(uint32_t (&h)[2]) { return read_status_word(g_device_status, h); }

constexpr int64_t kL8MaxTokens = 0x7FFFFF00ll, kL8MaxChannels = (int64_t)1 << 25, kL8MaxPitch = (int64_t)1 << 38;
constexpr int64_t kL8MaxK = 131071;  // 128 * 128 * K stays below 2^31

static bool l8_sizes_ok(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N <= 0 || K <= 0 || M > kL8MaxTokens || N > kL8MaxChannels || K > kL8MaxK) return false;
    return ceil_div(M, kLinTile) * ceil_div(N, 32) < (int64_t)1 << 27;  // tiles
}
// Rows start on 16 bytes; the pitch of a single row is not read.
static dvdq_status check_l8_matrix(const void* p, int64_t rows, int64_t cols, int64_t* ld, int per16, bool required) {
    if (!p) return required ? DVDQ_ERR_NULL : DVDQ_OK;
    if (rows <= 1) *ld = align_up(cols, per16);
    if (*ld < cols || *ld > kL8MaxPitch) return DVDQ_ERR_SHAPE;
    return *ld % per16 == 0 && aligned_to(p, 16) ? DVDQ_OK : DVDQ_ERR_ALIGN;
}

}  // namespace dvdq

using namespace dvdq;

extern "C" {

size_t dvdq_linear_int8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (!l8_sizes_ok(M, N, K) || M <= kL8FewTokens) return 0;
    return (size_t)l8_plan(M, N, K).part_bytes;
}

dvdq_status dvdq_linear_int8(const int8_t* A, const float* a_scales, int64_t M, int64_t lda, const int8_t* W, const float* w_scales, int64_t N,
                             int64_t K, int64_t ldw, const void* bias, const void* R, int64_t ldr, int32_t act, void* Y, int64_t ldy, int32_t dtype,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!l8_sizes_ok(M, N, K)) return DVDQ_ERR_SHAPE;
    if ((act != DVDQ_ACT_NONE && act != DVDQ_ACT_GELU_TANH && act != DVDQ_ACT_SILU) || (dtype != DVDQ_BF16 && dtype != DVDQ_F16)) return DVDQ_ERR_UNSUPPORTED;
    if (M == 0) return DVDQ_OK;
    if (!a_scales || !w_scales) return DVDQ_ERR_NULL;
    dvdq_status s;
    if ((s = check_l8_matrix(A, M, K, &lda, 16, true)) != DVDQ_OK || (s = check_l8_matrix(W, N, K, &ldw, 16, true)) != DVDQ_OK ||
        (s = check_l8_matrix(R, M, N, &ldr, 8, false)) != DVDQ_OK || (s = check_l8_matrix(Y, M, N, &ldy, 8, true)) != DVDQ_OK)
        return s;
    if (R == Y && ldr != ldy) return DVDQ_ERR_SHAPE;  // in place: an output may not land on a residual still to be read
    if (!aligned_to(a_scales, 4) || !aligned_to(w_scales, 4) || (bias && !aligned_to(bias, 2))) return DVDQ_ERR_ALIGN;
    const LinPlan plan = M <= kL8FewTokens ? LinPlan{} : l8_plan(M, N, K);
    if (plan.part_bytes > 0) {
        if (!workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(workspace, 256)) return DVDQ_ERR_ALIGN;
        if (workspace_bytes < (size_t)plan.part_bytes) return DVDQ_ERR_WORKSPACE;
    }
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    const LinMatrix a{A, lda}, w{W, ldw}, y{Y, ldy};
    const LinEpilogue e{bias, {R, ldr}, {nullptr, 0}, act};
    const L8Scales sc{a_scales, w_scales};
    int32_t* part = static_cast<int32_t*>(workspace);
    return dtype == DVDQ_BF16 ? launch_linear_int8<__nv_bfloat16>(a, w, M, N, K, plan, sc, e, y, part, (cudaStream_t)stream)
                              : launch_linear_int8<__half>(a, w, M, N, K, plan, sc, e, y, part, (cudaStream_t)stream);
}

}  // extern "C"
