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
static dvdq_status check_l8_matrix(LinMatrix* m, int64_t rows, int64_t cols, int per16, bool required) {
    if (!m->p) return required ? DVDQ_ERR_NULL : DVDQ_OK;
    if (rows <= 1) m->ld = align_up(cols, per16);
    if (m->ld < cols || m->ld > kL8MaxPitch) return DVDQ_ERR_SHAPE;
    return m->ld % per16 == 0 && aligned_to(m->p, 16) ? DVDQ_OK : DVDQ_ERR_ALIGN;
}

}  // namespace dvdq

using namespace dvdq;

extern "C" {

size_t dvdq_linear_int8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (!l8_sizes_ok(M, N, K) || l8_few(M, N, K)) return 0;
    return (size_t)l8_plan(M, N, K).part_bytes;
}

dvdq_status dvdq_linear_int8(const dvdq_linear_int8_args* args, void* stream) {
    if (!args) return DVDQ_ERR_NULL;
    const dvdq_linear_int8_args& p = *args;
    const int64_t M = p.M, N = p.N, K = p.K;
    if (!l8_sizes_ok(M, N, K)) return DVDQ_ERR_SHAPE;
    if ((p.act != DVDQ_ACT_NONE && p.act != DVDQ_ACT_GELU_TANH && p.act != DVDQ_ACT_SILU) || (p.dtype != DVDQ_BF16 && p.dtype != DVDQ_F16)) return DVDQ_ERR_UNSUPPORTED;
    if (M == 0) return DVDQ_OK;
    if (!p.a_scales || !p.w_scales) return DVDQ_ERR_NULL;
    LinMatrix a{p.A, p.lda}, w{p.W, p.ldw}, r{p.R, p.ldr}, y{p.Y, p.ldy};
    dvdq_status s;
    if ((s = check_l8_matrix(&a, M, K, 16, true)) != DVDQ_OK || (s = check_l8_matrix(&w, N, K, 16, true)) != DVDQ_OK ||
        (s = check_l8_matrix(&r, M, N, 8, false)) != DVDQ_OK || (s = check_l8_matrix(&y, M, N, 8, true)) != DVDQ_OK)
        return s;
    if (r.p == y.p && r.ld != y.ld) return DVDQ_ERR_SHAPE;  // in place: an output may not land on a residual still to be read
    if (!aligned_to(p.a_scales, 4) || !aligned_to(p.w_scales, 4) || (p.bias && !aligned_to(p.bias, 2))) return DVDQ_ERR_ALIGN;
    const LinPlan plan = l8_few(M, N, K) ? LinPlan{} : l8_plan(M, N, K);
    if (plan.part_bytes > 0) {
        if (!p.workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(p.workspace, 256)) return DVDQ_ERR_ALIGN;
        if (p.workspace_bytes < (uint64_t)plan.part_bytes) return DVDQ_ERR_WORKSPACE;
    }
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    const LinEpilogue e{p.bias, r, {nullptr, 0}, p.act};
    const L8Scales sc{p.a_scales, p.w_scales};
    int32_t* part = static_cast<int32_t*>(p.workspace);
    return p.dtype == DVDQ_BF16 ? launch_linear_int8<__nv_bfloat16>(a, w, M, N, K, plan, sc, e, y, part, (cudaStream_t)stream)
                                : launch_linear_int8<__half>(a, w, M, N, K, plan, sc, e, y, part, (cudaStream_t)stream);
}

}  // extern "C"
