// C ABI (see include/dvdq.h) of the operators that a transformer block and a latent decoder need around
// the quantized linear layers: the 16-bit linear layer and its gradients (linear.cuh), rotary
// positions (rope.cuh), group norm (group_norm.cuh).  Argument validation, size queries, launches.
#include <math.h>

#include "block_common.cuh"

#include "group_norm.cuh"
#include "linear.cuh"
#include "linear_few.cuh"
#include "rope.cuh"

namespace dvdq {

dvdq_status read_block_status(uint32_t (&h)[2]) { return read_status_word(g_device_status, h); }

static bool valid_dtype16(int32_t t) { return t == DVDQ_BF16 || t == DVDQ_F16; }
static bool valid_dtype(int32_t t) { return valid_dtype16(t) || t == DVDQ_F32; }
static bool valid_act(int32_t a) { return a == DVDQ_ACT_NONE || a == DVDQ_ACT_GELU_TANH || a == DVDQ_ACT_SILU; }

// A matrix operand of the linear layer: rows start on 16 bytes; the pitch of a single row is not read.
constexpr int64_t kLinMaxTokens = 0x7FFFFF00ll, kLinMaxChannels = (int64_t)1 << 25, kLinMaxPitch = (int64_t)1 << 38;
static dvdq_status check_matrix(const void* p, int64_t rows, int64_t cols, int64_t* ld, bool required) {
    if (!p) return required ? DVDQ_ERR_NULL : DVDQ_OK;
    if (rows <= 1) *ld = align_up(cols, 8);
    if (*ld < cols || *ld > kLinMaxPitch) return DVDQ_ERR_SHAPE;
    if (*ld % 8 != 0 || !aligned_to(p, 16)) return DVDQ_ERR_ALIGN;
    return DVDQ_OK;
}
static bool linear_sizes_ok(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N <= 0 || K <= 0 || M > kLinMaxTokens || N > kLinMaxChannels || K > kLinMaxChannels) return false;
    const int64_t m = ceil_div(M, kLinTile), n = ceil_div(N, kLinTile), k = ceil_div(K, kLinTile), most = (int64_t)1 << 24;
    return m * n < most && m * k < most && n * k < most;  // tiles of y, dX and dW
}

static int64_t dz_chunks(int64_t M, int64_t N) {
    // One chunk: its sums are the result, no second kernel.  Both ways with 1536 -> 1536: 64 tokens 9.7 and 9.9 us, 128 12.5 and 11.5,
    // 256 16.6 and 12.7.
    if (M <= 64) return 1;
    int64_t c = ceil_div(148 * 6, ceil_div(N, kLinDzCols));
    const int64_t most = ceil_div(M, 32);
    c = c > most ? most : c;
    return c < 1 ? 1 : c;
}
struct LinBackwardPlan {
    LinPlan dx, dw;          // a launch each
    LinPlan dx_two, dw_two;  // in one launch, where `two`
    int64_t lddz, dz_off, sums_off, part_off, total;
    int64_t chunks, rows;
    bool two;  // dX and dW in one launch
    int low;   // M where dz comes in two parts: rows M .. 2 M hold the second; or 0
    // What a call needs of it: pieces only of the products it asks for.  (K matters to those alone: a call for the
    // bias's gradient need not know it.)
    int64_t room(bool with_dx, bool with_dw, bool few) const {
        int64_t part = 0;
        if (with_dx && !(two && with_dw)) part = dx.part_bytes;
        if (with_dw && !few && !(two && with_dx) && part < dw.part_bytes) part = dw.part_bytes;
        return part_off + part;
    }
};
static LinBackwardPlan linear_backward_plan(int64_t M, int64_t N, int64_t K, int32_t act) {
    LinBackwardPlan p;
    p.low = act != DVDQ_ACT_NONE && dz_in_two_parts(M, N) ? (int)M : 0;
    double e_dx, e_dw;
    p.dx = lin_plan(M, K, N, 64, &e_dx);
    p.dw = lin_plan(N, K, M, 64, &e_dw);
    p.two = !few_weight_gradient(M) && lin_plan_two(M, N, K, e_dx, e_dw, &p.dx_two, &p.dw_two);
    p.lddz = align_up(N, 8);
    p.rows = ceil_div(M, dz_chunks(M, N));
    p.chunks = ceil_div(M, p.rows);
    p.dz_off = 0;
    p.sums_off = act == DVDQ_ACT_NONE ? 0 : align_up((M + p.low) * p.lddz * 2, 256);
    p.part_off = p.sums_off + align_up(p.chunks * N * 4, 256);
    p.total = p.part_off + (p.dx.part_bytes > p.dw.part_bytes ? p.dx.part_bytes : p.dw.part_bytes);
    return p;
}

template <typename T>
static dvdq_status linear_t(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinPlan& plan, const LinEpilogue& e,
                            const LinMatrix& y, void* ws, cudaStream_t st) {
    if (M <= kFewTokens) return launch_linear_few<T>(x, w, M, N, K, e, y, st);
    return launch_linear<T, false, false>(x, w, M, N, K, plan, e, y, static_cast<float*>(ws), 0, st);
}

template <typename T>
static dvdq_status linear_backward_t(const LinMatrix& dy, const LinMatrix& z, const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N,
                                     int64_t K, int32_t act, const LinBackwardPlan& p, const LinMatrix& dx, const LinMatrix& dw, float* db,
                                     uint8_t* ws, cudaStream_t st) {
    const bool few = few_weight_gradient(M);  // dW and dbias by their own kernel
    float* sums = !db || few ? nullptr : p.chunks == 1 ? db : reinterpret_cast<float*>(ws + p.sums_off);
    float* part = reinterpret_cast<float*>(ws + p.part_off);
    LinMatrix dz = dy;
    if (act != DVDQ_ACT_NONE) dz = LinMatrix{ws + p.dz_off, p.lddz};
    dvdq_status s;
    if (sums || (act != DVDQ_ACT_NONE && (dx.p || (dw.p && !few)))) {
        const dim3 grid((unsigned)ceil_div(N, kLinDzCols), (unsigned)p.chunks);
        auto k = act == DVDQ_ACT_GELU_TANH ? linear_dz_kernel<T, DVDQ_ACT_GELU_TANH>
                 : act == DVDQ_ACT_SILU    ? linear_dz_kernel<T, DVDQ_ACT_SILU>
                                           : linear_dz_kernel<T, DVDQ_ACT_NONE>;
        if ((s = cuda_status(launch_after(k, grid, dim3(kStreamThreads), 0, st, static_cast<const T*>(dy.p), dy.ld, static_cast<const T*>(z.p),
                                          z.ld, M, (int)N, p.rows, static_cast<T*>(const_cast<void*>(dz.p)), dz.ld, p.low, sums))) != DVDQ_OK)
            return s;
        if (sums && sums != db && (s = cuda_status(launch_after(linear_colsum_kernel, dim3((unsigned)ceil_div(N, 32)), dim3(256), 0, st, sums, (int)p.chunks,
                                                (int)N, db))) != DVDQ_OK)
            return s;
    }
    const LinEpilogue none = {};
    if (p.two && dx.p && dw.p) return launch_linear_two<T>(dz, x, w, M, N, K, p.dx_two, p.dw_two, dx, dw, p.low, st);
    if (dx.p && (s = launch_linear<T, false, true>(dz, w, M, K, N, p.dx, none, dx, part, p.low, st)) != DVDQ_OK) return s;
    if (few && (dw.p || db))
        return M == 1 ? launch_linear_few_dw<T, 1>(dy, z, x, M, N, K, act, dw, db, st) : launch_linear_few_dw<T, 4>(dy, z, x, M, N, K, act, dw, db, st);
    if (dw.p && (s = launch_linear<T, true, true>(dz, x, N, K, M, p.dw, none, dw, part, p.low, st)) != DVDQ_OK) return s;
    return DVDQ_OK;
}

}  // namespace dvdq

using namespace dvdq;

extern "C" {

// ---- the 16-bit linear layer ------------------------------------------------------------------

size_t dvdq_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (!linear_sizes_ok(M, N, K) || M <= kFewTokens) return 0;
    return (size_t)lin_plan(M, N, K, 32).part_bytes;
}

dvdq_status dvdq_linear(const void* X, int64_t M, int64_t ldx, const void* W, int64_t N, int64_t K, int64_t ldw, const void* bias,
                        const void* R, int64_t ldr, int32_t act, void* Y, int64_t ldy, void* Z, int64_t ldz, int32_t dtype,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!linear_sizes_ok(M, N, K)) return DVDQ_ERR_SHAPE;
    if (!valid_act(act) || !valid_dtype16(dtype)) return DVDQ_ERR_UNSUPPORTED;
    if (M == 0) return DVDQ_OK;
    dvdq_status s;
    if ((s = check_matrix(X, M, K, &ldx, true)) != DVDQ_OK || (s = check_matrix(W, N, K, &ldw, true)) != DVDQ_OK ||
        (s = check_matrix(R, M, N, &ldr, false)) != DVDQ_OK || (s = check_matrix(Y, M, N, &ldy, true)) != DVDQ_OK ||
        (s = check_matrix(Z, M, N, &ldz, false)) != DVDQ_OK)
        return s;
    if (R == Y && ldr != ldy) return DVDQ_ERR_SHAPE;  // in place: an output may not land on a residual still to be read
    if (bias && !aligned_to(bias, 2)) return DVDQ_ERR_ALIGN;
    const LinPlan plan = M <= kFewTokens ? LinPlan{} : lin_plan(M, N, K, 32);
    if (plan.part_bytes > 0) {
        if (!workspace) return DVDQ_ERR_NULL;
        if (!aligned_to(workspace, 256)) return DVDQ_ERR_ALIGN;
        if (workspace_bytes < (size_t)plan.part_bytes) return DVDQ_ERR_WORKSPACE;
    }
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    const LinMatrix x{X, ldx}, w{W, ldw}, y{Y, ldy};
    const LinEpilogue e{bias, {R, ldr}, {Z, ldz}, act};
    return dtype == DVDQ_BF16 ? linear_t<__nv_bfloat16>(x, w, M, N, K, plan, e, y, workspace, (cudaStream_t)stream)
                              : linear_t<__half>(x, w, M, N, K, plan, e, y, workspace, (cudaStream_t)stream);
}

size_t dvdq_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t act) {
    if (!linear_sizes_ok(M, N, K) || M == 0 || !valid_act(act)) return 0;
    return (size_t)linear_backward_plan(M, N, K, act).total;
}

dvdq_status dvdq_linear_backward(const void* dY, int64_t lddy, const void* Z, int64_t ldz, const void* X, int64_t ldx, const void* W,
                                 int64_t ldw, int64_t M, int64_t N, int64_t K, int32_t act, void* dX, int64_t lddx, void* dW, int64_t lddw,
                                 float* dbias, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!linear_sizes_ok(M, N, K)) return DVDQ_ERR_SHAPE;
    if (!valid_act(act) || !valid_dtype16(dtype)) return DVDQ_ERR_UNSUPPORTED;
    dvdq_status s;
    const bool some = M > 0;
    if ((s = check_matrix(dY, M, N, &lddy, some)) != DVDQ_OK || (s = check_matrix(Z, M, N, &ldz, some && act != DVDQ_ACT_NONE)) != DVDQ_OK ||
        (s = check_matrix(X, M, K, &ldx, some && dW)) != DVDQ_OK || (s = check_matrix(W, N, K, &ldw, some && dX)) != DVDQ_OK ||
        (s = check_matrix(dX, M, K, &lddx, false)) != DVDQ_OK || (s = check_matrix(dW, N, K, &lddw, false)) != DVDQ_OK)
        return s;
    if (dbias && !aligned_to(dbias, 4)) return DVDQ_ERR_ALIGN;
    if (!some) {  // no tokens: sums over nothing
        if (dW || dbias) {
            if ((s = check_device_arch()) != DVDQ_OK) return s;
            if (dW && cudaMemset2DAsync(dW, (size_t)lddw * 2, 0, (size_t)K * 2, (size_t)N, (cudaStream_t)stream) != cudaSuccess) return DVDQ_ERR_CUDA;
            if (dbias && cudaMemsetAsync(dbias, 0, (size_t)N * 4, (cudaStream_t)stream) != cudaSuccess) return DVDQ_ERR_CUDA;
        }
        return DVDQ_OK;
    }
    if (!workspace) return DVDQ_ERR_NULL;
    if (!aligned_to(workspace, 256)) return DVDQ_ERR_ALIGN;
    const LinBackwardPlan plan = linear_backward_plan(M, N, K, act);
    if (workspace_bytes < (size_t)plan.room(dX != nullptr, dW != nullptr, few_weight_gradient(M))) return DVDQ_ERR_WORKSPACE;
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    const LinMatrix dy{dY, lddy}, z{act == DVDQ_ACT_NONE ? nullptr : Z, ldz}, x{X, ldx}, w{W, ldw}, dx{dX, lddx}, dw{dW, lddw};
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return dtype == DVDQ_BF16 ? linear_backward_t<__nv_bfloat16>(dy, z, x, w, M, N, K, act, plan, dx, dw, dbias, ws, (cudaStream_t)stream)
                              : linear_backward_t<__half>(dy, z, x, w, M, N, K, act, plan, dx, dw, dbias, ws, (cudaStream_t)stream);
}

// ---- rotary positions ---------------------------------------------------------------------------

dvdq_status dvdq_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double original_length, double beta_fast,
                                  double beta_slow, double* freqs_out, double* amplitude_out) {
    if (!freqs_out || !amplitude_out) return DVDQ_ERR_NULL;
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 2 * kRopeMaxPairs || !(theta > 0.0)) return DVDQ_ERR_SHAPE;
    if (scaling < DVDQ_ROPE_PLAIN || scaling > DVDQ_ROPE_BY_PARTS) return DVDQ_ERR_UNSUPPORTED;
    if (scaling != DVDQ_ROPE_PLAIN && !(factor >= 1.0)) return DVDQ_ERR_SHAPE;
    if (scaling == DVDQ_ROPE_BASE && rot_dim == 2) return DVDQ_ERR_SHAPE;  // the one frequency is 1 whatever the base
    // (theta <= 1: no pair turns slower than the one before it, and there is no ramp over the pairs)
    if (scaling == DVDQ_ROPE_BY_PARTS && (!(theta > 1.0) || !(original_length > 0.0) || !isfinite(original_length) || !(beta_fast > beta_slow) || !(beta_slow > 0.0))) return DVDQ_ERR_SHAPE;
    const int pairs = rot_dim / 2;
    const double two_pi = 6.283185307179586476925286766559;
    // base: theta' so that the lowest frequency is divided by factor and the highest stays
    const double base = scaling == DVDQ_ROPE_BASE ? theta * pow(factor, (double)rot_dim / (rot_dim - 2)) : theta;
    // by parts: the pair index that turns r times over the original length is where theta^(2i/rot) = length / (2 pi r)
    double low = 0.0, high = 1.0;
    if (scaling == DVDQ_ROPE_BY_PARTS) {
        auto index_of = [&](double turns) { return rot_dim * log(original_length / (turns * two_pi)) / (2.0 * log(theta)); };
        low = floor(index_of(beta_fast));
        high = ceil(index_of(beta_slow));
        if (!(low >= 0.0)) low = 0.0;
        if (!(high <= rot_dim - 1)) high = rot_dim - 1;
        if (high <= low) high = low + 0.001;
    }
    for (int i = 0; i < pairs; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == DVDQ_ROPE_LINEAR) f /= factor;
        if (scaling == DVDQ_ROPE_BY_PARTS) {
            double t = (i - low) / (high - low);  // 0: kept, 1: divided by factor
            t = t < 0.0 ? 0.0 : t > 1.0 ? 1.0 : t;
            f = f * (1.0 - t) + f / factor * t;
        }
        freqs_out[i] = f;
    }
    *amplitude_out = scaling == DVDQ_ROPE_BY_PARTS ? 0.1 * log(factor) + 1.0 : 1.0;
    return DVDQ_OK;
}

dvdq_status dvdq_rope_table(const double* freqs, const int32_t* axis_of_pair, int32_t pairs, const int32_t* positions, int64_t rows,
                            int32_t axes, double amplitude, float* table_out, void* stream) {
    if (!freqs) return DVDQ_ERR_NULL;
    if (pairs < 1 || pairs > kRopeMaxPairs || rows < 0 || rows > ((int64_t)1 << 40) || axes < 1 || axes > 8) return DVDQ_ERR_SHAPE;
    if (!positions && axes != 1) return DVDQ_ERR_NULL;
    RopeAngles ang = {};
    for (int i = 0; i < pairs; ++i) {
        const int32_t a = axis_of_pair ? axis_of_pair[i] : 0;
        if (a < 0 || a >= axes) return DVDQ_ERR_SHAPE;
        ang.freq[i] = freqs[i];
        ang.axis[i] = (uint8_t)a;
    }
    if (rows == 0) return DVDQ_OK;
    if (!table_out) return DVDQ_ERR_NULL;
    if (!aligned_to(table_out, 16) || (positions && !aligned_to(positions, 4))) return DVDQ_ERR_ALIGN;
    dvdq_status s = check_device_arch();
    if (s != DVDQ_OK) return s;
    const int64_t total = rows * pairs, ctas = ceil_div(total, kRopeThreads);
    rope_table_kernel<<<(unsigned)(ctas < 148 * 16 ? ctas : 148 * 16), kRopeThreads, 0, (cudaStream_t)stream>>>(
        ang, positions, total, pairs, axes, amplitude, reinterpret_cast<float2*>(table_out));
    return cuda_status(cudaGetLastError());
}

static dvdq_status check_rope_side(const dvdq_rope_tensor* t, int64_t B, int64_t S, int32_t D, int bytes, RopeSide* out) {
    if (t->heads < 1 || t->heads > 65536) return DVDQ_ERR_SHAPE;
    if (!t->x || !t->y) return DVDQ_ERR_NULL;
    if (!aligned_to(t->x, bytes) || !aligned_to(t->y, bytes)) return DVDQ_ERR_ALIGN;
    const int64_t extent[3] = {B, S, t->heads};
    const int64_t xs[3] = {t->x_batch, t->x_token, t->x_head}, ys[3] = {t->y_batch, t->y_token, t->y_head};
    int64_t x[3], y[3];
    for (int i = 0; i < 3; ++i) {
        x[i] = extent[i] == 1 ? 0 : xs[i];  // the stride of an extent of one is not read
        y[i] = extent[i] == 1 ? 0 : ys[i];
        if (x[i] < 0 || (extent[i] > 1 && y[i] < D)) return DVDQ_ERR_SHAPE;  // outputs of two heads may not overlap
    }
    if (t->x == t->y && (x[0] != y[0] || x[1] != y[1] || x[2] != y[2])) return DVDQ_ERR_SHAPE;
    *out = RopeSide{t->x, t->y, (int)t->heads, x[0], x[1], x[2], y[0], y[1], y[2]};
    return DVDQ_OK;
}

dvdq_status dvdq_rope(const dvdq_rope_tensor* q, const dvdq_rope_tensor* k, int64_t B, int64_t S, int32_t head_dim, int32_t rot_dim,
                      const float* table, int64_t table_rows, const int32_t* rows, int64_t rows_batch, int32_t layout, int32_t inverse,
                      int32_t dtype, void* stream) {
    if (!q) return DVDQ_ERR_NULL;
    if (B < 0 || S < 0 || B > 0x7FFFFFFFll || S > 0x7FFFFFFFll || head_dim < 1 || head_dim > 4096) return DVDQ_ERR_SHAPE;
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim || rot_dim > 2 * kRopeMaxPairs || table_rows < 0) return DVDQ_ERR_SHAPE;
    if (!valid_dtype(dtype) || (layout != DVDQ_ROPE_PAIRS && layout != DVDQ_ROPE_HALVES)) return DVDQ_ERR_UNSUPPORTED;
    if (B == 0 || S == 0) return DVDQ_OK;
    if (!table) return DVDQ_ERR_NULL;
    if (!rows && table_rows < S) return DVDQ_ERR_SHAPE;  // without rows, token s takes row s
    if (table_rows == 0) return DVDQ_ERR_SHAPE;          // a row outside the table is read as row 0 before its NaN is written
    if (!aligned_to(table, 16) || (rows && !aligned_to(rows, 4))) return DVDQ_ERR_ALIGN;
    RopeSide side[2] = {};
    const int bytes = dtype_bytes(dtype);
    dvdq_status s = check_rope_side(q, B, S, head_dim, bytes, &side[0]);
    if (s == DVDQ_OK && k) s = check_rope_side(k, B, S, head_dim, bytes, &side[1]);
    if (s != DVDQ_OK) return s;
    if ((s = check_device_arch()) != DVDQ_OK) return s;
    RopeArgs A = {};
    A.q = side[0];
    A.k = side[1];
    A.table = reinterpret_cast<const float2*>(table);
    A.rows = rows;
    A.rows_batch = rows_batch;
    A.table_rows = table_rows;
    A.S = S;
    A.rot = rot_dim;
    A.head_dim = head_dim;
    A.inverse = inverse != 0;
    const bool halves = layout == DVDQ_ROPE_HALVES;
    const int w = rope_access(side, k ? 2 : 1, head_dim, rot_dim, halves, bytes);
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t tokens = B * S;
    cudaError_t e;
    if (dtype == DVDQ_BF16) e = halves ? launch_rope_t<__nv_bfloat16, true>(A, w, tokens, st) : launch_rope_t<__nv_bfloat16, false>(A, w, tokens, st);
    else if (dtype == DVDQ_F16) e = halves ? launch_rope_t<__half, true>(A, w, tokens, st) : launch_rope_t<__half, false>(A, w, tokens, st);
    else e = halves ? launch_rope_t<float, true>(A, w, tokens, st) : launch_rope_t<float, false>(A, w, tokens, st);
    return cuda_status(e);
}

// ---- group norm ---------------------------------------------------------------------------------

static bool group_norm_sizes_ok(int64_t N, int64_t S, int64_t C, int64_t G) {
    return N >= 0 && N <= 65535 && S >= 0 && S <= 0x7FFFFFFFll && C > 0 && C <= (1 << 20) && G > 0 && C % G == 0 && G <= 65535 / gn_pieces(C / G);
}

size_t dvdq_group_norm_workspace_bytes(int64_t N, int64_t S, int64_t C, int64_t G) {
    if (!group_norm_sizes_ok(N, S, C, G) || N == 0 || S == 0) return 0;
    return (size_t)gn_room(N, S, C, G).total;
}

// pitches of samples and places of an [N, S, C] tensor; those of an extent of one are not read
static dvdq_status check_gn_tensor(const void* p, int64_t N, int64_t S, int64_t C, int64_t* pn, int64_t* ps, int bytes, bool written) {
    if (!p) return DVDQ_OK;
    if (N == 1) *pn = 0;
    if (S == 1) *ps = 0;
    if (*pn < 0 || *ps < 0) return DVDQ_ERR_SHAPE;
    if (written && ((S > 1 && *ps < C) || (N > 1 && *pn < C))) return DVDQ_ERR_SHAPE;  // outputs may not overlap
    return aligned_to(p, bytes) ? DVDQ_OK : DVDQ_ERR_ALIGN;
}

// A tensor written over the one it is made from has the same pitches (after check_gn_tensor).
static bool gn_in_place_ok(const void* from, int64_t fn, int64_t fs, const void* to, int64_t tn, int64_t ts) {
    return from != to || (fn == tn && fs == ts);
}

static dvdq_status group_norm_run(const GnArgs& A0, int64_t N, int64_t S, int32_t act, int32_t dtype, int32_t param_dtype, bool backward,
                                  void* workspace, size_t workspace_bytes, cudaStream_t st) {
    GnArgs A = A0;
    if (!workspace) return DVDQ_ERR_NULL;
    if (!aligned_to(workspace, 256)) return DVDQ_ERR_ALIGN;
    const GnRoom room = gn_room(N, S, A.C, A.G);
    if (workspace_bytes < (size_t)room.total) return DVDQ_ERR_WORKSPACE;
    dvdq_status s = check_device_arch();
    if (s != DVDQ_OK) return s;
    const GnPlan p = gn_plan(N, S, backward ? 2 : 4);
    A.N = (int)N;
    A.S = S;
    A.inv = 1.0 / ((double)S * A.per);
    A.chunks = p.chunks;
    A.rows = p.rows;
    A.params_f32 = param_dtype == DVDQ_F32;
    A.params_bf16 = param_dtype == DVDQ_BF16;
    A.part = static_cast<float2*>(workspace);
    A.part64 = static_cast<double2*>(workspace);
    A.pivot = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + room.pivot_off);
    A.arrived = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + room.arrived_off);
    A.stat = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + room.stat_off);
    A.part_c = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + room.part_c_off);
    const cudaError_t e = dtype == DVDQ_BF16  ? launch_gn_t<__nv_bfloat16>(A, backward, act, st)
                          : dtype == DVDQ_F16 ? launch_gn_t<__half>(A, backward, act, st)
                                              : launch_gn_t<float>(A, backward, act, st);
    return cuda_status(e);
}

dvdq_status dvdq_group_norm(const void* X, int64_t x_sample, int64_t x_place, int64_t N, int64_t S, int64_t C, int64_t G, const void* gamma,
                            const void* beta, int32_t param_dtype, float eps, int32_t act, void* Y, int64_t y_sample, int64_t y_place,
                            float* mean_out, float* rstd_out, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!group_norm_sizes_ok(N, S, C, G) || !(eps >= 0.0f)) return DVDQ_ERR_SHAPE;
    if (!valid_act(act) || !valid_dtype(dtype) || (param_dtype != dtype && param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    if (N == 0) return DVDQ_OK;
    if (S > 0 && (!X || !Y)) return DVDQ_ERR_NULL;
    dvdq_status s;
    const int bytes = dtype_bytes(dtype), pb = dtype_bytes(param_dtype);
    if ((s = check_gn_tensor(X, N, S, C, &x_sample, &x_place, bytes, false)) != DVDQ_OK ||
        (s = check_gn_tensor(Y, N, S, C, &y_sample, &y_place, bytes, true)) != DVDQ_OK)
        return s;
    if (S > 0 && !gn_in_place_ok(X, x_sample, x_place, Y, y_sample, y_place)) return DVDQ_ERR_SHAPE;
    if ((gamma && !aligned_to(gamma, pb)) || (beta && !aligned_to(beta, pb)) || (mean_out && !aligned_to(mean_out, 4)) ||
        (rstd_out && !aligned_to(rstd_out, 4)))
        return DVDQ_ERR_ALIGN;
    if (S == 0) {
        if (!mean_out && !rstd_out) return DVDQ_OK;
        if ((s = check_device_arch()) != DVDQ_OK) return s;
        gn_empty_kernel<<<(unsigned)ceil_div(N * G, 256), 256, 0, (cudaStream_t)stream>>>(mean_out, rstd_out, N * G, nullptr, nullptr, 0, eps);
        return cuda_status(cudaGetLastError());
    }
    GnArgs A = {};
    A.x = X;
    A.y = Y;
    A.gamma = gamma;
    A.beta = beta;
    A.mean = mean_out;
    A.rstd = rstd_out;
    A.xn = x_sample;
    A.xs = x_place;
    A.yn = y_sample;
    A.ys = y_place;
    A.C = (int)C;
    A.G = (int)G;
    A.per = (int)(C / G);
    A.eps = eps;
    return group_norm_run(A, N, S, act, dtype, param_dtype, false, workspace, workspace_bytes, (cudaStream_t)stream);
}

dvdq_status dvdq_group_norm_backward(const void* dY, int64_t dy_sample, int64_t dy_place, const void* X, int64_t x_sample, int64_t x_place,
                                     const float* mean, const float* rstd, int64_t N, int64_t S, int64_t C, int64_t G, const void* gamma,
                                     const void* beta, int32_t param_dtype, int32_t act, void* dX, int64_t dx_sample, int64_t dx_place,
                                     float* dgamma, float* dbeta, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!group_norm_sizes_ok(N, S, C, G)) return DVDQ_ERR_SHAPE;
    if (!valid_act(act) || !valid_dtype(dtype) || (param_dtype != dtype && param_dtype != DVDQ_F32)) return DVDQ_ERR_UNSUPPORTED;
    dvdq_status s;
    const int bytes = dtype_bytes(dtype), pb = dtype_bytes(param_dtype);
    if ((gamma && !aligned_to(gamma, pb)) || (beta && !aligned_to(beta, pb)) || (dgamma && !aligned_to(dgamma, 4)) ||
        (dbeta && !aligned_to(dbeta, 4)) || (mean && !aligned_to(mean, 4)) || (rstd && !aligned_to(rstd, 4)))
        return DVDQ_ERR_ALIGN;
    if (N == 0 || S == 0) {  // sums over nothing
        if (!dgamma && !dbeta) return DVDQ_OK;
        if ((s = check_device_arch()) != DVDQ_OK) return s;
        gn_empty_kernel<<<(unsigned)ceil_div(C, 256), 256, 0, (cudaStream_t)stream>>>(nullptr, nullptr, 0, dgamma, dbeta, (int)C, 1.0f);
        return cuda_status(cudaGetLastError());
    }
    if (!dY || !X || !mean || !rstd) return DVDQ_ERR_NULL;
    if ((s = check_gn_tensor(dY, N, S, C, &dy_sample, &dy_place, bytes, false)) != DVDQ_OK ||
        (s = check_gn_tensor(X, N, S, C, &x_sample, &x_place, bytes, false)) != DVDQ_OK ||
        (s = check_gn_tensor(dX, N, S, C, &dx_sample, &dx_place, bytes, true)) != DVDQ_OK)
        return s;
    if (!gn_in_place_ok(dY, dy_sample, dy_place, dX, dx_sample, dx_place) || !gn_in_place_ok(X, x_sample, x_place, dX, dx_sample, dx_place))
        return DVDQ_ERR_SHAPE;
    GnArgs A = {};
    A.x = X;
    A.dy = dY;
    A.y = dX;
    A.gamma = gamma;
    A.beta = beta;
    A.mean = const_cast<float*>(mean);
    A.rstd = const_cast<float*>(rstd);
    A.dgamma = dgamma;
    A.dbeta = dbeta;
    A.xn = x_sample;
    A.xs = x_place;
    A.dn = dy_sample;
    A.ds = dy_place;
    A.yn = dX ? dx_sample : 0;
    A.ys = dX ? dx_place : 0;
    A.C = (int)C;
    A.G = (int)G;
    A.per = (int)(C / G);
    return group_norm_run(A, N, S, act, dtype, param_dtype, true, workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // extern "C"
