// The linear layer for a few tokens (M <= 16): modulation of one conditioning vector, single decoded
// tokens, and the gradients of such a step.
//
// What bounds it: reading W (or writing dW) once, 2 N K bytes; the products are a rounding error beside
// that.  So W goes from memory straight into registers, 16 bytes per lane, and whatever multiplies it
// is chosen to keep the load pipe fed:
//   forward  y = x W^T   warp-level mma.sync m16n8k16 with 16 rows of W as its A operand and 8 tokens as B: a dot
//            product does not care for the order of k, so a lane's 8 consecutive values of a row fill its A
//            slots of two MMAs, and the same 8 values of a token its B slots.  The warps of a CTA take
//            neighbouring pieces of k and add up through shared memory.
//   dX = dz W            a thread keeps 8 neighbouring columns of W, walks down rows n and adds dz[m, n] W[n, k] for all m
//   dW = dz^T x          a thread keeps 8 columns of x for all m, and writes one row of dW after another
// dz = dy act'(z) stays in fp32 throughout.
#pragma once

#include "linear.cuh"

namespace dvdq {

constexpr int kFewTokens = 16;

// 8 elements of a row from column k on; those past K are zero (and are not read: what follows a row's last element may be anything).
template <typename T>
__device__ __forceinline__ uint4 few_load(const T* row, int k, int K) {
    if (k + 8 <= K) return *reinterpret_cast<const uint4*>(row + k);
    Vec<T, 8> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.e[j] = k + j < K ? row[k + j] : from_f32<T>(0.f);
    return *reinterpret_cast<const uint4*>(&v);
}

template <typename T>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (IsBf16<T>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// MT groups of 8 tokens; WARPS warps share the contraction of 16 channels.
template <typename T, int MT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
linear_few_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ W, int64_t ldw, int M, int N, int K, int k_per_warp,
                  const T* __restrict__ bias, const T* R, int64_t ldr, int act, T* Y, int64_t ldy, T* Z, int64_t ldz) {
    constexpr int U = 4;  // k-steps of 32 in flight: 128 bytes of W per lane
    __shared__ float sh[WARPS][MT * 8][16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * 16;
    release_successor();
    wait_predecessor();
    // rows past N repeat the last one: their results are not stored
    const T* w0 = W + (int64_t)min(n0 + g, N - 1) * ldw;
    const T* w1 = W + (int64_t)min(n0 + g + 8, N - 1) * ldw;
    float c[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.f;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const int k1 = min(K, (warp + 1) * k_per_warp);
    auto step = [&](const uint4& a, const uint4& b, int k) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = i * 8 + g;
            const uint4 x = m < M ? few_load(X + m * ldx, k, K) : none;
            mma_16x8x16<T>(c[i], a.x, b.x, a.y, b.y, x.x, x.y);
            mma_16x8x16<T>(c[i], a.z, b.z, a.w, b.w, x.z, x.w);
        }
    };
    int k = warp * k_per_warp + t * 8;
    for (; k - t * 8 + 32 * U <= k1; k += 32 * U) {
        uint4 a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            a[u] = __ldg(reinterpret_cast<const uint4*>(w0 + k + 32 * u));
            b[u] = __ldg(reinterpret_cast<const uint4*>(w1 + k + 32 * u));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) step(a[u], b[u], k + 32 * u);
    }
    for (; k - t * 8 < k1; k += 32) {
        const bool in = k < k1;  // k_per_warp is a multiple of 32: only the end of K cuts a step short
        step(in ? few_load(w0, k, K) : none, in ? few_load(w1, k, K) : none, k);
    }
    // c[i] = (row g, tokens 2t, 2t + 1), (row g + 8, the same)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        sh[warp][i * 8 + 2 * t][g] = c[i][0];
        sh[warp][i * 8 + 2 * t + 1][g] = c[i][1];
        sh[warp][i * 8 + 2 * t][g + 8] = c[i][2];
        sh[warp][i * 8 + 2 * t + 1][g + 8] = c[i][3];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < MT * 8 * 16; o += WARPS * 32) {
        const int m = o >> 4, n = n0 + (o & 15);
        if (m >= M || n >= N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += sh[w][m][o & 15];
        if (bias) v += to_f32(bias[n]);
        if (Z) Z[m * ldz + n] = from_f32<T>(v);
        v = act_value_rt(act, v);
        if (R) v += to_f32(R[m * ldr + n]);
        Y[m * ldy + n] = from_f32<T>(v);
    }
}

// ------------------------------------------------------------------ gradients

template <typename T>
__device__ __forceinline__ float few_dz(const T* dy, int64_t lddy, const T* z, int64_t ldz, int act, int m, int n) {
    float v = to_f32(dy[m * lddy + n]);
    if (act == DVDQ_ACT_GELU_TANH) v *= act_slope<DVDQ_ACT_GELU_TANH>(to_f32(z[m * ldz + n]));
    else if (act == DVDQ_ACT_SILU) v *= act_slope<DVDQ_ACT_SILU>(to_f32(z[m * ldz + n]));
    return v;
}

constexpr int kFewCols = 128 * 8;  // columns of a CTA of the gradients: 128 threads, 8 each
constexpr int kFewRows = 32;       // rows of W whose dz a CTA holds at a time

// part[chunk][m][k] = sum over the chunk's rows n of dz[m, n] W[n, k]
template <typename T, int MT>
__global__ void __launch_bounds__(128)
linear_few_dx_kernel(const T* __restrict__ dY, int64_t lddy, const T* __restrict__ Z, int64_t ldz, int act, const T* __restrict__ W, int64_t ldw,
                     int M, int N, int K, int rows, float* __restrict__ part) {
    __shared__ float dz[kFewRows][MT];
    const int k = blockIdx.x * kFewCols + threadIdx.x * 8;
    const int n0 = blockIdx.y * rows, n1 = min(N, n0 + rows);
    Pairs<8> acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m].p[i] = 0ull;
    release_successor();
    wait_predecessor();
    for (int nb = n0; nb < n1; nb += kFewRows) {
        __syncthreads();
        for (int i = threadIdx.x; i < kFewRows * MT; i += 128) {
            const int n = nb + i / MT, m = i % MT;
            dz[i / MT][m] = n < n1 && m < M ? few_dz(dY, lddy, Z, ldz, act, m, n) : 0.f;
        }
        __syncthreads();
        if (k >= K) continue;
        const int here = min(kFewRows, n1 - nb);
        const T* w = W + (int64_t)nb * ldw;
        int r = 0;
        auto add = [&](const uint4& raw, int row) {
            const Pairs<8> v = widen2<T, 8>(*reinterpret_cast<const Vec<T, 8>*>(&raw));
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint64_t d = f2_splat(dz[row][m]);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m].p[i] = f2_fma(v.p[i], d, acc[m].p[i]);
            }
        };
        for (; r + 8 <= here; r += 8) {
            uint4 raw[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) raw[u] = few_load(w + (int64_t)(r + u) * ldw, k, K);
#pragma unroll
            for (int u = 0; u < 8; ++u) add(raw[u], r + u);
        }
        for (; r < here; ++r) add(few_load(w + (int64_t)r * ldw, k, K), r);
    }
    if (k >= K) return;
    float* out = part + ((int64_t)blockIdx.y * M) * align_up(K, 8) + k;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (m < M) {
            float4* o = reinterpret_cast<float4*>(out + m * align_up(K, 8));  // pitch: whole groups of 8
            o[0] = make_float4(acc[m].get(0), acc[m].get(1), acc[m].get(2), acc[m].get(3));
            o[1] = make_float4(acc[m].get(4), acc[m].get(5), acc[m].get(6), acc[m].get(7));
        }
    }
}
// dX[m, k] = sum of the chunks, a warp for each eighth of them
template <typename T>
__global__ void __launch_bounds__(256) linear_few_join_kernel(const float* __restrict__ part, int chunks, int M, int K, T* __restrict__ dX, int64_t lddx) {
    __shared__ float sh[8][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, k = blockIdx.x * 32 + lane, m = blockIdx.y;
    const int64_t pitch = align_up(K, 8), step = (int64_t)M * pitch;
    release_successor();
    wait_predecessor();
    float t = 0.f;
    if (k < K) {
        const float* p = part + m * pitch + k;
#pragma unroll 8
        for (int c = w; c < chunks; c += 8) t += p[c * step];
    }
    sh[w][lane] = t;
    __syncthreads();
    if (w == 0 && k < K) {
#pragma unroll
        for (int y = 1; y < 8; ++y) t += sh[y][lane];
        dX[m * lddx + k] = from_f32<T>(t);
    }
}

// dW[n, k] = sum over m of dz[m, n] x[m, k], and dbias[n] = sum over m of dz[m, n]
template <typename T, int MT>
__global__ void __launch_bounds__(128)
linear_few_dw_kernel(const T* __restrict__ dY, int64_t lddy, const T* __restrict__ Z, int64_t ldz, int act, const T* __restrict__ X, int64_t ldx,
                     int M, int N, int K, T* __restrict__ dW, int64_t lddw, float* __restrict__ db) {
    __shared__ float dz[kFewRows][MT];
    const int k = blockIdx.y * kFewCols + threadIdx.x * 8, n0 = blockIdx.x * kFewRows, here = min(kFewRows, N - n0);
    release_successor();
    wait_predecessor();
    for (int i = threadIdx.x; i < kFewRows * MT; i += 128) {
        const int n = n0 + i / MT, m = i % MT;
        dz[i / MT][m] = n < N && m < M ? few_dz(dY, lddy, Z, ldz, act, m, n) : 0.f;
    }
    Pairs<8> x[MT];
    if (dW && k < K) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint4 raw = m < M ? few_load(X + m * ldx, k, K) : make_uint4(0u, 0u, 0u, 0u);
            x[m] = widen2<T, 8>(*reinterpret_cast<const Vec<T, 8>*>(&raw));
        }
    }
    __syncthreads();
    if (db && blockIdx.y == 0 && (int)threadIdx.x < here) {
        float t = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m) t += dz[threadIdx.x][m];
        db[n0 + threadIdx.x] = t;
    }
    if (!dW || k >= K) return;
    T* out = dW + (int64_t)n0 * lddw + k;
    const int cols = min(8, K - k);
#pragma unroll 2
    for (int r = 0; r < here; ++r, out += lddw) {
        Pairs<8> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.p[i] = f2_mul(x[0].p[i], f2_splat(dz[r][0]));
#pragma unroll
        for (int m = 1; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) v.p[i] = f2_fma(x[m].p[i], f2_splat(dz[r][m]), v.p[i]);
        const Vec<T, 8> o = narrow2<T, 8>(v);
        if (cols == 8) {
            *reinterpret_cast<Vec<T, 8>*>(out) = o;
        } else {
            for (int j = 0; j < cols; ++j) out[j] = o.e[j];
        }
    }
}

// ------------------------------------------------------------------ host side

template <typename T, int MT, int WARPS>
static cudaError_t launch_linear_few_w(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinEpilogue& e,
                                       const LinMatrix& y, cudaStream_t st) {
    const int per_warp = (int)align_up(ceil_div(K, WARPS), 32);
    return launch_after(linear_few_kernel<T, MT, WARPS>, dim3((unsigned)ceil_div(N, 16)), dim3(WARPS * 32), 0, st, static_cast<const T*>(x.p), x.ld,
                        static_cast<const T*>(w.p), w.ld, (int)M, (int)N, (int)K, per_warp, static_cast<const T*>(e.bias),
                        static_cast<const T*>(e.residual.p), e.residual.ld, e.act, static_cast<T*>(const_cast<void*>(y.p)), y.ld,
                        static_cast<T*>(const_cast<void*>(e.z.p)), e.z.ld);
}
// Sixteen warps per 16 channels where the channels alone do not fill the SMs and k is long enough to share.
template <typename T>
static dvdq_status launch_linear_few(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinEpilogue& e,
                                     const LinMatrix& y, cudaStream_t st) {
    const bool wide = N / 16 < 148 * 4 && K >= 1024;
    if (M <= 8)
        return cuda_status(wide ? launch_linear_few_w<T, 1, 16>(x, w, M, N, K, e, y, st) : launch_linear_few_w<T, 1, 8>(x, w, M, N, K, e, y, st));
    return cuda_status(wide ? launch_linear_few_w<T, 2, 16>(x, w, M, N, K, e, y, st) : launch_linear_few_w<T, 2, 8>(x, w, M, N, K, e, y, st));
}

struct FewDxPlan {
    int chunks, rows;
    int64_t bytes;
};
inline FewDxPlan few_dx_plan(int64_t M, int64_t N, int64_t K) {
    // about six CTAs of 128 threads per SM; fewer chunks for more tokens, whose partial sums weigh more
    const int64_t cols = ceil_div(K, kFewCols);
    int64_t chunks = ceil_div(148 * (M <= 4 ? 6 : 3), cols);
    const int64_t most = ceil_div(N, kFewRows);
    if (chunks > most) chunks = most;
    FewDxPlan p;
    p.rows = (int)align_up(ceil_div(N, chunks), 8);
    p.chunks = (int)ceil_div(N, p.rows);
    p.bytes = (int64_t)p.chunks * M * align_up(K, 8) * 4;
    return p;
}

template <typename T, int MT>
static dvdq_status launch_linear_few_grad(const LinMatrix& dy, const LinMatrix& z, const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K,
                                          int act, const LinMatrix& dx, const LinMatrix& dw, float* db, float* part, cudaStream_t st) {
    const T *pdy = static_cast<const T*>(dy.p), *pz = static_cast<const T*>(z.p);
    const unsigned cols = (unsigned)ceil_div(K, kFewCols);
    cudaError_t e = cudaSuccess;
    if (dx.p) {
        const FewDxPlan p = few_dx_plan(M, N, K);
        e = launch_after(linear_few_dx_kernel<T, MT>, dim3(cols, (unsigned)p.chunks), dim3(128), 0, st, pdy, dy.ld, pz, z.ld, act,
                         static_cast<const T*>(w.p), w.ld, (int)M, (int)N, (int)K, p.rows, part);
        if (e == cudaSuccess)
            e = launch_after(linear_few_join_kernel<T>, dim3((unsigned)ceil_div(K, 32), (unsigned)M), dim3(256), 0, st, part, p.chunks, (int)M, (int)K,
                             static_cast<T*>(const_cast<void*>(dx.p)), dx.ld);
    }
    if (e == cudaSuccess && (dw.p || db))
        e = launch_after(linear_few_dw_kernel<T, MT>, dim3((unsigned)ceil_div(N, kFewRows), dw.p ? cols : 1u), dim3(128), 0, st, pdy, dy.ld, pz, z.ld,
                         act, static_cast<const T*>(x.p), x.ld, (int)M, (int)N, (int)K, static_cast<T*>(const_cast<void*>(dw.p)), dw.ld, db);
    return cuda_status(e);
}

}  // namespace dvdq
