// The linear layer for a few tokens: modulation of one conditioning vector, single decoded tokens (M <= 8), and
// the weights' gradient of such a step (M <= 4).  With more tokens the kernel of linear.cuh is faster
// (5120 x 5120: 17 us for 16 tokens there, 24 here with a second group of tokens, 14.6 for 4).
//
// What bounds it: reading W (or writing dW) once, 2 N K bytes (3072 -> 18432, 1 token: 21.2 us, 5.3 TB/s); the products are a rounding
// error beside that.  So W comes in 16-byte pieces per lane, always several in flight, and whatever multiplies it
// is chosen to keep the loads going:
//   forward  y = x W^T   warp-level mma.sync m16n8k16 with 16 rows of W as its A operand and 8 tokens as B: a dot
//            product does not care for the order of k, so a lane's 8 consecutive values of a row fill its A
//            slots of two MMAs, and the same 8 values of a token its B slots.  Warps that share channels take
//            neighbouring pieces of k and add up through shared memory.
//   dW = dz^T x          a thread keeps 8 columns of x for all m, and writes one row of dW after another; dz = dy act'(z)
//            stays in fp32 (so few terms would not average a rounding of dz away)
// dX = dz W takes linear.cuh's kernel, with dz in two 16-bit parts, one below the other: streaming W by columns with fp32 sums was slower (18432 x 3072, 1 token: 33 us, 26 there).
#pragma once

#include "linear.cuh"

namespace dvdq {

constexpr int kFewTokens = 8;
// The gradients are formed from dz in two parts where a sum over tokens (dW) or over channels (dX) has so few terms that their roundings
// do not average out, or dz is small altogether.  Both ways with 1536 -> 1536: 32 tokens 10.4 and 8.5 us; 32760 tokens, 1536 ->
// 16, cold: 90 and 74.  (Rows of the second part begin at M, and a tile's coordinate is 32 bits.)
inline bool dz_in_two_parts(int64_t M, int64_t N) { return M <= 32 || (N <= 32 && M < ((int64_t)1 << 30)) || M * N < 4096; }

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

// A CTA's warps are WARPS / KS groups of 16 channels times KS neighbouring pieces of k; each
// lane streams its two rows of W through its own ring (thread_stream), so that loads never pause.
constexpr int kFewDepth = 6;
template <typename T, int WARPS, int KS>
__global__ void __launch_bounds__(WARPS * 32)
linear_few_kernel(const T* __restrict__ X, int64_t ldx, const T* __restrict__ W, int64_t ldw, int M, int N, int K, int k_per_warp,
                  const T* __restrict__ bias, const T* R, int64_t ldr, int act, T* Y, int64_t ldy, T* Z, int64_t ldz) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int piece = warp % KS, group = warp / KS;
    const int n0 = (blockIdx.x * (WARPS / KS) + group) * 16;
    wait_predecessor();
    release_successor();
    float c[4] = {0.f, 0.f, 0.f, 0.f};
    if (n0 < N) {
        // rows past N repeat the last one: their results are not stored
        const T* w0 = W + (int64_t)min(n0 + g, N - 1) * ldw;
        const T* w1 = W + (int64_t)min(n0 + g + 8, N - 1) * ldw;
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        int k = piece * k_per_warp + t * 8;
        const int k1 = min(K, (piece + 1) * k_per_warp);  // k_per_warp is a multiple of 32
        auto step = [&](const uint4& a, const uint4& b) {
            const uint4 x = g < M ? few_load(X + g * ldx, k, K) : none;
            mma_16x8x16<T>(c, a.x, b.x, a.y, b.y, x.x, x.y);
            mma_16x8x16<T>(c, a.z, b.z, a.w, b.w, x.z, x.w);
            k += 32;
        };
        const int whole = k1 > k - t * 8 ? (k1 - (k - t * 8)) / 32 : 0;  // steps of 32 that lie in the rows
        thread_stream<kFewDepth, 2, T, 8, WARPS * 32>(smem_u32(raw) + threadIdx.x * 16, whole, w0 + k, 32, w1 + k, 32,
            [&](const Vec<T, 8>& a, const Vec<T, 8>& b) { step(*reinterpret_cast<const uint4*>(&a), *reinterpret_cast<const uint4*>(&b)); });
        if (k - t * 8 < k1) {  // the end of the rows
            const bool in = k < K;
            step(in ? few_load(w0, k, K) : none, in ? few_load(w1, k, K) : none);
        }
    }
    __syncthreads();  // the ring's memory becomes the sums'
    float* sh = reinterpret_cast<float*>(raw);  // [warp][token][16]
    constexpr int kTile = 8 * 16;
    float* mine = sh + warp * kTile + 2 * t * 16 + g;  // c = (row g, tokens 2t, 2t + 1), (row g + 8, the same)
    mine[0] = c[0];
    mine[16] = c[1];
    mine[8] = c[2];
    mine[24] = c[3];
    __syncthreads();
    for (int o = threadIdx.x; o < (WARPS / KS) * kTile; o += WARPS * 32) {
        const int gr = o / kTile, r = o - gr * kTile, m = r >> 4, n = (blockIdx.x * (WARPS / KS) + gr) * 16 + (r & 15);
        if (m >= M || n >= N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < KS; ++w) v += sh[(gr * KS + w) * kTile + r];
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
constexpr int kFewRows = 16;       // rows of dW that a CTA writes, at most

// dW[n, k] = sum over m of dz[m, n] x[m, k], and dbias[n] = sum over m of dz[m, n]
template <typename T, int MT>
__global__ void __launch_bounds__(128)
linear_few_dw_kernel(const T* __restrict__ dY, int64_t lddy, const T* __restrict__ Z, int64_t ldz, int act, const T* __restrict__ X, int64_t ldx,
                     int M, int N, int K, int rows, T* __restrict__ dW, int64_t lddw, float* __restrict__ db) {
    __shared__ float dz[kFewRows][MT];
    const int k = blockIdx.y * kFewCols + threadIdx.x * 8, n0 = blockIdx.x * rows, here = min(rows, N - n0);
    wait_predecessor();
    release_successor();
    for (int i = threadIdx.x; i < here * MT; i += 128) {
        const int n = n0 + i / MT, m = i % MT;
        dz[i / MT][m] = m < M ? few_dz(dY, lddy, Z, ldz, act, m, n) : 0.f;
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

// dW by linear_few_dw_kernel (5120 x 5120, 4 tokens: 10.0 us, 13.7 in linear.cuh).
inline bool few_weight_gradient(int64_t M) { return M <= 4; }

template <typename T, int WARPS, int KS>
static cudaError_t launch_linear_few_w(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinEpilogue& e,
                                       const LinMatrix& y, cudaStream_t st) {
    constexpr int smem = WARPS * 32 * 32 * kFewDepth;  // the rings; the sums take their place
    auto kern = linear_few_kernel<T, WARPS, KS>;
    static PerDevice<int> ready;
    if (smem > 48 * 1024 &&
        !ready.get([&](int&, int) { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess; }))
        return cudaErrorInvalidValue;
    const int per_warp = (int)align_up(ceil_div(K, KS), 32);
    return launch_after(kern, dim3((unsigned)ceil_div(N, 16 * (WARPS / KS))), dim3(WARPS * 32), smem, st, static_cast<const T*>(x.p), x.ld,
                        static_cast<const T*>(w.p), w.ld, (int)M, (int)N, (int)K, per_warp, static_cast<const T*>(e.bias),
                        static_cast<const T*>(e.residual.p), e.residual.ld, e.act, static_cast<T*>(const_cast<void*>(y.p)), y.ld,
                        static_cast<T*>(const_cast<void*>(e.z.p)), e.z.ld);
}
// Warps that share 16 channels (KS): as many as keep all CTAs in one wave (four of eight warps per SM): the longer a
// warp's piece of k, the less its start and the joining weigh, but a second, partial wave costs more.  Few
// channels and a long k: sixteen warps share them, two such CTAs per SM.  One token, KS = 1, 2, 4, 8, 16, in us: 3072 -> 18432 40.8, 26.1,
// 21.2, 22.9, 23.4; 5120 -> 5120 66, 37, 21.8, 14.2, 16.9; 8960 -> 1536 122, 63, 36, 19.2, 11.8; 512 -> 40000 10.9, 12.3, 10.2, 11.4, 17.5.
template <typename T>
static dvdq_status launch_linear_few(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinEpilogue& e,
                                     const LinMatrix& y, cudaStream_t st) {
    const int64_t groups = ceil_div(N, 16), wave = 148 * 4 * 8;
    if (groups <= 148 * 2 && K >= 1024) return cuda_status(launch_linear_few_w<T, 16, 16>(x, w, M, N, K, e, y, st));
    if (groups * 8 <= wave) return cuda_status(launch_linear_few_w<T, 8, 8>(x, w, M, N, K, e, y, st));
    if (groups * 4 <= wave) return cuda_status(launch_linear_few_w<T, 8, 4>(x, w, M, N, K, e, y, st));
    if (groups * 2 <= wave) return cuda_status(launch_linear_few_w<T, 8, 2>(x, w, M, N, K, e, y, st));
    return cuda_status(launch_linear_few_w<T, 8, 1>(x, w, M, N, K, e, y, st));
}

// Rows of a CTA: 16, fewer where that leaves SMs with little to do.  32, 16, 8, 4, 2 rows: 4 tokens 5120 -> 5120 14.5, 10.0, 10.9, 12.7,
// 17.9 us, 1536 -> 1536 5.0, 3.8, 3.2, 3.6, 3.8.
inline int few_rows(int64_t N, int64_t cols) {
    int rows = kFewRows;
    while (rows > 4 && ceil_div(N, rows) * cols < 148 * 4) rows /= 2;
    return rows;
}
template <typename T, int MT>
static dvdq_status launch_linear_few_dw(const LinMatrix& dy, const LinMatrix& z, const LinMatrix& x, int64_t M, int64_t N, int64_t K, int act,
                                        const LinMatrix& dw, float* db, cudaStream_t st) {
    const unsigned cols = dw.p ? (unsigned)ceil_div(K, kFewCols) : 1u;
    const int rows = few_rows(N, cols);
    return cuda_status(launch_after(linear_few_dw_kernel<T, MT>, dim3((unsigned)ceil_div(N, rows), cols), dim3(128), 0, st,
                                    static_cast<const T*>(dy.p), dy.ld, static_cast<const T*>(z.p), z.ld, act, static_cast<const T*>(x.p), x.ld, (int)M,
                                    (int)N, (int)K, rows, static_cast<T*>(const_cast<void*>(dw.p)), dw.ld, db));
}

}  // namespace dvdq
