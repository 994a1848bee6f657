// The gradients of the RMS norm (rms_norm.cuh):
//
//   dh = gamma dy,  dx = q (dh - hh mean(dh hh)) + the residual stream's own gradient,  dgamma = sum over rows of dy hh,  hh = h q
//
// Laid out as the forward pass: a row in registers, its threads' channels the same from row to row, so that dgamma's sums stay with
// them; each CTA then writes one row of sums, and a second kernel adds those.  Bound by memory: dy, h, dh in, dx out.
#pragma once

#include "rms_rows.cuh"

namespace dvdq {

struct RmsBackwardArgs {
    RowsShape shape;
    RowsOf dy, h, dh, dx;
    const void* gamma;
    const float* rstd;
    float* part;           // [CTAs, C]: each CTA's sums for dgamma; or NULL
    int params_f32;
    float inv_c;
    int lanes, lanes_log2;
};

// q (gamma dy - h (q mean))
template <int V>
__device__ __forceinline__ Pairs<V> row_gradient(const Pairs<V>& d, const Pairs<V>& h, const Pairs<V>& g, float q, float mean) {
    Pairs<V> o;
    const uint64_t along = f2_splat(-q * mean);
#pragma unroll
    for (int j = 0; j < Pairs<V>::N; ++j) o.p[j] = f2_mul(f2_fma(h.p[j], along, f2_mul(d.p[j], g.p[j])), f2_splat(q));
    return o;
}
// What one piece adds to dgamma, and to the row's <dh hh>.
template <int V>
__device__ __forceinline__ Pairs<V> row_terms(const Pairs<V>& d, const Pairs<V>& h, const Pairs<V>& g, float q, uint64_t& sum) {
    Pairs<V> t;
#pragma unroll
    for (int j = 0; j < Pairs<V>::N; ++j) {
        t.p[j] = f2_mul(d.p[j], f2_mul(h.p[j], f2_splat(q)));
        sum = f2_fma(t.p[j], g.p[j], sum);
    }
    return t;
}
__host__ __device__ constexpr int rows_threads_backward(int V, int P) { return P * V > 16 ? 256 : P * V > 4 ? 512 : kRowThreads; }

// A thread's channels are the same in every row that it meets, so dgamma's sums stay with it (P > 0: in registers; P = 0: in the CTA's own
// row of `part`) until the CTA has been through its rows.  FULL: dX is asked for, and every thread has P whole pieces.
template <typename T, int V, int P, bool WIDE, bool FULL>
__global__ void __launch_bounds__(WIDE ? rows_threads_backward(V, P) : kSmallThreads)
rms_norm_backward_kernel(const __grid_constant__ RmsBackwardArgs A) {
    constexpr int N = Pairs<V>::N, K = P > 0 ? P : 1, U = !WIDE && P > 0 && P <= 2 ? 2 : 1;
    constexpr bool KEEP = P > 0 && P * V <= 16;
    __shared__ float2 slots[64];
    extern __shared__ float joined[];
    const int lanes = WIDE ? (int)blockDim.x : A.lanes, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    const int groups = WIDE ? 1 : kSmallThreads >> A.lanes_log2, group = WIDE ? 0 : (int)threadIdx.x >> A.lanes_log2;
    const int C = A.shape.C;
    const bool with_dx = FULL || A.dx.p != nullptr, with_dh = with_dx && A.dh.p != nullptr;
    const RowLanes<V, P, FULL> L(C, lanes, lane);
    RowMeet<WIDE> meet(slots, lanes);
    Pairs<V> acc[K + 1];
#pragma unroll
    for (int i = 0; i <= K; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i].p[j] = 0ull;
    float* mine = A.part ? A.part + (int64_t)blockIdx.x * C : nullptr;
    wait_predecessor();
    release_successor();
    RowGamma<T, V, P, FULL, KEEP> gamma;
    gamma.init(L, A.gamma, A.params_f32);
    bool first = true;
    for (int64_t at = (int64_t)blockIdx.x * (groups * U); at < A.shape.rows; at += (int64_t)gridDim.x * (groups * U)) {
        Piece<T, V> a[U][K + 1], b[U][K + 1], e[U][K + 1];  // dy, h, dh; the last: the row's end
        const T *dy[U], *h[U], *dh[U];
        T* dx[U];
        float q[U];
        bool active[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = at + u * groups + group;
            active[u] = WIDE || row < A.shape.rows;
            const uint32_t index = (uint32_t)(active[u] ? row : at), n = A.shape.by_s(index), s = index - n * (uint32_t)A.shape.S;
            dy[u] = static_cast<const T*>(A.dy.p) + row_at(A.dy, n, s);
            h[u] = static_cast<const T*>(A.h.p) + row_at(A.h, n, s);
            if (with_dh) dh[u] = static_cast<const T*>(A.dh.p) + row_at(A.dh, n, s);
            if (with_dx) dx[u] = static_cast<T*>(A.dx.p) + row_at(A.dx, n, s);
            q[u] = A.rstd[index];
        }
        auto ask = [&](int u, int i, int c, auto whole, bool there) {
            constexpr bool W = decltype(whole)::value;
            if (W && !there) {
                a[u][i].clear();
                b[u][i].clear();
                return;
            }
            a[u][i] = row_load<T, V, W>(dy[u], c, C);
            b[u][i] = row_load<T, V, W>(h[u], c, C);
        };
        auto ask_more = [&](int u, int i, int c, auto whole, bool there) {
            if (there) e[u][i] = row_load<T, V, decltype(whole)::value>(dh[u], c, C);
        };
        // f(u, piece, channel, Whole or Part, whether the piece is there)
        auto visit = [&](int u, auto f) {
            if constexpr (P > 0) {
#pragma unroll
                for (int i = 0; i < P; ++i) f(u, i, L.channel(i), Whole(), active[u] && L.has(i));
                if (!FULL && V > 1 && L.tail && active[u]) f(u, P, L.end(), Part(), true);
            } else {
                for (int p = L.lane; p < L.whole; p += L.lanes) {
                    ask(u, 0, p * V, Whole(), true);
                    f(u, 0, p * V, Whole(), true);
                }
                if (V > 1 && L.tail) {
                    ask(u, 0, L.end(), Part(), true);
                    f(u, 0, L.end(), Part(), true);
                }
            }
        };
        if constexpr (P > 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                visit(u, ask);
                if (with_dh) visit(u, ask_more);
            }
        }
#pragma unroll
        for (int v = 0; v < U; ++v) {
            uint64_t sum = 0ull;
            visit(v, [&](int u, int i, int c, auto whole, bool) {
                const Pairs<V> t = row_terms<V>(a[u][i].wide(), b[u][i].wide(), gamma.template get<decltype(whole)::value>(i, c), q[u], sum);
                if constexpr (P > 0) {
                    add_to<V>(acc[i], t);
                } else if (mine) {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (c + j < C) mine[c + j] = first ? t.get(j) : mine[c + j] + t.get(j);
                }
            });
            first = false;
            if (!with_dx) continue;
            float s0, s1;
            f2_unpack(sum, s0, s1);
            const float mean = meet(s0 + s1, 0.f, false).x * A.inv_c;
            visit(v, [&](int u, int i, int c, auto whole, bool there) {
                constexpr bool W = decltype(whole)::value;
                Pairs<V> o = row_gradient<V>(a[u][i].wide(), b[u][i].wide(), gamma.template get<W>(i, c), q[u], mean);
                if (with_dh) {
                    if constexpr (P == 0) ask_more(u, i, c, whole, there);
                    add_to<V>(o, e[u][i].wide());
                }
                row_store<T, V, W>(dx[u], c, C, o, there);
            });
        }
    }
    if constexpr (P > 0) {
        if (!mine) return;
        // rows that share the CTA: their sums are added up in shared memory
        float* to = groups > 1 ? joined + group * C : mine;
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (L.has(i)) {
#pragma unroll
                for (int j = 0; j < V; ++j) to[L.channel(i) + j] = acc[i].get(j);
            }
        if (!FULL && V > 1 && L.tail) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (L.end() + j < C) to[L.end() + j] = acc[P].get(j);
        }
        if (groups == 1) return;
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            float t = 0.f;
            for (int g = 0; g < groups; ++g) t += joined[g * C + c];
            mine[c] = t;
        }
    }
}

// dgamma from the CTAs' sums, in fp64 and in a fixed order: 32 channels a CTA, 16 warps share its rows.
constexpr int kRmsJoinWarps = 16;
static __global__ void __launch_bounds__(kRmsJoinWarps * 32) rms_norm_join_kernel(const float* __restrict__ part, int parts, int C, float* __restrict__ out) {
    __shared__ double sh[kRmsJoinWarps][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    wait_predecessor();
    release_successor();
    double t = 0.0;
    if (c < C) {
#pragma unroll 8
        for (int i = w; i < parts; i += kRmsJoinWarps) t += part[(int64_t)i * C + c];
    }
    sh[w][lane] = t;
    __syncthreads();
    if (w == 0 && c < C) {
#pragma unroll
        for (int i = 1; i < kRmsJoinWarps; ++i) t += sh[i][lane];
        out[c] = (float)t;
    }
}
static __global__ void __launch_bounds__(256) rms_norm_no_rows_kernel(float* __restrict__ dgamma, int C) {
    wait_predecessor();
    release_successor();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < C) dgamma[c] = 0.f;
}

// CTAs of the backward pass at most, and so rows of its sums for dgamma: 16 MB of them, but one for each SM up to 256 MB.
inline int64_t rms_parts(int64_t rows, int64_t C) {
    int64_t most = ((int64_t)16 << 20) / (4 * C);
    if (most > 148 * 16) most = 148 * 16;
    if (most < 148) most = 148;
    const int64_t room = ((int64_t)256 << 20) / (4 * C);
    if (most > room) most = room;
    return rows < most ? rows : most;
}

// ------------------------------------------------------------------ launches

template <typename T, int V, int P, bool WIDE, bool FULL>
static cudaError_t launch_rms_backward_p(const RmsBackwardArgs& A0, const RowsPlan& p, int64_t parts, int* ctas_out, cudaStream_t st) {
    RmsBackwardArgs A = A0;
    A.lanes = p.lanes;
    A.lanes_log2 = p.lanes_log2;
    auto kern = rms_norm_backward_kernel<T, V, P, WIDE, FULL>;
    static PerDevice<RowsHeld> cache;
    const int held = rows_held(cache, kern, p.threads);
    if (held == 0) return cudaErrorInvalidValue;
    const int groups = WIDE ? 1 : kSmallThreads / p.lanes;
    int64_t ctas = ceil_div(A.shape.rows, groups);
    ctas = ctas < 148 * held ? ctas : 148 * held;
    if (A.part && ctas > parts) ctas = parts;
    *ctas_out = (int)ctas;
    const size_t sums = A.part && groups > 1 ? (size_t)groups * A.shape.C * 4 : 0;  // of 128 threads with 8 pieces at most: 32 KB
    return launch_after(kern, dim3((unsigned)ctas), dim3(p.threads), sums, st, A);
}
template <typename T, int V, int P, bool FULL>
static cudaError_t launch_rms_backward_w(const RmsBackwardArgs& A, const RowsPlan& p, int64_t parts, int* ctas, cudaStream_t st) {
    return p.wide ? launch_rms_backward_p<T, V, P, true, FULL>(A, p, parts, ctas, st) : launch_rms_backward_p<T, V, P, false, FULL>(A, p, parts, ctas, st);
}
template <typename T, int V>
static cudaError_t launch_rms_backward_v(const RmsBackwardArgs& A, int64_t parts, int* ctas, cudaStream_t st) {
    constexpr bool kPieces16 = V * sizeof(T) == 16;
    const RowsPlan p = rows_plan(A.shape.rows, ceil_div(A.shape.C, V), kPieces16 && A.shape.C % V == 0 && A.dx.p, 8, [](int k) { return rows_threads_backward(V, k); });
    if constexpr (kPieces16) {
        if (p.full) {
            switch (p.pieces) {
                case 1: return launch_rms_backward_w<T, V, 1, true>(A, p, parts, ctas, st);
                case 2: return launch_rms_backward_w<T, V, 2, true>(A, p, parts, ctas, st);
                case 3: return launch_rms_backward_w<T, V, 3, true>(A, p, parts, ctas, st);
                case 4: return launch_rms_backward_w<T, V, 4, true>(A, p, parts, ctas, st);
                case 5: return launch_rms_backward_w<T, V, 5, true>(A, p, parts, ctas, st);
                case 6: return launch_rms_backward_w<T, V, 6, true>(A, p, parts, ctas, st);
                case 7: return launch_rms_backward_w<T, V, 7, true>(A, p, parts, ctas, st);
                default: return launch_rms_backward_w<T, V, 8, true>(A, p, parts, ctas, st);
            }
        }
    }
    switch (p.pieces) {
        case 0: return launch_rms_backward_p<T, V, 0, true, false>(A, p, parts, ctas, st);
        case 1: return launch_rms_backward_w<T, V, 1, false>(A, p, parts, ctas, st);
        case 2: return launch_rms_backward_w<T, V, 2, false>(A, p, parts, ctas, st);
        case 4: return launch_rms_backward_w<T, V, 4, false>(A, p, parts, ctas, st);
        default: return launch_rms_backward_w<T, V, 8, false>(A, p, parts, ctas, st);
    }
}
template <typename T>
static cudaError_t launch_rms_backward_t(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st) {
    if (access == 16) return launch_rms_backward_v<T, 16 / sizeof(T)>(A, parts, ctas, st);
    if (sizeof(T) == 2 && access == 4) return launch_rms_backward_v<T, 4 / sizeof(T)>(A, parts, ctas, st);
    return launch_rms_backward_v<T, 1>(A, parts, ctas, st);
}

}  // namespace dvdq
