// The gradients of the RMS norm (rms_norm.cuh):
//
//   dh = gamma dy,  dx = q (dh - hh mean(dh hh)) + the residual stream's own gradient,  dgamma = sum over rows of dy hh,  hh = h q
//
// Laid out as the forward pass: a thread's channels are the same from row to row, so that dgamma's sums and gamma stay with it; each CTA
// then writes one row of sums, and a second kernel adds those (few rows: dgamma by columns, below).  Bound by memory (dy, h, dh in, dx out): many rows come through a ring of cp.async, since
// sums, gamma and inputs together leave too few warps to hide a row's latency.  Measured: 32760 x 5120 bf16 with dh 196 us (1342 MB, 6.8 TB/s),
// 10000 x 16384 204 us (6.4 TB/s), 32760 x 12 heads of 128 53 us (5.7 TB/s), 20000 x 1541 (odd: single elements, no ring) 110 us (2.2 TB/s).
#pragma once

#include "rms_rows.cuh"

namespace dvdq {

struct RmsBackwardArgs {
    RowsShape shape;
    RowsOf dy, h, dh, dx;
    const void* gamma;
    const float* rstd;
    float* part;           // [CTAs, C]: each CTA's sums for dgamma; or NULL
    float* dgamma;         // of the first column_ctas CTAs, which form it of columns; or NULL
    int column_ctas;
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
// V sums on 16 bytes (whole rows: C is a multiple of V, which is 4 or 8)
template <int V>
__device__ __forceinline__ void sums_store(float* p, const Pairs<V>& f) {
#pragma unroll
    for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(f.get(j), f.get(j + 1), f.get(j + 2), f.get(j + 3));
}

// Few rows: no sums of CTAs and no second kernel. Given rstd, dgamma needs nothing of a row's other channels, so that CTAs of their own form it,
// 32 or 64 bytes of each row, while the others form dx; dy and h are read twice, the second time from L2. In a graph, by columns and by sums of CTAs, in us:
// 64 x 1536 bf16 1.8, 3.5; 509 x 1536 4.4, 8.1; 590 x 2560 5.0, 15.4; 512 x 5120 8.7, 17.4; 500 x 16384 30, 33; 509 x 1541 (single elements) 6.6, 6.7.
template <typename T, int V>
__host__ __device__ constexpr int column_lanes() { return V * sizeof(T) == 16 ? 4 : V * sizeof(T) == 2 ? 16 : 8; }
constexpr int kColumnsBelow = 148 * 4;  // rows; from there on the ring
constexpr int kColumnRows = 24;  // of a lane at most: its sum is one in fp32

template <typename T, int V>
__device__ __forceinline__ void rms_norm_columns(const RmsBackwardArgs& A, double* sums) {
    constexpr int LN = column_lanes<T, V>(), COLS = LN * V, U = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    const int C = A.shape.C, c = ((int)blockIdx.x * LN + lane % LN) * V;
    const uint32_t rows = (uint32_t)A.shape.rows, step = (uint32_t)warps * (32 / LN);
    Pairs<V> acc;
#pragma unroll
    for (int j = 0; j < Pairs<V>::N; ++j) acc.p[j] = 0ull;
    auto run = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        for (uint32_t at = (uint32_t)(warp * (32 / LN) + lane / LN); at < rows; at += U * step) {
            Piece<T, V> a[U], b[U];
            float q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t row = at + u * step;
                q[u] = 0.f;
                a[u].clear();
                b[u].clear();
                if (row < rows) {
                    const uint32_t n = A.shape.by_s(row), s = row - n * (uint32_t)A.shape.S;
                    a[u] = row_load<T, V, W>(static_cast<const T*>(A.dy.p) + row_at(A.dy, n, s), c, C);
                    b[u] = row_load<T, V, W>(static_cast<const T*>(A.h.p) + row_at(A.h, n, s), c, C);
                    q[u] = A.rstd[row];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Pairs<V> d = a[u].wide(), h = b[u].wide();
#pragma unroll
                for (int j = 0; j < Pairs<V>::N; ++j) acc.p[j] = f2_fma(d.p[j], f2_mul(h.p[j], f2_splat(q[u])), acc.p[j]);
            }
        }
    };
    if (c + V <= C) run(Whole());
    else if (c < C) run(Part());
    __syncwarp();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        double t = acc.get(j);
#pragma unroll
        for (int o = LN; o < 32; o *= 2) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
        if (lane < LN) sums[warp * COLS + lane * V + j] = t;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < COLS; i += blockDim.x) {
        double t = 0.0;
        for (int w = 0; w < warps; ++w) t += sums[w * COLS + i];
        if ((int)blockIdx.x * COLS + i < C) A.dgamma[blockIdx.x * COLS + i] = (float)t;
    }
}

// Registers of a thread, and with them threads of a CTA at most.
__host__ __device__ constexpr int rows_registers_backward(int V, int P) { return P * V > 40 ? 255 : P * V > 24 ? 168 : P * V > 8 ? 128 : 64; }
__host__ __device__ constexpr int rows_threads_backward(int V, int P) { return 65536 / rows_registers_backward(V, P) / 32 * 32; }

// A thread's channels are the same in every row that it meets, so dgamma's sums stay with it (P > 0: in registers; P = 0: in the CTA's own
// row of `part`) until the CTA has been through its rows.  FULL: dX is asked for, and every thread has P whole pieces.
// COLUMNS: the first CTAs are those of dgamma's columns (their code in the others' kernel costs those 8 registers).
template <typename T, int V, int P, bool WIDE, bool FULL, bool COLUMNS>
__global__ void __maxnreg__(rows_registers_backward(V, P))
rms_norm_backward_kernel(const __grid_constant__ RmsBackwardArgs A) {
    constexpr int N = Pairs<V>::N, K = P > 0 ? P : 1, U = !WIDE && P > 0 && P <= 2 ? 2 : 1;
    constexpr bool KEEP = P > 0 && P * V <= 16;
    constexpr int KIND = (FULL ? kFull : 0) | (WIDE ? kWide : 0);
    __shared__ float2 slots[64];
    extern __shared__ __align__(16) float joined[];
    if constexpr (COLUMNS)
        if ((int)blockIdx.x < A.column_ctas) {
            wait_predecessor();
            release_successor();
            rms_norm_columns<T, V>(A, reinterpret_cast<double*>(joined));
            return;
        }
    const int before = COLUMNS ? A.column_ctas : 0, cta = (int)blockIdx.x - before, ctas = (int)gridDim.x - before;
    const int lanes = WIDE ? (int)blockDim.x : A.lanes, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    const int groups = WIDE ? 1 : kSmallThreads >> A.lanes_log2, group = WIDE ? 0 : (int)threadIdx.x >> A.lanes_log2;
    const int C = A.shape.C;
    const bool with_dx = FULL || A.dx.p != nullptr, with_dh = with_dx && A.dh.p != nullptr;
    const RowLanes<V, P, KIND> L(C, lanes, lane);
    RowMeet<WIDE> meet(slots, lanes);
    Pairs<V> acc[K + 1];
#pragma unroll
    for (int i = 0; i <= K; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i].p[j] = 0ull;
    float* mine = !COLUMNS && A.part ? A.part + (int64_t)cta * C : nullptr;
    wait_predecessor();
    release_successor();
    RowGamma<T, V, P, KIND, KEEP> gamma;
    gamma.init(L, A.gamma, A.params_f32);
    bool first = true;
    for (int64_t at = (int64_t)cta * (groups * U); at < A.shape.rows; at += (int64_t)ctas * (groups * U)) {
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
#pragma unroll 2
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
                if constexpr (FULL) {
                    sums_store<V>(to + L.channel(i), acc[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) to[L.channel(i) + j] = acc[i].get(j);
                }
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

// Many rows of whole pieces (C a multiple of V), a CTA each: the next row's pieces are on their way (cp.async, into slots of shared memory that are a thread's own: no
// barrier) while this one's two passes read theirs from there.  Held in registers instead, inputs and sums leave an SM 10 warps, with nothing
// in flight while they compute: 32760 x 5120 266 us.
// A slot is asked for again only after both passes' stores, whose values came from it, have been issued.
__host__ __device__ constexpr int ring_registers(int P) { return P <= 3 ? 96 : P == 4 ? 128 : 80 + 16 * P; }
__host__ __device__ constexpr int ring_threads(int P) { return 65536 / ring_registers(P) / 32 * 32; }
// FULL: every thread has P pieces.
template <typename T, int V, int P, bool FULL>
__global__ void __maxnreg__(ring_registers(P))
rms_norm_backward_ring_kernel(const __grid_constant__ RmsBackwardArgs A) {
    constexpr int N = Pairs<V>::N;
    __shared__ float2 slots[64];
    extern __shared__ __align__(16) uint8_t ring[];
    const int lanes = (int)blockDim.x, lane = (int)threadIdx.x, C = A.shape.C;
    constexpr int KIND = (FULL ? kFull : 0) | kWide;
    const RowLanes<V, P, KIND> L(C, lanes, lane);
    RowMeet<true> meet(slots, lanes);
    Pairs<V> acc[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i].p[j] = 0ull;
    const bool with_dh = A.dh.p != nullptr;
    // a tensor's pieces as they lie in the row: a thread's are 512 bytes apart
    constexpr uint32_t step = 512u;
    const uint32_t tensor = (uint32_t)(P * lanes) * 16u, stage_bytes = (with_dh ? 3u : 2u) * tensor, mine = smem_u32(ring) + (uint32_t)L.first * 16u;
    auto ask = [&](int64_t row, uint32_t stage) {
        if (row < A.shape.rows) {
            const uint32_t n = A.shape.by_s((uint32_t)row), s = (uint32_t)row - n * (uint32_t)A.shape.S;
            uint32_t to = mine + stage * stage_bytes;
            auto copy = [&](const RowsOf& t) {
                const T* from = static_cast<const T*>(t.p) + row_at(t, n, s) + L.channel(0);
#pragma unroll
                for (int i = 0; i < P; ++i)
                    if (L.has(i)) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * step), "l"(from + i * (32 * V)) : "memory");
                to += tensor;
            };
            copy(A.dy);
            copy(A.h);
            if (with_dh) copy(A.dh);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    wait_predecessor();
    release_successor();
    RowGamma<T, V, P, KIND, true> gamma;
    gamma.init(L, A.gamma, A.params_f32);
    int64_t row = blockIdx.x;
    uint32_t stage = 0;
    ask(row, 0u);
    float q_next = A.rstd[row];
    for (; row < A.shape.rows; row += gridDim.x, stage ^= 1u) {
        const float q = q_next;
        ask(row + gridDim.x, stage ^ 1u);
        if (row + gridDim.x < A.shape.rows) q_next = A.rstd[row + gridDim.x];
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        const uint32_t at = mine + stage * stage_bytes;
        uint64_t sum = 0ull;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!L.has(i)) continue;
            Piece<T, V> d, h;
            d.load_shared(at + i * step);
            h.load_shared(at + tensor + i * step);
            add_to<V>(acc[i], row_terms<V>(d.wide(), h.wide(), gamma.template get<true>(i, L.channel(i)), q, sum));
        }
        float s0, s1;
        f2_unpack(sum, s0, s1);
        const float mean = meet(s0 + s1, 0.f, false).x * A.inv_c;
        const uint32_t n = A.shape.by_s((uint32_t)row), s = (uint32_t)row - n * (uint32_t)A.shape.S;
        T* dx = static_cast<T*>(A.dx.p) + row_at(A.dx, n, s);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!L.has(i)) continue;
            Piece<T, V> d, h, e;
            d.load_shared(at + i * step);
            h.load_shared(at + tensor + i * step);
            Pairs<V> o = row_gradient<V>(d.wide(), h.wide(), gamma.template get<true>(i, L.channel(i)), q, mean);
            if (with_dh) {
                e.load_shared(at + 2 * tensor + i * step);
                add_to<V>(o, e.wide());
            }
            row_store<T, V, true>(dx, L.channel(i), C, o, true);
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!A.part) return;
    float* to = A.part + (int64_t)blockIdx.x * C;
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (L.has(i)) sums_store<V>(to + L.channel(i), acc[i]);
}

// dgamma from the CTAs' sums, in fp64 and in a fixed order: COLS channels a CTA, whose other threads share the rows of sums.  Eight channels, where that
// is a wave or less (with 32 of them 592 rows of 128 sums took 6 us longer: too few loads in flight), otherwise 32.
constexpr int kJoinThreads = 1024;
template <int COLS>
static __global__ void __launch_bounds__(kJoinThreads) rms_norm_join_kernel(const float* __restrict__ part, int parts, int C, float* __restrict__ out) {
    constexpr int kRows = kJoinThreads / COLS;  // rows of sums side by side
    __shared__ double sh[32][COLS];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = threadIdx.x % COLS, c = blockIdx.x * COLS + col;
    wait_predecessor();
    release_successor();
    double t = 0.0;
    if (c < C) {
#pragma unroll 8
        for (int i = threadIdx.x / COLS; i < parts; i += kRows) t += part[(int64_t)i * C + c];
    }
#pragma unroll
    for (int o = COLS; o < 32; o *= 2) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    if (lane < COLS) sh[w][lane] = t;
    __syncthreads();
    if (w < COLS) {  // a warp for each channel
        t = sh[lane][w];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
        if (lane == 0 && blockIdx.x * COLS + w < C) out[blockIdx.x * COLS + w] = (float)t;
    }
}
inline cudaError_t launch_rms_join(const float* part, int parts, int C, float* out, cudaStream_t st) {
    return C <= 8 * 148 * 2 ? launch_after(rms_norm_join_kernel<8>, dim3((unsigned)ceil_div(C, 8)), dim3(kJoinThreads), 0, st, part, parts, C, out)
                            : launch_after(rms_norm_join_kernel<32>, dim3((unsigned)ceil_div(C, 32)), dim3(kJoinThreads), 0, st, part, parts, C, out);
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

// dgamma by columns: few rows of a lane (at_once: rows that a CTA's lanes take side by side), and few enough bytes for their second reading. Above 16 MB, and 2 MB of
// single elements, the sums of CTAs cost less: 590 x 8960 fp32 20 us, 27 by columns; 300 x 2049 fp32 7.3, 8.3; 500 x 5121 bf16 25, 32.
inline bool rms_by_columns(int64_t rows, int64_t C, int bytes, int v, int at_once) {
    return rows < kColumnsBelow && ceil_div(rows, at_once) <= kColumnRows && rows * C * bytes <= (int64_t)(v > 2 ? 16 : 2 * v) << 20;
}

// Whether that is built for P pieces that fill a CTA's threads: those that the fewest rounds (launch_rms_backward_v) ever choose.
__host__ __device__ constexpr bool full_columns(int V, int P) { return V == 8 ? P != 2 && P != 6 : P != 4; }

template <typename T, int V, int P, bool WIDE, bool FULL>
static cudaError_t launch_rms_backward_p(const RmsBackwardArgs& A0, const RowsPlan& p, int64_t parts, int* ctas_out, cudaStream_t st) {
    RmsBackwardArgs A = A0;
    A.lanes = p.lanes;
    A.lanes_log2 = p.lanes_log2;
    const int groups = WIDE ? 1 : kSmallThreads / p.lanes;
    const int64_t all = ceil_div(A.shape.rows, groups);
    if constexpr (P > 0 && !(WIDE && FULL && !full_columns(V, P))) {
        constexpr int LN = column_lanes<T, V>();
        if (A.dgamma && rms_by_columns(A.shape.rows, A.shape.C, (int)sizeof(T), V, p.threads / LN)) {
            auto kern = rms_norm_backward_kernel<T, V, P, WIDE, FULL, true>;
            const int columns = (int)ceil_div(A.shape.C, LN * V);
            const size_t sums = (size_t)(p.threads / 32) * LN * V * 8;
            A.part = nullptr;
            A.column_ctas = columns;
            *ctas_out = 0;
            if (!A.dx.p) return launch_after(kern, dim3((unsigned)columns), dim3(p.threads), sums, st, A);
            if (A.dx.p != A.dy.p && A.dx.p != A.h.p) return launch_after(kern, dim3((unsigned)(columns + all)), dim3(p.threads), sums, st, A);
            const cudaError_t e = launch_after(kern, dim3((unsigned)columns), dim3(p.threads), sums, st, A);  // in place the columns come first
            if (e != cudaSuccess) return e;
            A.column_ctas = 0;
            return launch_after(kern, dim3((unsigned)all), dim3(p.threads), 0, st, A);
        }
    }
    auto kern = rms_norm_backward_kernel<T, V, P, WIDE, FULL, false>;
    static PerDevice<RowsHeld> cache;
    const int held = rows_held(cache, kern, p.threads);
    if (held == 0) return cudaErrorInvalidValue;
    int64_t ctas = all < 148 * held ? all : 148 * held;
    if (A.part && ctas > parts) ctas = parts;
    *ctas_out = (int)ctas;
    const size_t sums = A.part && groups > 1 ? (size_t)groups * A.shape.C * 4 : 0;  // of 128 threads with 8 pieces at most: 32 KB
    return launch_after(kern, dim3((unsigned)ctas), dim3(p.threads), sums, st, A);
}
template <typename T, int V, int P, bool FULL>
static cudaError_t launch_rms_backward_w(const RmsBackwardArgs& A, const RowsPlan& p, int64_t parts, int* ctas, cudaStream_t st) {
    return p.wide ? launch_rms_backward_p<T, V, P, true, FULL>(A, p, parts, ctas, st) : launch_rms_backward_p<T, V, P, false, FULL>(A, p, parts, ctas, st);
}
constexpr int kRingRoom = 216 * 1024;  // of an SM's shared memory, for its CTAs' rings
// The ring's plan: pieces of a thread such that they fill a CTA; or 2 or 4 that do not; or none.  Two, where that is two warps or more, are the best (32760 x
// 5120, 2, 4 pieces: 200, 206 us; 2048: 85, 91; 20000 x 2560: 68, 86), but not three warps, which leave one of an SM's four schedulers idle (1536: 91 us, 69 with 3 pieces
// in two warps).
struct BackwardRing {
    int pieces, threads;
    bool full;
};
inline BackwardRing backward_ring(int64_t rows, int64_t nv, int tensors) {
    if (rows < 148 * 4 || 2 * tensors * (nv + 128) * 16 > kRingRoom) return {0, 0, false};  // threads beyond the row have slots too
    static const int order[] = {2, 4, 3, 5, 6, 7, 8, 0};
    for (const int* k = order; *k; ++k)
        if (nv % (32 * *k) == 0 && nv / *k >= 64 && nv / *k != 96 && nv / *k <= ring_threads(*k)) return {*k, (int)(nv / *k), true};
    // pieces that do not fill the threads: four in up to 224 threads if three quarters of the slots are used, else two (2, 4: 20000 x 1544 58.6, 51.4 us; 30000 x
    // 2052 fp32 245, 171; 5000 x 8008 65.5, 73.0; 32760 x 1200, whose 150 pieces take 256 slots with four, 63.5 with two, 97 without a ring)
    if (nv < 128) return {0, 0, false};
    const int64_t four = align_up(ceil_div(nv, 4), 32), two = align_up(ceil_div(nv, 2), 32);
    if (four >= 64 && four <= 224 && four * 3 <= nv) return {4, (int)four, false};
    if (two <= ring_threads(2)) return {2, (int)two, false};
    if (four <= ring_threads(4)) return {4, (int)four, false};
    return {0, 0, false};
}
template <typename T, int V, int P, bool FULL>
static cudaError_t launch_rms_backward_ring(const RmsBackwardArgs& A, int threads, int64_t parts, int* ctas_out, cudaStream_t st) {
    const int smem = 2 * (A.dh.p ? 3 : 2) * P * threads * 16;
    if (smem > kRingRoom) return cudaErrorInvalidValue;  // not reached
    auto kern = rms_norm_backward_ring_kernel<T, V, P, FULL>;
    static PerDevice<int> ready;
    if (!ready.get([&](int&, int) { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingRoom) == cudaSuccess; }))
        return cudaErrorInvalidValue;
    int held = kRingRoom / (smem + 1536);                                   // 1 KB that the system takes, and the slots
    const int by_registers = 65536 / (ring_registers(P) * threads);
    if (held > by_registers) held = by_registers;
    if (held < 1) held = 1;
    // with dgamma three rows a CTA at least: its sums, written and read, are as many bytes as a row (with up to 148 * held CTAs, three rows, eight, in us:
    // 600 x 1536 9.4, 6.3, 7.3; 1000 x 1536 11.1, 8.7, 10.0; 2000 x 1536 14.9, 13.2, 12.5; 4000 x 1536 17.5, 16.9, 19.6)
    const int64_t most = A.part ? ceil_div(A.shape.rows, 3) : A.shape.rows;
    int64_t ctas = most < 148 * held ? most : 148 * held;
    if (A.part && ctas > parts) ctas = parts;
    *ctas_out = (int)ctas;
    return launch_after(kern, dim3((unsigned)ctas), dim3(threads), (size_t)smem, st, A);
}
template <typename T, int V>
static cudaError_t launch_rms_backward_v(const RmsBackwardArgs& A, int64_t parts, int* ctas, cudaStream_t st) {
    constexpr bool kPieces16 = V * sizeof(T) == 16;
    if constexpr (kPieces16) {
        const BackwardRing r = A.dx.p && A.shape.C % V == 0 ? backward_ring(A.shape.rows, A.shape.C / V, A.dh.p ? 3 : 2) : BackwardRing{0, 0, false};
        if (r.full) {
            switch (r.pieces) {
                case 2: return launch_rms_backward_ring<T, V, 2, true>(A, r.threads, parts, ctas, st);
                case 3: return launch_rms_backward_ring<T, V, 3, true>(A, r.threads, parts, ctas, st);
                case 4: return launch_rms_backward_ring<T, V, 4, true>(A, r.threads, parts, ctas, st);
                case 5: return launch_rms_backward_ring<T, V, 5, true>(A, r.threads, parts, ctas, st);
                case 6: return launch_rms_backward_ring<T, V, 6, true>(A, r.threads, parts, ctas, st);
                case 7: return launch_rms_backward_ring<T, V, 7, true>(A, r.threads, parts, ctas, st);
                default: return launch_rms_backward_ring<T, V, 8, true>(A, r.threads, parts, ctas, st);
            }
        }
        if (r.pieces == 2) return launch_rms_backward_ring<T, V, 2, false>(A, r.threads, parts, ctas, st);
        if (r.pieces == 4) return launch_rms_backward_ring<T, V, 4, false>(A, r.threads, parts, ctas, st);
    }
    // Rows whose pieces do not fill the threads: 4 (20000 x 1541, odd: 1, 2, 4, 8 pieces 478, 196, 119, 186 us; 30000 x 2049 fp32 666, 665, 333, 368).
    static const int order[] = {5, 3, 4, 2, 6, 7, 8, 1, 0};
    RowsPlan p = rows_plan(A.shape.rows, ceil_div(A.shape.C, V), kPieces16 && A.shape.C % V == 0 && A.dx.p, 2, 8, 4,
                                 [](int k) { return rows_threads_backward(V, k); }, order);
    if constexpr (kPieces16) {
        // Few rows, dgamma by columns: the pieces with which the CTAs of rows and columns come in the fewest rounds, and of those the fewest
        // (1, 2, 5 pieces: 509 x 1536 4.5, 8.4 (3 pieces), - us; 512 x 5120 11.1, 11.4, 9.3; 590 x 2560 5.4, 15.5 (5, which is too few threads for columns))
        if (p.full && p.wide && A.dgamma && A.shape.rows < kColumnsBelow) {
            const int64_t nv = A.shape.C / V, ctas = A.shape.rows + ceil_div(nv, column_lanes<T, V>());
            int64_t least = INT64_MAX;
            for (int k = 1; k <= 8; ++k) {
                const int64_t threads = nv / k;
                if (!full_columns(V, k) || nv % (32 * k) != 0 || threads < 64 || threads > kRowThreads || threads > rows_threads_backward(V, k)) continue;
                if (!rms_by_columns(A.shape.rows, A.shape.C, (int)sizeof(T), V, (int)threads / column_lanes<T, V>())) continue;
                const int64_t rounds = ceil_div(ctas, 148 * (65536 / (rows_registers_backward(V, k) * threads)));
                if (rounds >= least) continue;
                least = rounds;
                p.pieces = k;
                p.lanes = p.threads = (int)threads;
            }
        }
        if (p.full) {  // rows of a warp or less (at most 64 pieces) come in 1, 2, 3 or 5 a thread
            switch (p.pieces) {
                case 1: return launch_rms_backward_w<T, V, 1, true>(A, p, parts, ctas, st);
                case 2: return launch_rms_backward_w<T, V, 2, true>(A, p, parts, ctas, st);
                case 3: return launch_rms_backward_w<T, V, 3, true>(A, p, parts, ctas, st);
                case 4: return launch_rms_backward_p<T, V, 4, true, true>(A, p, parts, ctas, st);
                case 5: return launch_rms_backward_w<T, V, 5, true>(A, p, parts, ctas, st);
                case 6: return launch_rms_backward_p<T, V, 6, true, true>(A, p, parts, ctas, st);
                case 7: return launch_rms_backward_p<T, V, 7, true, true>(A, p, parts, ctas, st);
                default: return launch_rms_backward_p<T, V, 8, true, true>(A, p, parts, ctas, st);
            }
        }
    }
    switch (p.pieces) {
        case 0: return launch_rms_backward_p<T, V, 0, true, false>(A, p, parts, ctas, st);
        case 1: return launch_rms_backward_w<T, V, 1, false>(A, p, parts, ctas, st);
        case 2: return launch_rms_backward_w<T, V, 2, false>(A, p, parts, ctas, st);
        case 4: return launch_rms_backward_w<T, V, 4, false>(A, p, parts, ctas, st);
        default: return cudaErrorInvalidValue;  // not reached
    }
}
template <typename T>
static cudaError_t launch_rms_backward_t(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st) {
    if (access == 16) return launch_rms_backward_v<T, 16 / sizeof(T)>(A, parts, ctas, st);
    if (sizeof(T) == 2 && access == 4) return launch_rms_backward_v<T, 4 / sizeof(T)>(A, parts, ctas, st);
    return launch_rms_backward_v<T, 1>(A, parts, ctas, st);
}

}  // namespace dvdq
