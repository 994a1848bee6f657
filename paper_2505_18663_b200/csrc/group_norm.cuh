// Group norm with an activation, channels last: x [N, S, C], groups of C / G neighbouring channels,
//
//   h = (x - mean) rstd,  z = gamma_c h + beta_c,  y = act(z)        mean, rstd over a group's S C/G values
//   dz = dy act'(z),  dh = gamma_c dz,  dx = rstd (dh - <dh> - h <dh h>),  <.> the mean over the group,
//   dgamma_c = sum dz h,  dbeta_c = sum dz                           over samples and places
//
// What bounds it: reading x (and dy) and writing y (dx).  The statistics need all of a sample
// before its first output, so a tensor larger than the chip's shared memory is read twice; the
// second pass walks every chunk backwards, so that it begins with what the L2 cache still holds.
//
// Two launches.  Pass 1: a CTA sums one chunk of places of one sample over all channels (a thread keeps
// its 16 bytes of channels, so its loads are whole sectors) and writes two numbers per group.
// Pass 2: every CTA adds up its sample's chunks in a fixed order (no atomics: the same bits every
// time), then streams its chunk.  It is launched while pass 1 drains.  Sums are of x minus a value
// of the group itself (the first place's first channel), so that a mean far from zero costs no
// digits, in fp32 within a chunk and in fp64 across chunks.
#pragma once

#include "block_common.cuh"

namespace dvdq {

constexpr int kGnThreads = 256;
constexpr int kGnMaxVecs = kGnThreads;  // channel vectors of one CTA; wider rows are cut into channel blocks

struct GnArgs {
    const void* x;
    const void* dy;          // backward
    void* y;                 // forward: y; backward: dx
    const void* gamma;
    const void* beta;
    float* mean;             // [N, G]: written (forward, may be NULL) or read (backward)
    float* rstd;
    float* dgamma;
    float* dbeta;
    float2* part;            // [N, chunks, G]
    float* pivot;            // [N, G]: what pass 1 subtracted (y may be x: pass 2 cannot read it there)
    float2* part_c;          // backward: [N, chunks, C]
    int64_t xn, xs, dn, ds, yn, ys;  // pitches of samples and places, elements
    int64_t S;
    int N, C, G, per;        // per = C / G
    int chunks;              // chunks of places per sample
    int64_t rows;            // places per chunk
    int vecs, lanes;         // channel vectors of a CTA (its channel block), rows it walks side by side
    int blocks;              // channel blocks: each some whole groups, or (bpg > 1) a piece of one group
    int bpg;                 // blocks per group
    int params_f32, params_bf16;
    float eps;
};

__device__ __forceinline__ float gn_param(const void* p, int f32, int bf16, int c, float none) {
    if (!p) return none;
    if (f32) return static_cast<const float*>(p)[c];
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[c]) : __half2float(static_cast<const __half*>(p)[c]);
}

// Where this thread works: channel vector v of its CTA's channel block, row r of `lanes` side by side.
template <int V>
struct GnPlace {
    int cbase, here;  // the block's first channel, its channels
    int g0, g1;       // the groups it belongs to
    int v, c0;        // this thread's vector in the block, its first channel
    int r;
    bool on;
    int64_t s0, s1;
    __device__ __forceinline__ GnPlace(const GnArgs& A) {
        const int width = A.vecs * V;
        if (A.bpg == 1) {
            cbase = blockIdx.z * width;
            here = min(A.C - cbase, width);
            g0 = cbase / A.per;
            g1 = g0 + here / A.per;
        } else {
            g0 = blockIdx.z / A.bpg;
            g1 = g0 + 1;
            const int sub = blockIdx.z - g0 * A.bpg;
            cbase = g0 * A.per + sub * width;
            here = min(A.per - sub * width, width);
        }
        v = threadIdx.x % A.vecs;
        r = threadIdx.x / A.vecs;
        c0 = cbase + v * V;
        on = r < A.lanes && v * V < here;
        s0 = (int64_t)blockIdx.x * A.rows;
        s1 = s0 + A.rows < A.S ? s0 + A.rows : A.S;
    }
};

// Adds up [lanes][vecs * V] pairs in shared memory over the lanes, then over the channels of each group
// in this block, and writes one pair per group (and per channel).
template <int V, bool PER_CHANNEL>
__device__ __forceinline__ void gn_reduce_block(const GnArgs& A, const GnPlace<V>& P, const float (&s1)[V], const float (&s2)[V], float2* sh) {
    const int width = A.vecs * V;
    if (P.on) {
#pragma unroll
        for (int i = 0; i < V; ++i) sh[P.r * width + P.v * V + i] = make_float2(s1[i], s2[i]);
    }
    __syncthreads();
    const int64_t slot = (int64_t)blockIdx.y * A.chunks + blockIdx.x;
    for (int c = threadIdx.x; c < P.here; c += kGnThreads) {
        float2 t = sh[c];
        for (int l = 1; l < A.lanes; ++l) {
            const float2 u = sh[l * width + c];
            t.x += u.x;
            t.y += u.y;
        }
        if (PER_CHANNEL) {
            A.part_c[slot * A.C + P.cbase + c] = t;
            const float g = gn_param(A.gamma, A.params_f32, A.params_bf16, P.cbase + c, 1.0f);
            t.x *= g;
            t.y *= g;
        }
        sh[c] = t;
    }
    __syncthreads();
    const int groups = P.g1 - P.g0, span = A.bpg == 1 ? A.per : P.here;
    float2* out = A.part + slot * (A.G * A.bpg) + (A.bpg == 1 ? P.g0 : (int)blockIdx.z);
    if (span <= 8) {
        for (int g = threadIdx.x; g < groups; g += kGnThreads) {
            float2 t = sh[g * span];
            for (int i = 1; i < span; ++i) {
                t.x += sh[g * span + i].x;
                t.y += sh[g * span + i].y;
            }
            out[g] = t;
        }
    } else {  // wide groups: a warp each
        for (int g = threadIdx.x >> 5; g < groups; g += kGnThreads / 32) {
            float2 t = make_float2(0.f, 0.f);
            for (int i = threadIdx.x & 31; i < span; i += 32) {
                t.x += sh[g * span + i].x;
                t.y += sh[g * span + i].y;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, o);
                t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, o);
            }
            if ((threadIdx.x & 31) == 0) out[g] = t;
        }
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kGnThreads) gn_stats_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ float2 sh[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    float s1[V], s2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.f;
    if (P.on) {
        const T* base = static_cast<const T*>(A.x) + (int64_t)n * A.xn;
        float pv[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = (P.c0 + i) / A.per;
            pv[i] = to_f32(base[g * A.per]);
            if (blockIdx.x == 0 && P.r == 0 && P.c0 + i == g * A.per) A.pivot[(int64_t)n * A.G + g] = pv[i];
        }
        const T* p = base + P.c0;
        constexpr int U = 4;
        int64_t s = P.s0 + P.r;
        for (; s + (U - 1) * A.lanes < P.s1; s += (int64_t)U * A.lanes) {
            Vec<T, V> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const Vec<T, V>*>(p + (s + (int64_t)u * A.lanes) * A.xs);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = to_f32(v[u].e[i]) - pv[i];
                    s1[i] += d;
                    s2[i] = fmaf(d, d, s2[i]);
                }
        }
        for (; s < P.s1; s += A.lanes) {
            const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(p + s * A.xs);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = to_f32(v.e[i]) - pv[i];
                s1[i] += d;
                s2[i] = fmaf(d, d, s2[i]);
            }
        }
    }
    gn_reduce_block<V, false>(A, P, s1, s2, sh);
    release_successor();
}

// The two numbers of each group of sample n, added over the chunks: a warp per group, fp64.
// stat[g] = (mean, rstd) forward, (<dh>, <dh h>) backward.
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

template <bool BACKWARD>
__device__ __forceinline__ void gn_group_stats(const GnArgs& A, int n, int g0, int g1, float2* stat) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const double count = (double)A.S * A.per;
    for (int g = g0 + warp; g < g1; g += kGnThreads / 32) {
        double a = 0.0, b = 0.0;
        // entry i of the group: chunk i / bpg, piece i % bpg
        for (int i = lane; i < A.chunks * A.bpg; i += 32) {
            const int c = A.bpg == 1 ? i : i / A.bpg;
            const float2 t = A.part[((int64_t)n * A.chunks + c) * (A.G * A.bpg) + g * A.bpg + (i - c * A.bpg)];
            a += t.x;
            b += t.y;
        }
        a = warp_sum(a) / count;
        b = warp_sum(b) / count;
        if (lane == 0) {
            if (BACKWARD) {
                stat[g - g0] = make_float2((float)a, (float)b);
            } else {
                const double pivot = (double)A.pivot[(int64_t)n * A.G + g];
                const double var = b - a * a;
                const float m = (float)(pivot + a), r = (float)(1.0 / sqrt((var > 0.0 || var != var ? var : 0.0) + (double)A.eps));
                stat[g - g0] = make_float2(m, r);
                if (A.mean && blockIdx.x == 0) A.mean[(int64_t)n * A.G + g] = m;
                if (A.rstd && blockIdx.x == 0) A.rstd[(int64_t)n * A.G + g] = r;
            }
        }
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) gn_apply_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ float2 sh[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    float ga[V], be[V];
    if (P.on) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[i] = gn_param(A.gamma, A.params_f32, A.params_bf16, P.c0 + i, 1.0f);
            be[i] = gn_param(A.beta, A.params_f32, A.params_bf16, P.c0 + i, 0.0f);
        }
    }
    wait_predecessor();
    gn_group_stats<false>(A, n, P.g0, P.g1, sh);
    __syncthreads();
    if (!P.on) return;
    float mu[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 t = sh[(P.c0 + i) / A.per - P.g0];
        mu[i] = t.x;
        ga[i] *= t.y;
    }
    const T* p = static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0;
    T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + P.c0;
    constexpr int U = 4;
    auto one = [&](const Vec<T, V>& v, int64_t s) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = act_value<ACT>(fmaf(to_f32(v.e[i]) - mu[i], ga[i], be[i]));
        *reinterpret_cast<Vec<T, V>*>(q + s * A.ys) = narrow<T, V>(o);
    };
    // backwards: from the place pass 1 read last
    int64_t k = P.s1 - P.s0 - P.r;                      // places left for this thread: s0 + r, + lanes, ...
    int64_t left = k > 0 ? (k + A.lanes - 1) / A.lanes : 0;
    int64_t s = P.s0 + P.r + (left - 1) * A.lanes;
    for (; left >= U; left -= U, s -= (int64_t)U * A.lanes) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const Vec<T, V>*>(p + (s - (int64_t)u * A.lanes) * A.xs);
#pragma unroll
        for (int u = 0; u < U; ++u) one(v[u], s - (int64_t)u * A.lanes);
    }
    for (; left > 0; --left, s -= A.lanes) one(*reinterpret_cast<const Vec<T, V>*>(p + s * A.xs), s);
}

// ------------------------------------------------------------------ backward

// dz and h of V channels at one place
template <typename T, int V, int ACT>
__device__ __forceinline__ void gn_dz(const Vec<T, V>& xv, const Vec<T, V>& dv, const float (&mu)[V], const float (&rs)[V],
                                      const float (&ga)[V], const float (&be)[V], float (&dz)[V], float (&h)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        h[i] = (to_f32(xv.e[i]) - mu[i]) * rs[i];
        dz[i] = to_f32(dv.e[i]);
        if (ACT != DVDQ_ACT_NONE) dz[i] *= act_slope<ACT>(fmaf(ga[i], h[i], be[i]));
    }
}

template <typename T, int V, int ACT>
__device__ __forceinline__ void gn_constants(const GnArgs& A, int n, int c0, float (&mu)[V], float (&rs)[V], float (&ga)[V], float (&be)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int64_t g = (int64_t)n * A.G + (c0 + i) / A.per;
        mu[i] = A.mean[g];
        rs[i] = A.rstd[g];
        ga[i] = gn_param(A.gamma, A.params_f32, A.params_bf16, c0 + i, 1.0f);
        be[i] = gn_param(A.beta, A.params_f32, A.params_bf16, c0 + i, 0.0f);
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) gn_grad_stats_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ float2 sh[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    float s1[V], s2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.f;
    if (P.on) {
        float mu[V], rs[V], ga[V], be[V];
        gn_constants<T, V, ACT>(A, n, P.c0, mu, rs, ga, be);
        const T* p = static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0;
        const T* d = static_cast<const T*>(A.dy) + (int64_t)n * A.dn + P.c0;
        auto one = [&](const Vec<T, V>& xv, const Vec<T, V>& dv) {
            float dz[V], h[V];
            gn_dz<T, V, ACT>(xv, dv, mu, rs, ga, be, dz, h);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s1[i] += dz[i];
                s2[i] = fmaf(dz[i], h[i], s2[i]);
            }
        };
        constexpr int U = 2;
        int64_t s = P.s0 + P.r;
        for (; s + (U - 1) * A.lanes < P.s1; s += (int64_t)U * A.lanes) {
            Vec<T, V> xv[U], dv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                xv[u] = *reinterpret_cast<const Vec<T, V>*>(p + (s + (int64_t)u * A.lanes) * A.xs);
                dv[u] = *reinterpret_cast<const Vec<T, V>*>(d + (s + (int64_t)u * A.lanes) * A.ds);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) one(xv[u], dv[u]);
        }
        for (; s < P.s1; s += A.lanes)
            one(*reinterpret_cast<const Vec<T, V>*>(p + s * A.xs), *reinterpret_cast<const Vec<T, V>*>(d + s * A.ds));
    }
    gn_reduce_block<V, true>(A, P, s1, s2, sh);
    release_successor();
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) gn_grad_apply_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ float2 sh[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    float mu[V], rs[V], ga[V], be[V];
    if (P.on) gn_constants<T, V, ACT>(A, n, P.c0, mu, rs, ga, be);
    wait_predecessor();
    gn_group_stats<true>(A, n, P.g0, P.g1, sh);
    __syncthreads();
    if (P.on && A.y) {
        float m1[V], m2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 t = sh[(P.c0 + i) / A.per - P.g0];
            m1[i] = t.x;
            m2[i] = t.y;
        }
        const T* p = static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0;
        const T* d = static_cast<const T*>(A.dy) + (int64_t)n * A.dn + P.c0;
        T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + P.c0;
        auto one = [&](const Vec<T, V>& xv, const Vec<T, V>& dv, int64_t s) {
            float dz[V], h[V], o[V];
            gn_dz<T, V, ACT>(xv, dv, mu, rs, ga, be, dz, h);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = rs[i] * (fmaf(dz[i], ga[i], -m1[i]) - h[i] * m2[i]);
            *reinterpret_cast<Vec<T, V>*>(q + s * A.ys) = narrow<T, V>(o);
        };
        constexpr int U = 2;
        int64_t k = P.s1 - P.s0 - P.r;
        int64_t left = k > 0 ? (k + A.lanes - 1) / A.lanes : 0;
        int64_t s = P.s0 + P.r + (left - 1) * A.lanes;
        for (; left >= U; left -= U, s -= (int64_t)U * A.lanes) {
            Vec<T, V> xv[U], dv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                xv[u] = *reinterpret_cast<const Vec<T, V>*>(p + (s - (int64_t)u * A.lanes) * A.xs);
                dv[u] = *reinterpret_cast<const Vec<T, V>*>(d + (s - (int64_t)u * A.lanes) * A.ds);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) one(xv[u], dv[u], s - (int64_t)u * A.lanes);
        }
        for (; left > 0; --left, s -= A.lanes)
            one(*reinterpret_cast<const Vec<T, V>*>(p + s * A.xs), *reinterpret_cast<const Vec<T, V>*>(d + s * A.ds), s);
    }
    // the parameters' gradients: the first CTAs take 32 channels each, 8 rows of chunks side by side, fp64
    if (!A.dgamma && !A.dbeta) return;
    const int ctas = gridDim.x * gridDim.y * gridDim.z;
    const int cta = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ double2 red[kGnThreads / 32][32];
    for (int cb = cta; cb < (A.C + 31) / 32; cb += ctas) {
        const int c = cb * 32 + lane;
        double a = 0.0, b = 0.0;
        if (c < A.C)
            for (int64_t i = warp; i < (int64_t)A.N * A.chunks; i += kGnThreads / 32) {
                const float2 t = A.part_c[i * A.C + c];
                a += t.x;
                b += t.y;
            }
        __syncthreads();
        red[warp][lane] = make_double2(a, b);
        __syncthreads();
        if (warp == 0 && c < A.C) {
            for (int w = 1; w < kGnThreads / 32; ++w) {
                a += red[w][lane].x;
                b += red[w][lane].y;
            }
            if (A.dbeta) A.dbeta[c] = (float)a;
            if (A.dgamma) A.dgamma[c] = (float)b;
        }
    }
}

// An empty sample: nothing to normalise; its statistics are (0, 1 / sqrt(eps)), its gradients zero.
__global__ void gn_empty_kernel(float* mean, float* rstd, int64_t ng, float* dgamma, float* dbeta, int C, float eps) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < ng) {
        if (mean) mean[i] = 0.f;
        if (rstd) rstd[i] = rsqrtf(eps);
    }
    if (i < C) {
        if (dgamma) dgamma[i] = 0.f;
        if (dbeta) dbeta[i] = 0.f;
    }
}

// ------------------------------------------------------------------ host side

// How the places and channels are cut, from the shape alone (so that the workspace can be asked for
// without the tensors): V is decided at the call, and both widths use the same chunks.
struct GnPlan {
    int chunks;
    int64_t rows;
};
inline GnPlan gn_plan(int64_t N, int64_t S) {
    // One wave of CTAs, four per SM, over all samples; a chunk has at least 32 places, so that a small
    // tensor's second pass has few partial sums to add up.
    int64_t chunks = (148 * 4 + N - 1) / N;
    const int64_t most = ceil_div(S, 32);
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    GnPlan p;
    p.rows = ceil_div(S, chunks);
    p.chunks = (int)ceil_div(S, p.rows);
    return p;
}
// Pieces that a group wider than a CTA's vectors is cut into, at most (single-element accesses).
inline int64_t gn_pieces(int64_t per) { return ceil_div(per, kGnMaxVecs); }
struct GnRoom {
    int64_t pivot_off, part_c_off, total;
};
inline GnRoom gn_room(int64_t N, int64_t S, int64_t C, int64_t G) {
    const GnPlan p = gn_plan(N, S);
    GnRoom r;
    r.pivot_off = align_up(N * p.chunks * G * gn_pieces(C / G) * 8, 256);
    r.part_c_off = r.pivot_off + align_up(N * G * 4, 256);
    r.total = r.part_c_off + N * p.chunks * C * 8;
    return r;
}

// Channel blocks for accesses of V channels: some whole groups, or a piece of one wide group.
inline bool gn_cut(GnArgs& A, int V) {
    if (A.C % V != 0) return false;
    const int64_t cv = A.C / V;
    A.bpg = 1;
    int64_t unit = A.per;                      // channels of the fewest whole groups that are whole vectors
    while (unit % V != 0) unit += A.per;
    if (cv <= kGnMaxVecs) {
        A.vecs = (int)cv;
        A.blocks = 1;
    } else if (unit / V <= kGnMaxVecs) {
        A.vecs = (int)(kGnMaxVecs / (unit / V) * (unit / V));
        A.blocks = (int)ceil_div(cv, A.vecs);
    } else {
        if (A.per % V != 0) return false;
        const int64_t gv = A.per / V;
        A.bpg = (int)ceil_div(gv, kGnMaxVecs);
        A.vecs = (int)ceil_div(gv, A.bpg);
        A.blocks = A.G * A.bpg;
    }
    A.lanes = kGnThreads / A.vecs;
    return true;
}

template <typename T, int V>
static cudaError_t launch_gn_v(GnArgs A, bool backward, int act, cudaStream_t st) {
    const dim3 grid((unsigned)A.chunks, (unsigned)A.N, (unsigned)A.blocks);
    const size_t smem = (size_t)kGnThreads * V * sizeof(float2);
    cudaError_t e;
    if (!backward) {
        gn_stats_kernel<T, V><<<grid, kGnThreads, smem, st>>>(A);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        auto k = act == DVDQ_ACT_GELU_TANH ? gn_apply_kernel<T, V, DVDQ_ACT_GELU_TANH>
                 : act == DVDQ_ACT_SILU    ? gn_apply_kernel<T, V, DVDQ_ACT_SILU>
                                           : gn_apply_kernel<T, V, DVDQ_ACT_NONE>;
        return launch_after(k, grid, dim3(kGnThreads), smem, st, A);
    }
    if (act == DVDQ_ACT_GELU_TANH) gn_grad_stats_kernel<T, V, DVDQ_ACT_GELU_TANH><<<grid, kGnThreads, smem, st>>>(A);
    else if (act == DVDQ_ACT_SILU) gn_grad_stats_kernel<T, V, DVDQ_ACT_SILU><<<grid, kGnThreads, smem, st>>>(A);
    else gn_grad_stats_kernel<T, V, DVDQ_ACT_NONE><<<grid, kGnThreads, smem, st>>>(A);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    auto k = act == DVDQ_ACT_GELU_TANH ? gn_grad_apply_kernel<T, V, DVDQ_ACT_GELU_TANH>
             : act == DVDQ_ACT_SILU    ? gn_grad_apply_kernel<T, V, DVDQ_ACT_SILU>
                                       : gn_grad_apply_kernel<T, V, DVDQ_ACT_NONE>;
    return launch_after(k, grid, dim3(kGnThreads), smem, st, A);
}

// Whole 16-byte accesses where channels, pitches and pointers allow it, single elements otherwise.
template <typename T>
static cudaError_t launch_gn_t(GnArgs A, bool backward, int act, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    bool wide = A.C % V == 0 && aligned_to(A.x, 16) && aligned_to(A.y, 16) && aligned_to(A.dy, 16);
    for (int64_t p : {A.xn, A.xs, A.yn, A.ys, A.dn, A.ds}) wide = wide && p % V == 0;
    if (wide && gn_cut(A, V)) return launch_gn_v<T, V>(A, backward, act, st);
    return gn_cut(A, 1) ? launch_gn_v<T, 1>(A, backward, act, st) : cudaErrorInvalidValue;
}

}  // namespace dvdq
