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
// Large tensors, in one of two ways.  One cooperative launch of one CTA per SM: pass 1 sums a chunk of places of one sample over
// all channels (a thread keeps its 16 bytes of channels, so its loads are whole sectors) and writes two
// numbers per group; all CTAs meet once; every CTA adds up its sample's numbers in a fixed order (no
// atomics on data: the same bits every time); pass 2 walks the chunk backwards, first the pieces that pass 1
// left in shared memory (about 20 MB over the chip), then what the L2 cache still holds.  A thread sums in fp32, about a centre that
// follows its own mean (GnMoments), everything beyond in fp64: neither a mean far from zero nor a value far from the mean costs
// digits.
// Where that does not fit (places not made of 4-byte pieces, more than 512 or 1024 pieces in one, sample counts that leave SMs idle) or
// is the slower (kGnOneFrom): three launches, pass 1, join, pass 2, each started while its predecessor drains.
// Small tensors, one launch: where a slice of whole groups of one sample fits a CTA's shared memory,
// the CTA reads it once, and does both passes on it.
//
// Measured: 499200 places of 128 channels, bf16 with SiLU, 77 us (3.3 TB/s of x once and y once, 39 us at the copy rate); gradients
// of 2 x 18720 places of 512 channels 43 us (115 MB, 2.7 TB/s); 3 x 77 places of 180 fp32 channels 6.3 us in a graph.
#pragma once

#include <type_traits>

#include "block_common.cuh"

namespace dvdq {

constexpr int kGnThreads = kStreamThreads;
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
    float2* part;            // [N, chunks, G]: sums of the backward pass
    double2* part64;         // the same room: moments of the forward pass
    float* pivot;            // [N, G]: what pass 1 subtracted (y may be x: pass 2 cannot read it there)
    float2* part_c;          // backward: [N, chunks, C]
    float2* stat;            // [N, G]: (mean, rstd) forward, (<dh>, <dh h>) backward
    uint32_t* arrived;       // one-launch kernels: CTAs that have written their numbers
    int64_t xn, xs, dn, ds, yn, ys;  // pitches of samples and places, elements
    int64_t S;
    int N, C, G, per;        // per = C / G
    int chunks;              // chunks of places per sample
    int64_t rows;            // places per chunk
    int vecs, lanes;         // channel vectors of a CTA (its channel block), rows it walks side by side
    int blocks;              // channel blocks: each some whole groups, or (bpg > 1) a piece of one group
    int bpg;                 // blocks per group
    int params_f32, params_bf16;
    double inv;              // 1 / (S per)
    float eps;
};

__device__ __forceinline__ float gn_param(const void* p, int f32, int bf16, int c, float none) {
    if (!p) return none;
    if (f32) return static_cast<const float*>(p)[c];
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[c]) : __half2float(static_cast<const __half*>(p)[c]);
}

// Sums of d and d^2 of a thread's pieces, d = x - centre, where the centre is the group's mean already (small tensors).  Squares
// below half a unit in the last place of a long sum are lost, and small squares are the many: 250 normal values summed one after
// another are 2e-6 low.  So every 16 pieces the short sum moves on.
template <int V>
struct GnCentred {
    Pairs<V> s1, s2, outer;
    int n = 0;
    __device__ __forceinline__ GnCentred() {
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = s2.p[i] = outer.p[i] = 0ull;
    }
    __device__ __forceinline__ void add(const Pairs<V>& x, const Pairs<V>& centre) {
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            const uint64_t d = f2_sub(x.p[i], centre.p[i]);
            s1.p[i] = f2_add(s1.p[i], d);
            s2.p[i] = f2_fma(d, d, s2.p[i]);
        }
        if ((++n & 15) == 0) flush();
    }
    __device__ __forceinline__ void flush() {
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            outer.p[i] = f2_add(outer.p[i], s2.p[i]);
            s2.p[i] = 0ull;
        }
    }
};

// The same where the mean is not known yet: d = x - k with a centre k of the thread's own, channel by channel.  k is the first
// piece, and whenever the number of pieces has doubled it moves to their mean: by e, which takes n e from the sum and
// e (s1 + s1') from the squares.  So the squares about k are never more than about twice those about the mean, and no single value,
// the group's first or any other, decides how many digits are left.  (About one fixed value, -1000 among normal values: rstd off by 2e-3.)
template <int V>
struct GnMoments {
    Pairs<V> k, s1, s2, q;
    int n = 0, next = 0;  // pieces so far; how many there are when the short sum moves on: 0, 2, 4, 8, 16, then every 16
    __device__ __forceinline__ GnMoments() {
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) k.p[i] = s1.p[i] = s2.p[i] = q.p[i] = 0ull;
    }
    __device__ __forceinline__ void add(const Pairs<V>& x) {
        if (n == next) {
            if (n == 0) k = x;
            else flush();
            if ((n & (n - 1)) == 0 && n > 0) move();
            next = n == 0 ? 2 : n < 16 ? 2 * n : n + 16;
        }
        ++n;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            const uint64_t d = f2_sub(x.p[i], k.p[i]);
            s1.p[i] = f2_add(s1.p[i], d);
            s2.p[i] = f2_fma(d, d, s2.p[i]);
        }
    }
    __device__ __forceinline__ void flush() {
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            q.p[i] = f2_add(q.p[i], s2.p[i]);
            s2.p[i] = 0ull;
        }
    }
    __device__ __forceinline__ void move() {  // n is a power of two
        const float count = (float)n;
        const uint64_t minus_n = f2_splat(-count), one_nth = f2_splat(__int_as_float(0x7F000000 - __float_as_int(count)));
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            const uint64_t to = f2_fma(s1.p[i], one_nth, k.p[i]), e = f2_sub(to, k.p[i]), s = f2_fma(minus_n, e, s1.p[i]);
            q.p[i] = f2_sub(q.p[i], f2_mul(e, f2_add(s1.p[i], s)));
            s1.p[i] = s;
            k.p[i] = to;
        }
    }
    // use(u, sums of x - pivot and its square over unit u) after the last flush(); a unit is 1 << log channels of one group.  Within it
    // the sums are brought to the mean of the channels' centres in fp32 (to one of them, a centre that lies far out would have its
    // square counted for each of the others), then to the group's pivot in fp64, in which they stay.
    template <typename Use>
    __device__ __forceinline__ void by_unit(int log, const float (&pivot)[V], Use use) const {
        const int last = (1 << log) - 1;
        const float count = (float)n, part = __int_as_float((127 - log) << 23);  // 1 / (channels of a unit)
        float c[V];
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = k.get(i) * part;
#pragma unroll
        for (int step = 1; step < V; step <<= 1) {
            if (step > last) continue;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if ((i & step) == 0) c[i] = c[i + step] = c[i] + c[i + step];
        }
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if ((i & last) == 0) a = b = 0.f;
            const float e = k.get(i) - c[i], s = s1.get(i), moved = fmaf(count, e, s);
            a += moved;
            b += fmaf(e, s + moved, q.get(i));
            if ((i & last) == last) {
                const double shift = (double)c[i] - (double)pivot[i], all = (double)(n << log), to = a + all * shift;
                use(i >> log, make_double2(to, b + shift * (a + to)));
            }
        }
    }
};
// log2 of the channels of a unit: as many as divide both a thread's vector and the group
__device__ __forceinline__ int gn_unit(int per, int V) { return __ffs(per | V) - 1; }

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
    // this thread's places: s0 + r, s0 + r + lanes, ...
    __device__ __forceinline__ int count(int lanes) const {
        const int64_t k = s1 - s0 - r;
        return k > 0 ? (int)((k + lanes - 1) / lanes) : 0;
    }
};

// Adds the threads' sums over the lanes, pairwise (a long sum of equal terms loses digits, and a serial walk over a thousand
// lanes takes 16 us).  Thread r * vecs + v of `on` threads has put its `sums` sums of vector v at sh[i * threads + thread]; the total
// of sum i ends in sh[i * threads + v].
template <typename Pair>
__device__ __forceinline__ void gn_sum_lanes(bool on, int r, int lanes, int vecs, int sums, Pair* sh) {
    const int threads = lanes * vecs, t = threadIdx.x;
    __syncthreads();
    for (int left = lanes; left > 1;) {
        const int half = (left + 1) >> 1;
        if (on && r < left - half) {
#pragma unroll 4
            for (int i = 0; i < sums; ++i) {
                Pair a = sh[i * threads + t];
                const Pair b = sh[i * threads + t + half * vecs];
                a.x += b.x;
                a.y += b.y;
                sh[i * threads + t] = a;
            }
        }
        left = half;
        __syncthreads();
    }
}

template <int V>
__device__ __forceinline__ void gn_put_sums(int threads, const Pairs<V>& s1, const Pairs<V>& s2, float2* sh) {
#pragma unroll
    for (int i = 0; i < V; ++i) sh[i * threads + threadIdx.x] = make_float2(s1.get(i), s2.get(i));
}

// ... then over the `span` channels (or units) of each group: put(g, the sum of channel(g span) .. channel(g span + span - 1)).
template <int THREADS, typename Pair, typename Channel, typename Put>
__device__ __forceinline__ void gn_sum_groups(int groups, int span, Channel channel, Put put) {
    if (span <= 8) {
        for (int g = threadIdx.x; g < groups; g += THREADS) {
            Pair t = channel(g * span);
            for (int i = 1; i < span; ++i) {
                const Pair u = channel(g * span + i);
                t.x += u.x;
                t.y += u.y;
            }
            put(g, t);
        }
    } else {  // wide groups: a warp each
        for (int g = threadIdx.x >> 5; g < groups; g += THREADS / 32) {
            Pair t = {};
            for (int i = threadIdx.x & 31; i < span; i += 32) {
                const Pair u = channel(g * span + i);
                t.x += u.x;
                t.y += u.y;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, o);
                t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, o);
            }
            if ((threadIdx.x & 31) == 0) put(g, t);
        }
    }
}

// A block's moments about the groups' pivots, a pair per group, in fp64 from the threads on.
template <int V>
__device__ __forceinline__ void gn_block_moments(const GnArgs& A, const GnPlace<V>& P, const GnMoments<V>& m, const float (&pivot)[V], double2* sh) {
    const int threads = A.lanes * A.vecs, log = gn_unit(A.per, V), units = V >> log, wide = 31 - __clz(units);
    const bool on = P.r < A.lanes;  // vectors past the block's end carry zeros
    if (on) m.by_unit(log, pivot, [&](int u, const double2& t) { sh[u * threads + threadIdx.x] = t; });
    gn_sum_lanes(on, P.r, A.lanes, A.vecs, units, sh);
    double2* out = A.part64 + ((int64_t)blockIdx.y * A.chunks + blockIdx.x) * (A.G * A.bpg) + (A.bpg == 1 ? P.g0 : (int)blockIdx.z);
    gn_sum_groups<kGnThreads, double2>(P.g1 - P.g0, (A.bpg == 1 ? A.per : P.here) >> log,
                                       [&](int u) { return sh[(u & (units - 1)) * threads + (u >> wide)]; },
                                       [&](int g, const double2& t) { out[g] = t; });
}
// A block's sums of the backward pass, a pair per channel and, gamma in them, per group.
template <int V>
__device__ __forceinline__ void gn_block_sums(const GnArgs& A, const GnPlace<V>& P, const Pairs<V>& s1, const Pairs<V>& s2, float2* sh) {
    const int threads = A.lanes * A.vecs;
    if (P.r < A.lanes) gn_put_sums<V>(threads, s1, s2, sh);  // vectors past the block's end carry zeros
    gn_sum_lanes(P.r < A.lanes, P.r, A.lanes, A.vecs, V, sh);
    const int64_t slot = (int64_t)blockIdx.y * A.chunks + blockIdx.x;
    auto place = [&](int c) { return (c % V) * threads + c / V; };  // of the block's channel c
    for (int c = threadIdx.x; c < P.here; c += kGnThreads) {
        float2 t = sh[place(c)];
        A.part_c[slot * A.C + P.cbase + c] = t;
        const float g = gn_param(A.gamma, A.params_f32, A.params_bf16, P.cbase + c, 1.0f);
        sh[place(c)] = make_float2(t.x * g, t.y * g);
    }
    __syncthreads();
    float2* out = A.part + slot * (A.G * A.bpg) + (A.bpg == 1 ? P.g0 : (int)blockIdx.z);
    gn_sum_groups<kGnThreads, float2>(P.g1 - P.g0, A.bpg == 1 ? A.per : P.here, [&](int c) { return sh[place(c)]; },
                                      [&](int g, const float2& t) { out[g] = t; });
}

constexpr int kGnDepth = 8, kGnGradDepth = 5;  // slots: 32 KB a CTA, 40 KB for two tensors; four CTAs per SM

template <typename T, int V>
__global__ void __launch_bounds__(kGnThreads, 4) gn_stats_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    wait_predecessor();
    release_successor();
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    GnMoments<V> sums;
    float pivot[V] = {};
    if (P.on) {
        const T* base = static_cast<const T*>(A.x) + (int64_t)n * A.xn;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = (P.c0 + i) / A.per;
            pivot[i] = to_f32(base[g * A.per]);
            if (blockIdx.x == 0 && P.r == 0 && P.c0 + i == g * A.per) A.pivot[(int64_t)n * A.G + g] = pivot[i];
        }
        walk<kGnDepth, 1, T, V>(raw, P.count(A.lanes), base + P.c0 + (P.s0 + P.r) * A.xs, A.lanes * A.xs, nullptr, 0,
                                 [&](const Vec<T, V>& v) { sums.add(widen2<T, V>(v)); });
        sums.flush();
    }
    __syncthreads();  // the ring's memory becomes the sums'
    gn_block_moments<V>(A, P, sums, pivot, reinterpret_cast<double2*>(raw));
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// mean and rstd from the group's mean and mean square about its pivot
__device__ __forceinline__ float2 gn_mean_rstd(double pivot, double m1, double m2, float eps) {
    const double var = m2 - m1 * m1;
    return make_float2((float)(pivot + m1), (float)rsqrt((var > 0.0 || var != var ? var : 0.0) + (double)eps));
}

// Adds up the chunks: the first `group_ctas` CTAs a warp per group, the rest (backward) 32 channels each.
template <bool BACKWARD>
using GnPart = typename std::conditional<BACKWARD, float2, double2>::type;
template <bool BACKWARD>
__device__ __forceinline__ const GnPart<BACKWARD>* gn_part(const GnArgs& A) {
    if constexpr (BACKWARD) return A.part;
    else return A.part64;
}
template <bool BACKWARD>
__global__ void __launch_bounds__(kGnThreads) gn_join_kernel(const __grid_constant__ GnArgs A, int group_ctas) {
    constexpr int kWarps = kGnThreads / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wait_predecessor();
    release_successor();
    if ((int)blockIdx.x < group_ctas) {
        const int64_t ng = (int64_t)blockIdx.x * kWarps + warp;
        if (ng >= (int64_t)A.N * A.G) return;
        const int n = (int)(ng / A.G), g = (int)(ng - (int64_t)n * A.G);
        const int entries = A.chunks * A.bpg, pitch = A.G * A.bpg;
        using Part = GnPart<BACKWARD>;
        const Part* base = gn_part<BACKWARD>(A) + (int64_t)n * A.chunks * pitch + (int64_t)g * A.bpg;
        double a = 0.0, b = 0.0;
        auto entry = [&](int i) { return A.bpg == 1 ? base[(int64_t)i * pitch] : base[(int64_t)(i / A.bpg) * pitch + i % A.bpg]; };
        int i = lane;
        for (; i + 7 * 32 < entries; i += 8 * 32) {
            Part t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = entry(i + 32 * u);
#pragma unroll
            for (int u = 0; u < 8; ++u) { a += t[u].x; b += t[u].y; }
        }
        for (; i < entries; i += 32) {
            const Part t = entry(i);
            a += t.x;
            b += t.y;
        }
        a = warp_sum(a) * A.inv;
        b = warp_sum(b) * A.inv;
        if (lane == 0) {
            if (BACKWARD) {
                A.stat[ng] = make_float2((float)a, (float)b);
            } else {
                const float2 t = gn_mean_rstd((double)A.pivot[ng], a, b, A.eps);
                A.stat[ng] = t;
                if (A.mean) A.mean[ng] = t.x;
                if (A.rstd) A.rstd[ng] = t.y;
            }
        }
    } else if constexpr (BACKWARD) {
        __shared__ double2 red[kWarps][32];
        const int c = ((int)blockIdx.x - group_ctas) * 32 + lane;
        double a = 0.0, b = 0.0;
        if (c < A.C) {
            const int64_t rows = (int64_t)A.N * A.chunks;
            int64_t i = warp;
            for (; i + 7 * kWarps < rows; i += 8 * kWarps) {
                float2 t[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) t[u] = A.part_c[(i + u * kWarps) * A.C + c];
#pragma unroll
                for (int u = 0; u < 8; ++u) { a += t[u].x; b += t[u].y; }
            }
            for (; i < rows; i += kWarps) {
                const float2 t = A.part_c[i * A.C + c];
                a += t.x;
                b += t.y;
            }
        }
        red[warp][lane] = make_double2(a, b);
        __syncthreads();
        if (warp == 0 && c < A.C) {
            for (int w = 1; w < kWarps; ++w) {
                a += red[w][lane].x;
                b += red[w][lane].y;
            }
            if (A.dbeta) A.dbeta[c] = (float)a;
            if (A.dgamma) A.dgamma[c] = (float)b;
        }
    }
}

// Calls get(i, group of channel c0 + i) for V channels; where they all lie in one group, once, and copy(i) for the rest.
template <int V, typename Get, typename Copy>
__device__ __forceinline__ void gn_by_channel(int per, int c0, Get get, Copy copy) {
    if (per % V == 0) {
        get(0, c0 / per);
#pragma unroll
        for (int i = 1; i < V; ++i) copy(i);
    } else {
        int g = c0 / per, left = (g + 1) * per - c0;  // channels of this group still to come
#pragma unroll
        for (int i = 0; i < V; ++i) {
            get(i, g);
            if (--left == 0) {
                ++g;
                left = per;
            }
        }
    }
}
template <int V>
__device__ __forceinline__ void gn_params(const GnArgs& A, int c0, float (&ga)[V], float (&be)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ga[i] = gn_param(A.gamma, A.params_f32, A.params_bf16, c0 + i, 1.0f);
        be[i] = gn_param(A.beta, A.params_f32, A.params_bf16, c0 + i, 0.0f);
    }
}

// z = (x - mean) a + beta with a = gamma rstd.  The mean is taken off first: inside the constant (x a + (beta - mean a)) its
// rounding, 2^-24 |mean| a, is all that is left of a group whose values are equal, or nearly all.
template <int V>
struct GnScale {
    Pairs<V> mean, a, b;
    __device__ __forceinline__ GnScale(const float (&mu)[V], const float (&sc)[V], const float (&sh)[V]) {
        mean.set(mu);
        a.set(sc);
        b.set(sh);
    }
    __device__ __forceinline__ uint64_t operator()(uint64_t x, int i) const {
        return f2_fma(f2_sub(x, mean.p[i]), a.p[i], b.p[i]);
    }
};

// ... from the groups' (mean, rstd)
template <int V>
__device__ __forceinline__ GnScale<V> gn_scale(const GnArgs& A, int c0, const float2* stat, const float (&ga)[V], const float (&be)[V]) {
    float mu[V], sc[V];
    gn_by_channel<V>(A.per, c0, [&](int i, int g) { const float2 t = stat[g]; mu[i] = t.x; sc[i] = t.y; },
                     [&](int i) { mu[i] = mu[0]; sc[i] = sc[0]; });
#pragma unroll
    for (int i = 0; i < V; ++i) sc[i] *= ga[i];
    return GnScale<V>(mu, sc, be);
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 4) gn_apply_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    wait_predecessor();
    release_successor();
    if (!P.on) return;
    float ga[V], be[V];
    gn_params<V>(A, P.c0, ga, be);
    const GnScale<V> scale = gn_scale<V>(A, P.c0, A.stat + (int64_t)n * A.G, ga, be);
    // backwards: from the place pass 1 read last
    const int count = P.count(A.lanes);
    const int64_t last = P.s0 + P.r + (int64_t)(count - 1) * A.lanes;
    T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + P.c0 + last * A.ys;
    const int64_t back = -(int64_t)A.lanes * A.ys;
    walk<kGnDepth, 1, T, V>(raw, count, static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0 + last * A.xs, -(int64_t)A.lanes * A.xs, nullptr, 0,
                               [&](const Vec<T, V>& v) {
        const Pairs<V> x = widen2<T, V>(v);
        Pairs<V> o;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) o.p[i] = act_value2<ACT, true>(scale(x.p[i], i));
        store_streaming<T, V>(q, narrow2<T, V>(o));
        q += back;
    });
}

// ------------------------------------------------------------------ backward

// What the backward passes hold per channel: h = (x - mean) rstd, z = gamma h + beta.
template <int V>
struct GnGrad {
    GnScale<V> h;
    Pairs<V> gamma, beta;
    template <int ACT>
    __device__ __forceinline__ void dz(uint64_t x, uint64_t dy, int i, uint64_t& out_dz, uint64_t& out_h) const {
        out_h = h(x, i);
        out_dz = ACT == DVDQ_ACT_NONE ? dy : f2_mul(dy, act_slope2<ACT, true>(f2_fma(gamma.p[i], out_h, beta.p[i])));
    }
};
template <int V>
__device__ __forceinline__ GnGrad<V> gn_constants(const GnArgs& A, int n, int c0, float (&rs)[V], float (&ga)[V]) {
    float mu[V], be[V], none[V];
    gn_by_channel<V>(A.per, c0, [&](int i, int g) { mu[i] = A.mean[(int64_t)n * A.G + g]; rs[i] = A.rstd[(int64_t)n * A.G + g]; },
                     [&](int i) { mu[i] = mu[0]; rs[i] = rs[0]; });
    gn_params<V>(A, c0, ga, be);
#pragma unroll
    for (int i = 0; i < V; ++i) none[i] = 0.f;
    GnGrad<V> r{GnScale<V>(mu, rs, none), {}, {}};
    r.gamma.set(ga);
    r.beta.set(be);
    return r;
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 2) gn_grad_stats_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    wait_predecessor();
    release_successor();
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    Pairs<V> s1, s2;
#pragma unroll
    for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = s2.p[i] = 0ull;
    if (P.on) {
        float rs[V], ga[V];
        const GnGrad<V> K = gn_constants<V>(A, n, P.c0, rs, ga);
        const int64_t s0 = P.s0 + P.r;
        walk<kGnGradDepth, 2, T, V>(raw, P.count(A.lanes), static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0 + s0 * A.xs, A.lanes * A.xs,
                                       static_cast<const T*>(A.dy) + (int64_t)n * A.dn + P.c0 + s0 * A.ds, A.lanes * A.ds,
                                       [&](const Vec<T, V>& xv, const Vec<T, V>& dv) {
            const Pairs<V> x = widen2<T, V>(xv), dy = widen2<T, V>(dv);
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) {
                uint64_t dz, h;
                K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
                s1.p[i] = f2_add(s1.p[i], dz);
                s2.p[i] = f2_fma(dz, h, s2.p[i]);
            }
        });
    }
    __syncthreads();  // the ring's memory becomes the sums'
    gn_block_sums<V>(A, P, s1, s2, reinterpret_cast<float2*>(raw));
}

// dx = rstd (gamma dz - m1 - h m2) = dz (rstd gamma) + (h (-rstd m2) + (-rstd m1))
template <int V>
struct GnDx {
    Pairs<V> c1, c2, c3;
    __device__ __forceinline__ GnDx(const float (&rs)[V], const float (&ga)[V], const float (&m1)[V], const float (&m2)[V]) {
        float a[V], b[V], c[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = rs[i] * ga[i];
            b[i] = -rs[i] * m2[i];
            c[i] = -rs[i] * m1[i];
        }
        c1.set(a);
        c2.set(b);
        c3.set(c);
    }
    __device__ __forceinline__ uint64_t operator()(uint64_t dz, uint64_t h, int i) const { return f2_fma(dz, c1.p[i], f2_fma(h, c2.p[i], c3.p[i])); }
};

// ... from the groups' (<dh>, <dh h>)
template <int V>
__device__ __forceinline__ GnDx<V> gn_dx(const GnArgs& A, int c0, const float2* stat, const float (&rs)[V], const float (&ga)[V]) {
    float m1[V], m2[V];
    gn_by_channel<V>(A.per, c0, [&](int i, int g) { const float2 t = stat[g]; m1[i] = t.x; m2[i] = t.y; },
                     [&](int i) { m1[i] = m1[0]; m2[i] = m2[0]; });
    return GnDx<V>(rs, ga, m1, m2);
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads, 2) gn_grad_apply_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    const GnPlace<V> P(A);
    const int n = blockIdx.y;
    wait_predecessor();
    release_successor();
    if (!P.on) return;
    float rs[V], ga[V];
    const GnGrad<V> K = gn_constants<V>(A, n, P.c0, rs, ga);
    const GnDx<V> dx = gn_dx<V>(A, P.c0, A.stat + (int64_t)n * A.G, rs, ga);
    const int count = P.count(A.lanes);
    const int64_t last = P.s0 + P.r + (int64_t)(count - 1) * A.lanes;
    T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + P.c0 + last * A.ys;
    const int64_t back = -(int64_t)A.lanes * A.ys;
    walk<kGnGradDepth, 2, T, V>(raw, count, static_cast<const T*>(A.x) + (int64_t)n * A.xn + P.c0 + last * A.xs, -(int64_t)A.lanes * A.xs,
                                   static_cast<const T*>(A.dy) + (int64_t)n * A.dn + P.c0 + last * A.ds, -(int64_t)A.lanes * A.ds,
                                   [&](const Vec<T, V>& xv, const Vec<T, V>& dv) {
        const Pairs<V> x = widen2<T, V>(xv), dy = widen2<T, V>(dv);
        Pairs<V> o;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            uint64_t dz, h;
            K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
            o.p[i] = dx(dz, h, i);
        }
        store_streaming<T, V>(q, narrow2<T, V>(o));
        q += back;
    });
}

// ------------------------------------------------------------------ large tensors: one cooperative launch

// Threads, and slots of the ring: it and the sums fill the shared memory of an SM.  Channel counts that 16 bytes do not divide
// go in pieces of 8 or 4 bytes, more of them.
constexpr int kGnFusedThreads = 1024, kGnFusedGradThreads = 512, kGnFusedGroups = 1024;
template <typename T, int V> struct GnDepth {
    static constexpr int fused = 9 * 16 / (int)sizeof(Vec<T, V>), fused_grad = 10 * 16 / (int)sizeof(Vec<T, V>);
};

// The CTA's place: sample n, chunk j of `chunks`.
template <int V, int THREADS>
struct GnTeam {
    int n, j, v, c0, r, lanes, count;
    int64_t s0;
    bool on;
    __device__ __forceinline__ GnTeam(const GnArgs& A) {
        n = blockIdx.x / A.chunks;
        j = blockIdx.x - n * A.chunks;
        lanes = THREADS / A.vecs;
        v = threadIdx.x % A.vecs;
        r = threadIdx.x / A.vecs;
        c0 = v * V;
        on = r < lanes;
        s0 = (int64_t)j * A.rows + r;
        const int64_t s1 = min((int64_t)(j + 1) * A.rows, A.S);
        count = on && s0 < s1 ? (int)((s1 - s0 + lanes - 1) / lanes) : 0;
    }
};

// The CTA's moments about the groups' pivots, a pair per group, in fp64 from the threads on; four units of each vector at a
// time, since the ring keeps the rest of the shared memory (eight only where a group has an odd number of 16-bit channels).
template <int V> struct GnRound { static constexpr int units = V < 4 ? V : 4; };
template <int V, int THREADS>
__device__ __forceinline__ void gn_team_moments(const GnArgs& A, const GnTeam<V, THREADS>& P, const GnMoments<V>& m, const float (&pivot)[V], double2* sh) {
    const int threads = P.lanes * A.vecs, log = gn_unit(A.per, V), units = V >> log, wide = 31 - __clz(units), w = min(units, GnRound<V>::units);
    double2* out = A.part64 + (int64_t)P.n * A.G * A.chunks + P.j;
#pragma unroll 1
    for (int first = 0; first < units; first += w) {
        if (first > 0) __syncthreads();
        auto here = [&](int u) { return (uint32_t)(u - first) < (uint32_t)w; };
        if (P.on)
            m.by_unit(log, pivot, [&](int u, const double2& t) {
                if (here(u)) sh[(u - first) * threads + threadIdx.x] = t;
            });
        gn_sum_lanes(P.on, P.r, P.lanes, A.vecs, w, sh);
        gn_sum_groups<THREADS, double2>(A.G, A.per >> log,
            [&](int u) {
                const int i = u & (units - 1);
                return here(i) ? sh[(i - first) * threads + (u >> wide)] : make_double2(0.0, 0.0);
            },
            [&](int g, double2 t) {
                double2* to = out + (int64_t)g * A.chunks;
                if (first > 0) {  // this thread's own number of the round before
                    t.x += to->x;
                    t.y += to->y;
                }
                *to = t;
            });
    }
}
// The CTA's sums of the backward pass, a pair per channel and, gamma in them, per group.
template <int V, int THREADS>
__device__ __forceinline__ void gn_team_sums(const GnArgs& A, const GnTeam<V, THREADS>& P, const Pairs<V>& s1, const Pairs<V>& s2, float2* sh) {
    const int threads = P.lanes * A.vecs;
    if (P.on) gn_put_sums<V>(threads, s1, s2, sh);
    gn_sum_lanes(P.on, P.r, P.lanes, A.vecs, V, sh);
    auto channel = [&](int c) -> float2& { return sh[(c % V) * threads + c / V]; };
    for (int c = threadIdx.x; c < A.C; c += THREADS) {
        const float2 t = channel(c);
        A.part_c[(int64_t)c * gridDim.x + blockIdx.x] = t;
        const float g = gn_param(A.gamma, A.params_f32, A.params_bf16, c, 1.0f);
        channel(c) = make_float2(t.x * g, t.y * g);
    }
    __syncthreads();
    float2* out = A.part + (int64_t)P.n * A.G * A.chunks + P.j;
    gn_sum_groups<THREADS, float2>(A.G, A.per, channel, [&](int g, const float2& t) { out[(int64_t)g * A.chunks] = t; });
}

// All CTAs of the (cooperative, hence co-resident) launch meet: what each wrote before is seen by all after.
// A wait that runs out is reported and left, as every wait of the library.
__device__ __forceinline__ void gn_meet(uint32_t* arrived) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(arrived) : "memory");
        uint64_t t0 = 0;
        for (uint32_t it = 1;; ++it) {
            uint32_t v;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(arrived) : "memory");
            if (v >= gridDim.x) break;
            if ((it & 0x3FFu) == 0u) {
                const uint64_t now = global_timer_ns();
                if (t0 == 0) t0 = now;
                if (now - t0 > kWaitLimitNs) {
                    report_timeout(kWaitMeet);
                    break;
                }
            }
        }
    }
    __syncthreads();
}

// The sample's numbers ([N, G, chunks]: a group's are neighbours), a warp per group: stat[g] = finish(g, mean of the first, mean of the second).
template <int THREADS, typename Part, typename Finish>
__device__ __forceinline__ void gn_team_join(const GnArgs& A, int n, const Part* part, float2* stat, Finish finish) {
    const int lane = threadIdx.x & 31;
    for (int g = threadIdx.x >> 5; g < A.G; g += THREADS / 32) {
        const Part* base = part + ((int64_t)n * A.G + g) * A.chunks;
        double a = 0.0, b = 0.0;
        Part t[5];
        for (int i = lane; i < A.chunks; i += 5 * 32) {  // at most 148 chunks: once
#pragma unroll
            for (int u = 0; u < 5; ++u) t[u] = i + 32 * u < A.chunks ? __ldcg(base + i + 32 * u) : Part{};
#pragma unroll
            for (int u = 0; u < 5; ++u) {
                a += t[u].x;
                b += t[u].y;
            }
        }
        a = warp_sum(a) * A.inv;
        b = warp_sum(b) * A.inv;
        if (lane == 0) stat[g] = finish(g, a, b);
    }
    __syncthreads();
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnFusedThreads, 1) gn_fused_kernel(const __grid_constant__ GnArgs A) {
    constexpr int THREADS = kGnFusedThreads, D = GnDepth<T, V>::fused;
    extern __shared__ __align__(16) uint8_t raw[];
    float2* sums = reinterpret_cast<float2*>(raw + TwoWay<D, 1, THREADS, T, V>::kRingBytes);
    __shared__ float pivots[kGnFusedGroups];  // y may be x: what was subtracted is kept
    const GnTeam<V, THREADS> P(A);
    const T* x = static_cast<const T*>(A.x) + (int64_t)P.n * A.xn;
    TwoWay<D, 1, THREADS, T, V> walk(raw, P.count, x + P.c0 + P.s0 * A.xs, P.lanes * A.xs, nullptr, 0);
    for (int g = threadIdx.x; g < A.G; g += THREADS) pivots[g] = to_f32(x[g * A.per]);
    __syncthreads();
    {
        GnMoments<V> moments;
        walk.forward([&](const Vec<T, V>& in) { moments.add(widen2<T, V>(in)); });
        moments.flush();
        float pivot[V];
        gn_by_channel<V>(A.per, P.c0, [&](int i, int g) { pivot[i] = pivots[g]; }, [&](int i) { pivot[i] = pivot[0]; });
        gn_team_moments<V, THREADS>(A, P, moments, pivot, reinterpret_cast<double2*>(sums));
    }
    float ga[V], be[V];
    gn_params<V>(A, P.c0, ga, be);  // before the wait; at the start, next to the streams, 148 CTAs' reads of one line took 4 us
    gn_meet(A.arrived);
    gn_team_join<THREADS>(A, P.n, A.part64, sums, [&](int g, double m1, double m2) {
        const float2 t = gn_mean_rstd((double)pivots[g], m1, m2, A.eps);
        if (P.j == 0 && A.mean) A.mean[(int64_t)P.n * A.G + g] = t.x;
        if (P.j == 0 && A.rstd) A.rstd[(int64_t)P.n * A.G + g] = t.y;
        return t;
    });
    if (!P.on) return;
    const GnScale<V> scale = gn_scale<V>(A, P.c0, sums, ga, be);
    T* q = static_cast<T*>(A.y) + (int64_t)P.n * A.yn + P.c0 + (P.s0 + (int64_t)(P.count - 1) * P.lanes) * A.ys;
    const int64_t back = -(int64_t)P.lanes * A.ys;
    walk.backward([&](const Vec<T, V>& in) {
        const Pairs<V> f = widen2<T, V>(in);
        Pairs<V> o;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) o.p[i] = act_value2<ACT, true>(scale(f.p[i], i));
        store_streaming<T, V>(q, narrow2<T, V>(o));
        q += back;
    });
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnFusedGradThreads, 1) gn_fused_grad_kernel(const __grid_constant__ GnArgs A) {
    constexpr int THREADS = kGnFusedGradThreads, D = GnDepth<T, V>::fused_grad;
    extern __shared__ __align__(16) uint8_t raw[];
    float2* sums = reinterpret_cast<float2*>(raw + TwoWay<D, 2, THREADS, T, V>::kRingBytes);
    const GnTeam<V, THREADS> P(A);
    TwoWay<D, 2, THREADS, T, V> walk(raw, P.count, static_cast<const T*>(A.x) + (int64_t)P.n * A.xn + P.c0 + P.s0 * A.xs, P.lanes * A.xs,
                                     static_cast<const T*>(A.dy) + (int64_t)P.n * A.dn + P.c0 + P.s0 * A.ds, P.lanes * A.ds);
    float rs[V], ga[V];
    const GnGrad<V> K = gn_constants<V>(A, P.n, P.c0, rs, ga);
    {
        Pairs<V> s1, s2;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = s2.p[i] = 0ull;
        walk.forward([&](const Vec<T, V>& xv, const Vec<T, V>& dv) {
            const Pairs<V> x = widen2<T, V>(xv), dy = widen2<T, V>(dv);
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) {
                uint64_t dz, h;
                K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
                s1.p[i] = f2_add(s1.p[i], dz);
                s2.p[i] = f2_fma(dz, h, s2.p[i]);
            }
        });
        gn_team_sums<V, THREADS>(A, P, s1, s2, sums);
    }
    gn_meet(A.arrived);
    gn_team_join<THREADS>(A, P.n, A.part, sums, [](int, double m1, double m2) { return make_float2((float)m1, (float)m2); });
    if (P.on && A.y) {
        const GnDx<V> dx = gn_dx<V>(A, P.c0, sums, rs, ga);
        T* q = static_cast<T*>(A.y) + (int64_t)P.n * A.yn + P.c0 + (P.s0 + (int64_t)(P.count - 1) * P.lanes) * A.ys;
        const int64_t back = -(int64_t)P.lanes * A.ys;
        walk.backward([&](const Vec<T, V>& xv, const Vec<T, V>& dv) {
            const Pairs<V> x = widen2<T, V>(xv), dy = widen2<T, V>(dv);
            Pairs<V> o;
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) {
                uint64_t dz, h;
                K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
                o.p[i] = dx(dz, h, i);
            }
            store_streaming<T, V>(q, narrow2<T, V>(o));
            q += back;
        });
    }
    if (!A.dgamma && !A.dbeta) return;
    // the parameters' gradients: a warp per channel, the channels dealt out over the CTAs
    const int lane = threadIdx.x & 31, ctas = (int)gridDim.x;
    for (int c = (threadIdx.x >> 5) * ctas + blockIdx.x; c < A.C; c += ctas * (THREADS / 32)) {
        double a = 0.0, b = 0.0;
#pragma unroll 5
        for (int i = lane; i < ctas; i += 32) {
            const float2 t = __ldcg(A.part_c + (int64_t)c * ctas + i);
            a += t.x;
            b += t.y;
        }
        a = warp_sum(a);
        b = warp_sum(b);
        if (lane == 0) {
            if (A.dbeta) A.dbeta[c] = (float)a;
            if (A.dgamma) A.dgamma[c] = (float)b;
        }
    }
}

// ------------------------------------------------------------------ small tensors: one launch

// Sums of one pair per (lane, channel) over the lanes and the channels of each group, in fp64: out[g].
__device__ __forceinline__ void gn_small_groups(const float2* red, int lanes, int width, int per, int groups, double2* out) {
    __syncthreads();
    for (int g = threadIdx.x >> 5; g < groups; g += kGnThreads / 32) {
        double a = 0.0, b = 0.0;
        for (int i = threadIdx.x & 31; i < lanes * per; i += 32) {
            const int l = i / per;
            const float2 u = red[l * width + g * per + (i - l * per)];
            a += u.x;
            b += u.y;
        }
        a = warp_sum(a);
        b = warp_sum(b);
        if ((threadIdx.x & 31) == 0) out[g] = make_double2(a, b);
    }
    __syncthreads();
}

// Brings a thread's pieces (places r, r + lanes, ...) into shared memory, all in flight together; gn_small_brought() waits for them.
template <typename T, int V>
__device__ __forceinline__ void gn_small_bring(bool on, int r, int lanes, int S, const T* from, int64_t pitch, Vec<T, V>* to, int vecs) {
    if (!on) return;
    if constexpr (sizeof(Vec<T, V>) >= 4) {
        for (int s = r; s < S; s += lanes) {
            const uint32_t at = smem_u32(to + s * vecs);
            if constexpr (sizeof(Vec<T, V>) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from + s * pitch) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(from + s * pitch) : "memory");
        }
    } else {
        constexpr int U = 16;
        for (int s = r; s < S; s += U * lanes) {
            Vec<T, V> in[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u * lanes < S) in[u] = *reinterpret_cast<const Vec<T, V>*>(from + (s + u * lanes) * pitch);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u * lanes < S) to[(s + u * lanes) * vecs] = in[u];
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void gn_small_brought() {
    if constexpr (sizeof(Vec<T, V>) >= 4) asm volatile("cp.async.wait_all;" ::: "memory");
}

// A CTA: `vecs` vectors of whole groups, all places of sample blockIdx.y.  Every thread keeps to the places it
// loaded itself, so only the sums go through barriers.  The mean first, from sums about the first place's first
// channel; then the squares about that mean.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) gn_small_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int width = A.vecs * V, v = threadIdx.x % A.vecs, r = threadIdx.x / A.vecs, n = blockIdx.y;
    const int cbase = blockIdx.x * width, here = min(A.C - cbase, width), groups = here / A.per, c0 = cbase + v * V;
    const bool on = r < A.lanes && v * V < here;
    const int S = (int)A.S;
    Vec<T, V>* data = reinterpret_cast<Vec<T, V>*>(raw);
    float2* red = reinterpret_cast<float2*>(raw + align_up((int64_t)S * width * sizeof(T), 16));
    double2* totals = reinterpret_cast<double2*>(red + align_up(A.lanes * width, 2));
    const T* base = static_cast<const T*>(A.x) + (int64_t)n * A.xn;
    wait_predecessor();
    release_successor();
    Pairs<V> mu, s1;
    gn_small_bring<T, V>(on, r, A.lanes, S, base + c0, A.xs, data + v, A.vecs);
    if (on) {
        float pv[V];
        gn_by_channel<V>(A.per, c0, [&](int i, int g) { pv[i] = to_f32(base[g * A.per]); }, [&](int i) { pv[i] = pv[0]; });
        mu.set(pv);
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = 0ull;
        gn_small_brought<T, V>();
        for (int s = r; s < S; s += A.lanes) {
            const Pairs<V> x = widen2<T, V>(data[s * A.vecs + v]);
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = f2_add(s1.p[i], f2_sub(x.p[i], mu.p[i]));
        }
#pragma unroll
        for (int i = 0; i < V; ++i) red[r * width + v * V + i] = make_float2(s1.get(i), 0.f);
    }
    gn_small_groups(red, A.lanes, width, A.per, groups, totals);  // about the pivot
    float mean[V], rs[V];
    if (on) {
        const int g0 = cbase / A.per;
        gn_by_channel<V>(A.per, c0, [&](int i, int g) { mean[i] = (float)((double)mu.get(i) + totals[g - g0].x * A.inv); },
                         [&](int i) { mean[i] = mean[0]; });
        mu.set(mean);
        GnCentred<V> m;
        for (int s = r; s < S; s += A.lanes) m.add(widen2<T, V>(data[s * A.vecs + v]), mu);
        m.flush();
#pragma unroll
        for (int i = 0; i < V; ++i) red[r * width + v * V + i] = make_float2(m.s1.get(i), m.outer.get(i));
    }
    gn_small_groups(red, A.lanes, width, A.per, groups, totals);
    if (!on) return;
    {
        const int g0 = cbase / A.per;
        gn_by_channel<V>(A.per, c0, [&](int i, int g) {
            const double m1 = totals[g - g0].x * A.inv;  // what the first pass's fp32 sums, and the mean's rounding, left
            rs[i] = gn_mean_rstd(0.0, m1, totals[g - g0].y * A.inv, A.eps).y;
            mean[i] = (float)((double)mean[i] + m1);
            if (r == 0 && c0 + i == g * A.per) {
                if (A.mean) A.mean[(int64_t)n * A.G + g] = mean[i];
                if (A.rstd) A.rstd[(int64_t)n * A.G + g] = rs[i];
            }
        }, [&](int i) { rs[i] = rs[0]; mean[i] = mean[0]; });
    }
    float ga[V], be[V];
    gn_params<V>(A, c0, ga, be);
#pragma unroll
    for (int i = 0; i < V; ++i) ga[i] *= rs[i];
    const GnScale<V> scale(mean, ga, be);
    T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + c0;
    for (int s = r; s < S; s += A.lanes) {
        const Pairs<V> x = widen2<T, V>(data[s * A.vecs + v]);
        Pairs<V> o;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) o.p[i] = act_value2<ACT, true>(scale(x.p[i], i));
        *reinterpret_cast<Vec<T, V>*>(q + s * A.ys) = narrow2<T, V>(o);
    }
}

// Its gradients; the parameters' are final where there is one sample, and otherwise left in part_c [N, C] for gn_small_join_kernel.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kGnThreads) gn_small_grad_kernel(const __grid_constant__ GnArgs A) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int width = A.vecs * V, v = threadIdx.x % A.vecs, r = threadIdx.x / A.vecs, n = blockIdx.y;
    const int cbase = blockIdx.x * width, here = min(A.C - cbase, width), groups = here / A.per, c0 = cbase + v * V;
    const bool on = r < A.lanes && v * V < here;
    const int S = (int)A.S;
    const int64_t slice = align_up((int64_t)S * width * sizeof(T), 16);
    Vec<T, V>* xd = reinterpret_cast<Vec<T, V>*>(raw);
    Vec<T, V>* dd = reinterpret_cast<Vec<T, V>*>(raw + slice);
    float2* red = reinterpret_cast<float2*>(raw + 2 * slice);
    float2* sums = red + A.lanes * width;   // per channel
    float2* gsum = sums + width;            // per group
    wait_predecessor();
    release_successor();
    const T* p = static_cast<const T*>(A.x) + (int64_t)n * A.xn + c0;
    const T* d = static_cast<const T*>(A.dy) + (int64_t)n * A.dn + c0;
    // everything of this thread at once; it reads only what it brought itself
    gn_small_bring<T, V>(on, r, A.lanes, S, p, A.xs, xd + v, A.vecs);
    gn_small_bring<T, V>(on, r, A.lanes, S, d, A.ds, dd + v, A.vecs);
    float rs[V], ga[V];
    const GnGrad<V> K = gn_constants<V>(A, n, on ? c0 : cbase, rs, ga);
    gn_small_brought<T, V>();
    Pairs<V> s1, s2;
#pragma unroll
    for (int i = 0; i < Pairs<V>::N; ++i) s1.p[i] = s2.p[i] = 0ull;
    if (on) {
        for (int s = r; s < S; s += A.lanes) {
            const Pairs<V> x = widen2<T, V>(xd[s * A.vecs + v]), dy = widen2<T, V>(dd[s * A.vecs + v]);
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) {
                uint64_t dz, h;
                K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
                s1.p[i] = f2_add(s1.p[i], dz);
                s2.p[i] = f2_fma(dz, h, s2.p[i]);
            }
        }
    }
    if (r < A.lanes) gn_put_sums<V>(A.lanes * A.vecs, s1, s2, red);
    gn_sum_lanes(r < A.lanes, r, A.lanes, A.vecs, V, red);
    for (int c = threadIdx.x; c < here; c += kGnThreads) {
        const float2 t = red[(c % V) * (A.lanes * A.vecs) + c / V];
        if (A.N > 1) {
            A.part_c[(int64_t)n * A.C + cbase + c] = t;
        } else {
            if (A.dbeta) A.dbeta[cbase + c] = t.x;
            if (A.dgamma) A.dgamma[cbase + c] = t.y;
        }
        const float g = gn_param(A.gamma, A.params_f32, A.params_bf16, cbase + c, 1.0f);
        sums[c] = make_float2(t.x * g, t.y * g);
    }
    __syncthreads();
    const float inv = (float)A.inv;
    for (int g = threadIdx.x >> 5; g < groups; g += kGnThreads / 32) {
        float2 t = make_float2(0.f, 0.f);
        for (int i = threadIdx.x & 31; i < A.per; i += 32) {
            t.x += sums[g * A.per + i].x;
            t.y += sums[g * A.per + i].y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            t.x += __shfl_xor_sync(0xFFFFFFFFu, t.x, o);
            t.y += __shfl_xor_sync(0xFFFFFFFFu, t.y, o);
        }
        if ((threadIdx.x & 31) == 0) gsum[g] = make_float2(t.x * inv, t.y * inv);
    }
    __syncthreads();
    if (!on || !A.y) return;
    T* q = static_cast<T*>(A.y) + (int64_t)n * A.yn + c0;
    const GnDx<V> dx = gn_dx<V>(A, c0, gsum - cbase / A.per, rs, ga);
    for (int s = r; s < S; s += A.lanes) {
        const Pairs<V> x = widen2<T, V>(xd[s * A.vecs + v]), dy = widen2<T, V>(dd[s * A.vecs + v]);
        Pairs<V> o;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            uint64_t dz, h;
            K.template dz<ACT>(x.p[i], dy.p[i], i, dz, h);
            o.p[i] = dx(dz, h, i);
        }
        *reinterpret_cast<Vec<T, V>*>(q + s * A.ys) = narrow2<T, V>(o);
    }
}

__global__ void __launch_bounds__(kGnThreads) gn_small_join_kernel(const __grid_constant__ GnArgs A) {
    const int c = blockIdx.x * kGnThreads + threadIdx.x;
    wait_predecessor();
    release_successor();
    if (c >= A.C) return;
    double a = 0.0, b = 0.0;
#pragma unroll 8
    for (int n = 0; n < A.N; ++n) {
        const float2 t = A.part_c[(int64_t)n * A.C + c];
        a += t.x;
        b += t.y;
    }
    if (A.dbeta) A.dbeta[c] = (float)a;
    if (A.dgamma) A.dgamma[c] = (float)b;
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
// without the tensors): V is decided at the call, and all widths use the same chunks.
struct GnPlan {
    int chunks;
    int64_t rows;
};
inline GnPlan gn_plan(int64_t N, int64_t S, int per_sm) {
    // One wave of CTAs (four per SM forward, two backward) over all samples; a chunk has at least 32 places, so that a small
    // tensor's second pass has few partial sums to add up.
    int64_t chunks = (148 * per_sm + N - 1) / N;
    const int64_t most = ceil_div(S, 32);
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    GnPlan p;
    p.rows = ceil_div(S, chunks);
    p.chunks = (int)ceil_div(S, p.rows);
    return p;
}
constexpr int kGnFusedCtas = 148;  // SMs of a B200: the most CTAs of a one-launch kernel
// Pieces that a group wider than a CTA's vectors is cut into, at most (single-element accesses).
inline int64_t gn_pieces(int64_t per) { return ceil_div(per, kGnMaxVecs); }
struct GnRoom {
    int64_t pivot_off, stat_off, part_c_off, arrived_off, total;
};
inline GnRoom gn_room(int64_t N, int64_t S, int64_t C, int64_t G) {
    const GnPlan p = gn_plan(N, S, 4);
    const int64_t slots = N * p.chunks > kGnFusedCtas ? N * p.chunks : kGnFusedCtas;  // CTAs that write sums, either way
    GnRoom r;
    r.pivot_off = align_up(slots * G * gn_pieces(C / G) * 16, 256);  // two fp64 numbers
    r.stat_off = r.pivot_off + align_up(N * G * 4, 256);
    r.part_c_off = r.stat_off + align_up(N * G * 8, 256);
    r.arrived_off = r.part_c_off + align_up(slots * C * 8, 256);
    r.total = r.arrived_off + 256;
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

// The one-launch kernels: the fewest whole groups that fill 64 bytes of a place (or all channels, if
// those are fewer), so that a warp's loads are whole sectors; used where their places fit kGnSmallSmem, which
// leaves room for three CTAs per SM.  A tensor of more than kGnSmallBytes is left to the kernels above, whose loads are whole rows:
// samples of 1000 places of 512 channels, small kernel and those: 8 MB 13.4 and 15.8 us, 16 MB 19.0 and 22.2, but 16 MB in 64 samples 26.6 and 22.1.
constexpr int64_t kGnSmallSmem = 64 << 10, kGnSmallBytes = 8 << 20;
template <typename T, int V>
static bool gn_small_cut(GnArgs& A, bool backward, size_t* smem) {
    if (A.C % V != 0) return false;
    int64_t width = A.per;
    while (width % V != 0 || (width * (int64_t)sizeof(T) < 64 && width < A.C)) width += A.per;
    if (width > A.C) width = A.C;
    if (width % V != 0 || width / V > kGnThreads) return false;
    const int64_t bytes = A.S * width * (int64_t)sizeof(T);
    if (bytes * (backward ? 2 : 1) > kGnSmallSmem || (int64_t)A.N * A.S * A.C * (int64_t)sizeof(T) > kGnSmallBytes) return false;
    A.vecs = (int)(width / V);
    A.lanes = kGnThreads / A.vecs;
    if (A.lanes > A.S) A.lanes = (int)A.S;
    A.blocks = (int)ceil_div(A.C, width);
    const int64_t slice = align_up(bytes, 16), red = (int64_t)A.lanes * width;
    *smem = (size_t)((backward ? 2 : 1) * slice + (align_up(red, 2) + 2 * width) * 8);
    return true;
}

template <typename Kern>
static bool gn_small_ready(PerDevice<int>& cache, Kern kern) {
    return cache.get([&](int&, int) {
        // 64 KB of data, at most 256 x 8 sums of 8 bytes, two numbers of 8 bytes for each of at most 2048 channels
        return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGnSmallSmem + 52 * 1024) == cudaSuccess;
    }) != nullptr;
}

// One CTA per SM, shared evenly among the samples; taken where that keeps at least two SMs in three busy.  Samples of 2000 places
// of 512 channels, this and three launches: 100 samples (100 SMs) 126 and 121 us forward, 206 and 230 backward; 80 samples 127 and
// 108, 205 and 179.
// Returns whether the call was made; *e says how it went.
template <typename Kern>
static bool launch_gn_fused(PerDevice<int>& cache, Kern kern, GnArgs A, int V, int threads, size_t smem, int64_t most_channels, cudaStream_t st,
                            cudaError_t* e) {
    if (A.C % V != 0 || A.C > most_channels || A.G > kGnFusedGroups) return false;
    const int* sms = cache.get([&](int& n, int dev) {
        int per_sm = 0, coop = 0;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, smem) != cudaSuccess ||
            cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&coop, cudaDevAttrCooperativeLaunch, dev) != cudaSuccess)
            return false;
        if (per_sm < 1 || !coop) n = 0;
        if (n > kGnFusedCtas) n = kGnFusedCtas;
        return true;
    });
    if (!sms || *sms == 0) return false;
    int chunks = *sms / A.N;
    if (chunks < 1 || (int64_t)chunks * A.N * 3 < (int64_t)*sms * 2) return false;
    A.rows = ceil_div(A.S, chunks);
    A.chunks = (int)ceil_div(A.S, A.rows);
    A.vecs = A.C / V;
    if ((*e = cudaMemsetAsync(A.arrived, 0, sizeof(uint32_t), st)) != cudaSuccess) return true;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(A.chunks * A.N));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    *e = cudaLaunchKernelEx(&cfg, kern, A);
    return true;
}

template <typename T, int V, int ACT>
static bool launch_gn_small(GnArgs A, bool backward, cudaStream_t st, cudaError_t* e) {
    size_t smem = 0;
    if (!gn_small_cut<T, V>(A, backward, &smem)) return false;
    static PerDevice<int> ready, ready_grad;
    const dim3 block(kGnThreads);
    *e = cudaErrorInvalidValue;
    if (!backward) {
        if (gn_small_ready(ready, gn_small_kernel<T, V, ACT>))
            *e = launch_after(gn_small_kernel<T, V, ACT>, dim3((unsigned)A.blocks, (unsigned)A.N), block, smem, st, A);
    } else if (gn_small_ready(ready_grad, gn_small_grad_kernel<T, V, ACT>)) {
        *e = launch_after(gn_small_grad_kernel<T, V, ACT>, dim3((unsigned)A.blocks, (unsigned)A.N), block, smem, st, A);
        if (*e == cudaSuccess && A.N > 1 && (A.dgamma || A.dbeta))
            *e = launch_after(gn_small_join_kernel, dim3((unsigned)ceil_div(A.C, kGnThreads)), block, 0, st, A);
    }
    return true;
}

template <typename T, int V, int ACT>
static bool launch_gn_one(const GnArgs& A, bool backward, cudaStream_t st, cudaError_t* e) {
    static PerDevice<int> fused, fused_grad;
    constexpr size_t sums = (size_t)kGnFusedThreads * GnRound<V>::units * sizeof(double2), grad_sums = (size_t)kGnFusedGradThreads * V * sizeof(float2);
    constexpr size_t ring = TwoWay<GnDepth<T, V>::fused, 1, kGnFusedThreads, T, V>::kRingBytes;
    constexpr size_t grad_ring = TwoWay<GnDepth<T, V>::fused_grad, 2, kGnFusedGradThreads, T, V>::kRingBytes;
    static_assert(ring + sums + kGnFusedGroups * 4 <= 232448 && grad_ring + grad_sums <= 232448, "more than the 227 KB of shared memory a CTA can have");
    return !backward ? launch_gn_fused(fused, gn_fused_kernel<T, V, ACT>, A, V, kGnFusedThreads, ring + sums, kGnFusedThreads * V, st, e)
                     : launch_gn_fused(fused_grad, gn_fused_grad_kernel<T, V, ACT>, A, V, kGnFusedGradThreads, grad_ring + grad_sums,
                                       kGnFusedGradThreads * V, st, e);
}

template <typename T, int V, int ACT>
static bool launch_gn_three(GnArgs A, bool backward, cudaStream_t st, cudaError_t* e) {
    if (!gn_cut(A, V)) return false;
    const dim3 grid((unsigned)A.chunks, (unsigned)A.N, (unsigned)A.blocks), block(kGnThreads);
    const unsigned group_ctas = (unsigned)ceil_div((int64_t)A.N * A.G, kGnThreads / 32);
    // the rings; the sums of pass 1 (V pairs per thread) take their place
    constexpr bool ring = WholePieces<T, V>::value;
    constexpr size_t sums = (size_t)kGnThreads * V * sizeof(double2), grad_sums = (size_t)kGnThreads * V * sizeof(float2);
    constexpr size_t one = ring ? (size_t)kGnThreads * 16 * kGnDepth : 0, two = ring ? (size_t)kGnThreads * 16 * 2 * kGnGradDepth : 0;
    static_assert(one <= 48 * 1024 && two <= 48 * 1024 && sums <= 48 * 1024, "more than a kernel has without asking");
    if (!backward) {
        if ((*e = launch_after(gn_stats_kernel<T, V>, grid, block, sums > one ? sums : one, st, A)) != cudaSuccess) return true;
        if ((*e = launch_after(gn_join_kernel<false>, dim3(group_ctas), block, 0, st, A, (int)group_ctas)) != cudaSuccess) return true;
        *e = launch_after(gn_apply_kernel<T, V, ACT>, grid, block, one, st, A);
        return true;
    }
    if ((*e = launch_after(gn_grad_stats_kernel<T, V, ACT>, grid, block, grad_sums > two ? grad_sums : two, st, A)) != cudaSuccess) return true;
    const unsigned channel_ctas = A.dgamma || A.dbeta ? (unsigned)ceil_div(A.C, 32) : 0;
    *e = launch_after(gn_join_kernel<true>, dim3(group_ctas + channel_ctas), block, 0, st, A, (int)group_ctas);
    if (*e == cudaSuccess && A.y) *e = launch_after(gn_grad_apply_kernel<T, V, ACT>, grid, block, two, st, A);
    return true;
}

// Forward, 16-byte pieces: bytes of x for which one launch is the faster.  One and three launches, us: 8 MB 20.6 and 16.3, 32 MB 32.8 and
// 30.6, 61 MB 44.4 and 44.2, 98 MB 60.9 and 62.8, 128 MB 77.1 and 78.2, 205 MB in 100 samples 125.6 and 121.1, 256 MB 145.5 and 143.5.
// Backward the two lie within 13 % of each other either way (8 MB 24.2 and 21.1, 61 MB 61.9 and 63.5, 128 MB 120 and 112): one launch always.
constexpr int64_t kGnOneFrom = 64 << 20, kGnOneTo = 192 << 20;

// `wide`: channels per access that the channel count, pitches and pointers allow.
template <typename T, int ACT>
static cudaError_t launch_gn_act(const GnArgs& A, int wide, bool backward, cudaStream_t st) {
    constexpr int FULL = 16 / (int)sizeof(T);
    cudaError_t e = cudaErrorInvalidValue;
    if (wide == FULL) {
        const int64_t bytes = (int64_t)A.N * A.S * A.C * (int64_t)sizeof(T);
        const bool one = backward || (bytes >= kGnOneFrom && bytes < kGnOneTo);
        if (launch_gn_small<T, FULL, ACT>(A, backward, st, &e) || (one && launch_gn_one<T, FULL, ACT>(A, backward, st, &e)) ||
            launch_gn_three<T, FULL, ACT>(A, backward, st, &e) || (!one && launch_gn_one<T, FULL, ACT>(A, backward, st, &e)))
            return e;  // (three launches do not cut wide groups of an odd number of channels)
    }
    if (launch_gn_small<T, 1, ACT>(A, backward, st, &e)) return e;
    if (wide == FULL / 2 && launch_gn_one<T, FULL / 2, ACT>(A, backward, st, &e)) return e;
    if (wide == FULL / 4 && launch_gn_one<T, FULL / 4, ACT>(A, backward, st, &e)) return e;
    launch_gn_three<T, 1, ACT>(A, backward, st, &e);
    return e;
}

template <typename T>
static cudaError_t launch_gn_t(const GnArgs& A, bool backward, int act, cudaStream_t st) {
    int wide = 16 / (int)sizeof(T);
    for (; wide > 1; wide /= 2) {
        const uintptr_t bytes = (uintptr_t)wide * sizeof(T);
        bool ok = A.C % wide == 0 && aligned_to(A.x, bytes) && aligned_to(A.y, bytes) && aligned_to(A.dy, bytes);
        for (int64_t p : {A.xn, A.xs, A.yn, A.ys, A.dn, A.ds}) ok = ok && p % wide == 0;
        if (ok) break;
    }
    if (act == DVDQ_ACT_GELU_TANH) return launch_gn_act<T, DVDQ_ACT_GELU_TANH>(A, wide, backward, st);
    if (act == DVDQ_ACT_SILU) return launch_gn_act<T, DVDQ_ACT_SILU>(A, wide, backward, st);
    return launch_gn_act<T, DVDQ_ACT_NONE>(A, wide, backward, st);
}

}  // namespace dvdq
