// Rows of C values: RMS norm with the residual's addition, its output in the rows' type or in 8 bits with a scale for each
// row; its gradients; and the 8-bit quantization alone (NORM = false).
//
//   h = x + r,  q = 1 / sqrt(mean h^2 + eps),  y = h q gamma,  s = max|y| / 127,  c = round(y / s)
//   dh = gamma dy,  dx = q (dh - h q mean(dh h q)) + the residual stream's own gradient,  dgamma = sum over rows of dy h q
//
// Everything between the loads and the one rounding of each output is fp32; y and c come from the unrounded h.
//
// What bounds it: memory, each input read once and each output written once.  So a row is held in registers from its loads to its stores
// (P pieces of V channels a thread, 16 bytes where the tensors' alignment allows), and both things that the whole row decides, sum of h^2
// and max |h gamma| (max |y| is q times that), meet in one exchange.  Rows of few pieces share a warp, longer ones take a
// warp, and from there on a CTA each.  Rows beyond 1024 threads' registers (P = 0) are read again from L2 instead of kept.
#pragma once

#include "block_common.cuh"

namespace dvdq {

constexpr int kRowThreads = 1024;  // most threads of a row

// Pitches of a [N, S, C] tensor, in elements, unit stride of channels.
struct RowsOf {
    void* p;
    int64_t outer, row;
};
struct RowsShape {
    int64_t rows;    // N * S
    FastDiv by_s;    // row -> (n, s)
    int S, C;
};
struct RmsArgs {
    RowsShape shape;
    RowsOf x, r, h, y, codes;
    const void* gamma;
    float *scales, *rstd;  // dense [N, S]
    int params_f32;
    float eps, inv_c;
    int lanes;             // threads of a row: a power of two up to 32, or the CTA's
};
struct RmsBackwardArgs {
    RowsShape shape;
    RowsOf dy, h, dh, dx;
    const void* gamma;
    const float* rstd;
    float* part;           // [CTAs, C]: each CTA's sums for dgamma; or NULL
    int params_f32;
    float inv_c;
    int lanes;
};

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// max |.| of a pair and m, NaN if one of them is
__device__ __forceinline__ float max_abs2(float m, uint64_t v) {
    float a, b;
    f2_unpack(v, a, b);
    return max_nan(m, max_nan(fabsf(a), fabsf(b)));
}

// V values of a row from channel c on; those past the row's end are zero and are not read.
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> row_load(const T* p, int c, int C) {
    if (c + V <= C) return *reinterpret_cast<const Vec<T, V>*>(p + c);
    Vec<T, V> v;
#pragma unroll
    for (int j = 0; j < V; ++j) v.e[j] = c + j < C ? p[c + j] : from_f32<T>(0.f);
    return v;
}
template <typename T, int V>
__device__ __forceinline__ void row_store(T* p, int c, int C, const Pairs<V>& f) {
    const Vec<T, V> v = narrow2<T, V>(f);
    if (c + V <= C) {
        *reinterpret_cast<Vec<T, V>*>(p + c) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < C) p[c + j] = v.e[j];
    }
}
template <typename T, int V>
__device__ __forceinline__ Pairs<V> gamma_load(const void* gamma, int params_f32, int c, int C) {  // NULL: ones
    if (!gamma) {
        Pairs<V> g;
#pragma unroll
        for (int j = 0; j < Pairs<V>::N; ++j) g.p[j] = f2_splat(1.0f);
        return g;
    }
    if (sizeof(T) == 4 || !params_f32) return widen2<T, V>(row_load<T, V>(static_cast<const T*>(gamma), c, C));
    constexpr int H = V > 4 ? 4 : V;  // 16 bytes of fp32 at a time
    Pairs<V> g;
#pragma unroll
    for (int j = 0; j < V / H; ++j) {
        const Pairs<H> part = widen2<float, H>(row_load<float, H>(static_cast<const float*>(gamma), c + j * H, C));
#pragma unroll
        for (int i = 0; i < Pairs<H>::N; ++i) g.p[j * Pairs<H>::N + i] = part.p[i];
    }
    return g;
}
__device__ __forceinline__ int64_t row_at(const RowsOf& t, uint32_t n, uint32_t s) { return (int64_t)n * t.outer + (int64_t)s * t.row; }

// ------------------------------------------------------------------ what a whole row decides

// Sum of a and max of b over the threads of a row, the same bits in each of them.  A CTA's warps meet through shared memory;
// `turn` alternates between two sets of slots, so that one barrier a row is enough.
struct RowMeet {
    float2* slots;   // [2][32], where the row has the CTA to itself
    int lanes, turn = 0;
    __device__ __forceinline__ RowMeet(float2* s, int l) : slots(s), lanes(l) {}
    __device__ __forceinline__ float2 operator()(float a, float b) {
        for (int o = (lanes < 32 ? lanes : 32) >> 1; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
            b = max_nan(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
        }
        if (lanes > 32) {
            float2* at = slots + 32 * turn;
            turn ^= 1;
            if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = make_float2(a, b);
            __syncthreads();
            const int warps = lanes >> 5, lane = threadIdx.x & 31;
            if (warps <= 8) {
                a = at[0].x;
                b = at[0].y;
                for (int w = 1; w < warps; ++w) {
                    a += at[w].x;
                    b = max_nan(b, at[w].y);
                }
            } else {
                a = lane < warps ? at[lane].x : 0.f;
                b = lane < warps ? at[lane].y : 0.f;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
                    b = max_nan(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
                }
            }
        }
        return make_float2(a, b);
    }
};

// 2^-e for the power of two 2^e at or below v > 0, at most 2^126: brings v to [1, 2).
__device__ __forceinline__ float bring_to_one(float v) {
    const int e = (int)(__float_as_uint(v) >> 23) - 127;  // -127 below the normal numbers
    return __uint_as_float((uint32_t)(127 - (e < -126 ? -126 : e > 126 ? 126 : e)) << 23);
}

// ------------------------------------------------------------------ forward

// A row's values: kept (P > 0), or loaded at each visit (P = 0).
template <typename T, int V, int P>
struct Row {
    static constexpr int K = P > 0 ? P : 1, N = Pairs<V>::N;
    Pairs<V> v[K];
    const T *x, *r;
    int C, lanes, lane;
    __device__ __forceinline__ int column(int i) const { return (i * lanes + lane) * V; }
    __device__ __forceinline__ static Pairs<V> sum(const Vec<T, V>& a, const Vec<T, V>& b, bool both) {
        Pairs<V> h = widen2<T, V>(a);
        if (both) {
            const Pairs<V> f = widen2<T, V>(b);
#pragma unroll
            for (int j = 0; j < N; ++j) h.p[j] = f2_add(h.p[j], f.p[j]);
        }
        return h;
    }
    __device__ __forceinline__ void load(const T* from, const T* residual, bool active) {
        x = from;
        r = residual;
        if constexpr (P > 0) {
            const int here = active ? C : 0;
            Vec<T, V> a[P], b[P];
#pragma unroll
            for (int i = 0; i < P; ++i) a[i] = row_load<T, V>(x, column(i), here);
            if (r) {
#pragma unroll
                for (int i = 0; i < P; ++i) b[i] = row_load<T, V>(r, column(i), here);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) v[i] = sum(a[i], b[i], r != nullptr);
        }
    }
    // visit(channel, values) for each piece; pieces past the row's end are zero
    template <typename F>
    __device__ __forceinline__ void visit(F f) {
        if constexpr (P > 0) {
#pragma unroll
            for (int i = 0; i < P; ++i) f(column(i), v[i]);
        } else {
            for (int c = column(0); c < C; c += lanes * V) {
                const Vec<T, V> a = row_load<T, V>(x, c, C);
                f(c, sum(a, r ? row_load<T, V>(r, c, C) : a, r != nullptr));
            }
        }
    }
};

// Codes of V channels: y * inv, rounded to a whole number in the one rounding of its addition to 1.5 * 2^23, whose last byte then is the
// code.  |y| inv is at most 127 (1 + 2^-22).
template <int V>
__device__ __forceinline__ void codes_store(int8_t* p, int c, int C, const Pairs<V>& y, float lift, float inv) {
    constexpr int N = Pairs<V>::N;
    uint32_t w[2 * N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float a, b;
        f2_unpack(f2_fma(f2_mul(y.p[j], f2_splat(lift)), f2_splat(inv), f2_splat(12582912.0f)), a, b);
        w[2 * j] = __float_as_uint(a);
        w[2 * j + 1] = __float_as_uint(b);
    }
    if (V >= 2 && c + V <= C) {
        if constexpr (V == 8) {
            uint2 o;
            o.x = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
            o.y = __byte_perm(__byte_perm(w[4], w[5], 0x0040), __byte_perm(w[6], w[7], 0x0040), 0x5410);
            *reinterpret_cast<uint2*>(p + c) = o;
        } else if constexpr (V == 4) {
            *reinterpret_cast<uint32_t*>(p + c) = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
        } else if constexpr (V == 2) {
            *reinterpret_cast<uint16_t*>(p + c) = (uint16_t)__byte_perm(w[0], w[1], 0x0040);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < C) p[c + j] = (int8_t)(w[j] & 0xFFu);
    }
}

// Threads of a row at most: what lets a thread keep its pieces in registers.
template <int V, int P>
struct RowLimit {
    static constexpr int forward = P * V > 24 ? 512 : kRowThreads, backward = P * V > 16 ? 384 : kRowThreads;
};

template <typename T, int V, int P, bool NORM>
__global__ void __launch_bounds__(RowLimit<V, P>::forward)
rms_norm_kernel(const __grid_constant__ RmsArgs A) {
    __shared__ float2 slots[64];
    constexpr int N = Pairs<V>::N;
    const int lanes = A.lanes, lane = lanes > 32 ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    const int groups = lanes > 32 ? 1 : (int)blockDim.x / lanes, group = lanes > 32 ? 0 : (int)threadIdx.x / lanes;
    const int C = A.shape.C;
    RowMeet meet(slots, lanes);
    Row<T, V, P> row;
    row.C = C;
    row.lanes = lanes;
    row.lane = lane;
    wait_predecessor();
    release_successor();
    for (int64_t at = (int64_t)blockIdx.x * groups; at < A.shape.rows; at += (int64_t)gridDim.x * groups) {
        const bool active = at + group < A.shape.rows;
        const uint32_t index = (uint32_t)(active ? at + group : at);  // threads without a row of their own take part in the exchanges
        const uint32_t n = A.shape.by_s(index), s = index - n * (uint32_t)A.shape.S;
        row.load(static_cast<const T*>(A.x.p) + row_at(A.x, n, s), A.r.p ? static_cast<const T*>(A.r.p) + row_at(A.r, n, s) : nullptr, active);
        uint64_t sum = 0ull;
        float top = 0.f;
        row.visit([&](int c, const Pairs<V>& h) {
            if (NORM) {
#pragma unroll
                for (int j = 0; j < N; ++j) sum = f2_fma(h.p[j], h.p[j], sum);
            }
            if (A.scales) {
                const Pairs<V> g = NORM ? gamma_load<T, V>(A.gamma, A.params_f32, c, C) : h;
#pragma unroll
                for (int j = 0; j < N; ++j) top = max_abs2(top, NORM ? f2_mul(h.p[j], g.p[j]) : h.p[j]);
            }
        });
        float s0, s1;
        f2_unpack(sum, s0, s1);
        const float2 all = meet(s0 + s1, top);
        top = all.y;
        float q = 1.0f, f = 1.0f;  // y = (f h) q gamma
        if (NORM) {
            const float m = fmaf(all.x, A.inv_c, A.eps);
            q = 1.0f / sqrtf(m);
            top *= q;
            // Squares that left fp32's range, or an h gamma that did: once more with f h, f a power of two that brings the largest |h|
            // (or sqrt(eps), where that is larger) to 1.  The rows of a warp take the turn together and keep what is theirs.
            const bool far = !(m > 1e-30f && m < 1e30f && top < 3e38f);
            if (lanes > 32 ? far : __any_sync(0xFFFFFFFFu, far)) {
                float largest = 0.f;
                row.visit([&](int, const Pairs<V>& h) {
#pragma unroll
                    for (int j = 0; j < N; ++j) largest = max_abs2(largest, h.p[j]);
                });
                largest = fmaxf(meet(0.f, largest).y, sqrtf(A.eps));
                const float f2 = largest <= 3.4028235e38f && largest > 0.f ? bring_to_one(largest) : 1.0f;
                uint64_t ss = 0ull;
                row.visit([&](int, const Pairs<V>& h) {
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const uint64_t t = f2_mul(h.p[j], f2_splat(f2));
                        ss = f2_fma(t, t, ss);
                    }
                });
                f2_unpack(ss, s0, s1);
                const float q2 = 1.0f / sqrtf(fmaf(meet(s0 + s1, 0.f).x, A.inv_c, A.eps * f2 * f2));
                float top2 = 0.f;
                row.visit([&](int c, const Pairs<V>& h) {
                    const Pairs<V> g = gamma_load<T, V>(A.gamma, A.params_f32, c, C);
#pragma unroll
                    for (int j = 0; j < N; ++j) top2 = max_abs2(top2, f2_mul(f2_mul(f2_mul(h.p[j], f2_splat(f2)), f2_splat(q2)), g.p[j]));
                });
                top2 = meet(0.f, top2).y;
                if (far) {
                    f = f2;
                    q = q2;
                    top = top2;
                }
            }
        }
        if (A.rstd && lane == 0 && active) A.rstd[index] = q * f;
        // codes are y lift inv; a row near the smallest numbers is lifted first, so that 127 / top stays finite
        float lift = 0.f, inv = 0.f;
        if (A.scales) {
            const bool finite = top <= 3.4028235e38f;  // not NaN, not infinite
            if (finite && top > 0.f) {
                lift = top < 1e-30f ? 18446744073709551616.0f : 1.0f;
                inv = 127.0f / (top * lift);
            }
            if (lane == 0 && active) A.scales[index] = finite ? top / 127.0f : __uint_as_float(0x7FC00000u);
        }
        if (!active) continue;
        T* to_h = A.h.p ? static_cast<T*>(A.h.p) + row_at(A.h, n, s) : nullptr;
        T* to_y = A.y.p ? static_cast<T*>(A.y.p) + row_at(A.y, n, s) : nullptr;
        int8_t* to_c = A.codes.p ? static_cast<int8_t*>(A.codes.p) + row_at(A.codes, n, s) : nullptr;
        row.visit([&](int c, const Pairs<V>& h) {
            if (c >= C) return;
            if (to_h) row_store<T, V>(to_h, c, C, h);
            if (!to_y && !to_c) return;
            Pairs<V> y = h;
            if (NORM) {
                const Pairs<V> g = gamma_load<T, V>(A.gamma, A.params_f32, c, C);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (f != 1.0f) y.p[j] = f2_mul(y.p[j], f2_splat(f));
                    y.p[j] = f2_mul(f2_mul(y.p[j], f2_splat(q)), g.p[j]);
                }
            }
            if (to_y) row_store<T, V>(to_y, c, C, y);
            if (to_c) {
                if (inv == 0.f) {  // zeros, or not finite: codes 0
#pragma unroll
                    for (int j = 0; j < N; ++j) y.p[j] = 0ull;
                }
                codes_store<V>(to_c, c, C, y, lift, inv);
            }
        });
    }
}

// ------------------------------------------------------------------ gradients

// A thread's channels are the same in every row that it meets, so dgamma's sums stay with it (P > 0: in registers; P = 0: in the CTA's own
// row of `part`) until the CTA has been through its rows.
template <typename T, int V, int P>
__global__ void __launch_bounds__(RowLimit<V, P>::backward)
rms_norm_backward_kernel(const __grid_constant__ RmsBackwardArgs A) {
    __shared__ float2 slots[64];
    extern __shared__ float joined[];  // rows that share a CTA: their sums for dgamma, [groups][C]
    constexpr int N = Pairs<V>::N, K = P > 0 ? P : 1;
    const int lanes = A.lanes, lane = lanes > 32 ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    const int groups = lanes > 32 ? 1 : (int)blockDim.x / lanes, group = lanes > 32 ? 0 : (int)threadIdx.x / lanes;
    const int C = A.shape.C;
    RowMeet meet(slots, lanes);
    Pairs<V> acc[K];
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i].p[j] = 0ull;
    float* mine = A.part ? A.part + (int64_t)blockIdx.x * C : nullptr;
    wait_predecessor();
    release_successor();
    auto gamma = [&](int c) { return gamma_load<T, V>(A.gamma, A.params_f32, c, C); };
    bool first = true;
    for (int64_t at = (int64_t)blockIdx.x * groups; at < A.shape.rows; at += (int64_t)gridDim.x * groups) {
        const bool active = at + group < A.shape.rows;
        const uint32_t index = (uint32_t)(active ? at + group : at);
        const uint32_t n = A.shape.by_s(index), s = index - n * (uint32_t)A.shape.S;
        const T* dy = static_cast<const T*>(A.dy.p) + row_at(A.dy, n, s);
        const T* h = static_cast<const T*>(A.h.p) + row_at(A.h, n, s);
        const T* dh = A.dh.p ? static_cast<const T*>(A.dh.p) + row_at(A.dh, n, s) : nullptr;
        T* dx = A.dx.p ? static_cast<T*>(A.dx.p) + row_at(A.dx, n, s) : nullptr;
        const float q = A.rstd[index];
        uint64_t sum = 0ull;
        if constexpr (P > 0) {
            const int here = active ? C : 0;
            Vec<T, V> a[P], b[P], e[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                a[i] = row_load<T, V>(dy, (i * lanes + lane) * V, here);
                b[i] = row_load<T, V>(h, (i * lanes + lane) * V, here);
            }
            if (dh && dx) {
#pragma unroll
                for (int i = 0; i < P; ++i) e[i] = row_load<T, V>(dh, (i * lanes + lane) * V, here);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const Pairs<V> d = widen2<T, V>(a[i]), hh = widen2<T, V>(b[i]), g = gamma((i * lanes + lane) * V);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const uint64_t t = f2_mul(d.p[j], f2_mul(hh.p[j], f2_splat(q)));
                    acc[i].p[j] = f2_add(acc[i].p[j], t);
                    sum = f2_fma(t, g.p[j], sum);
                }
            }
            if (dx) {
                float s0, s1;
                f2_unpack(sum, s0, s1);
                const float mean = meet(s0 + s1, 0.f).x * A.inv_c;
                if (active) {
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const int c = (i * lanes + lane) * V;
                        if (c < C) {
                            const Pairs<V> d = widen2<T, V>(a[i]), hh = widen2<T, V>(b[i]), g = gamma(c);
                            Pairs<V> o;
#pragma unroll
                            for (int j = 0; j < N; ++j) {
                                const uint64_t along = f2_mul(f2_mul(hh.p[j], f2_splat(q)), f2_splat(mean));
                                o.p[j] = f2_mul(f2_sub(f2_mul(d.p[j], g.p[j]), along), f2_splat(q));
                            }
                            if (dh) {
                                const Pairs<V> more = widen2<T, V>(e[i]);
#pragma unroll
                                for (int j = 0; j < N; ++j) o.p[j] = f2_add(o.p[j], more.p[j]);
                            }
                            row_store<T, V>(dx, c, C, o);
                        }
                    }
                }
            }
        } else {
            for (int c = lane * V; c < C; c += lanes * V) {
                const Pairs<V> d = widen2<T, V>(row_load<T, V>(dy, c, C)), hh = widen2<T, V>(row_load<T, V>(h, c, C)), g = gamma(c);
                Pairs<V> t;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    t.p[j] = f2_mul(d.p[j], f2_mul(hh.p[j], f2_splat(q)));
                    sum = f2_fma(t.p[j], g.p[j], sum);
                }
                if (mine) {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (c + j < C) mine[c + j] = first ? t.get(j) : mine[c + j] + t.get(j);
                }
            }
            first = false;
            if (dx) {
                float s0, s1;
                f2_unpack(sum, s0, s1);
                const float mean = meet(s0 + s1, 0.f).x * A.inv_c;
                for (int c = lane * V; c < C; c += lanes * V) {
                    const Pairs<V> d = widen2<T, V>(row_load<T, V>(dy, c, C)), hh = widen2<T, V>(row_load<T, V>(h, c, C)), g = gamma(c);
                    Pairs<V> o;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const uint64_t along = f2_mul(f2_mul(hh.p[j], f2_splat(q)), f2_splat(mean));
                        o.p[j] = f2_mul(f2_sub(f2_mul(d.p[j], g.p[j]), along), f2_splat(q));
                    }
                    if (dh) {
                        const Pairs<V> more = widen2<T, V>(row_load<T, V>(dh, c, C));
#pragma unroll
                        for (int j = 0; j < N; ++j) o.p[j] = f2_add(o.p[j], more.p[j]);
                    }
                    row_store<T, V>(dx, c, C, o);
                }
            }
        }
    }
    if constexpr (P > 0) {
        if (!mine) return;
        if (lanes > 32) {
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = (i * lanes + lane) * V + j;
                    if (c < C) mine[c] = acc[i].get(j);
                }
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = (i * lanes + lane) * V + j;
                    if (c < C) joined[group * C + c] = acc[i].get(j);
                }
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += blockDim.x) {
                float t = 0.f;
                for (int g = 0; g < groups; ++g) t += joined[g * C + c];
                mine[c] = t;
            }
        }
    }
}

// dgamma from the CTAs' sums, in fp64 and in a fixed order: 32 channels a CTA, 16 warps share its rows.
constexpr int kRmsJoinWarps = 16;
__global__ void __launch_bounds__(kRmsJoinWarps * 32) rms_norm_join_kernel(const float* __restrict__ part, int parts, int C, float* __restrict__ out) {
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
__global__ void __launch_bounds__(256) rms_norm_no_rows_kernel(float* __restrict__ dgamma, int C) {
    wait_predecessor();
    release_successor();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < C) dgamma[c] = 0.f;
}

// ------------------------------------------------------------------ host side

struct RowsPlan {
    int lanes, threads, pieces;  // pieces 0: the row is read again instead of kept
};
// How `rows` rows of nv pieces are laid over threads.  pieces <= `most` can be kept by a thread, of CTAs of up to limit(pieces) threads.
template <typename Limit>
inline RowsPlan rows_plan(int64_t rows, int64_t nv, int most, Limit limit) {
    RowsPlan p;
    if (nv <= 64 || (nv <= 32 * most && rows >= 148 * 8)) {  // a warp or part of it
        int lanes = 32;
        while (lanes > 1 && nv <= lanes) lanes >>= 1;  // two pieces a thread, where there are two
        p.lanes = lanes;
        p.threads = 128;
        p.pieces = (int)ceil_div(nv, lanes);
        return p;
    }
    // a CTA: few rows take as many threads as there are pieces, many rows fewer threads with several pieces each
    p.pieces = 0;
    int64_t best = 0;
    for (int k = rows < 148 * 2 ? 1 : most < 4 ? most : 4; k <= most; ++k) {
        const int64_t threads = align_up(ceil_div(nv, k), 32);
        if (threads > limit(k)) continue;
        if (p.pieces == 0 || threads * k < best) {
            best = threads * k;
            p.pieces = k;
            p.threads = (int)(threads < 64 ? 64 : threads);
            if (rows < 148 * 2) break;
        }
    }
    if (p.pieces == 0) p.threads = kRowThreads;
    p.lanes = p.threads;
    return p;
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

constexpr int kRowsMost = 8, kRowsBackwardMost = 5;

template <typename T, int V, int P, bool NORM>
static cudaError_t launch_rms_p(const RmsArgs& A0, const RowsPlan& p, cudaStream_t st) {
    RmsArgs A = A0;
    A.lanes = p.lanes;
    const int64_t ctas = p.lanes > 32 ? A.shape.rows : ceil_div(A.shape.rows, p.threads / p.lanes);
    const int64_t most = 148 * (2048 / p.threads);
    return launch_after(rms_norm_kernel<T, V, P, NORM>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(p.threads), 0, st, A);
}
template <typename T, int V, bool NORM>
static cudaError_t launch_rms_v(const RmsArgs& A, cudaStream_t st) {
    const RowsPlan p = rows_plan(A.shape.rows, ceil_div(A.shape.C, V), kRowsMost, [](int k) { return k * V > 24 ? 512 : kRowThreads; });
    switch (p.pieces) {
        case 0: return launch_rms_p<T, V, 0, NORM>(A, p, st);
        case 1: return launch_rms_p<T, V, 1, NORM>(A, p, st);
        case 2: return launch_rms_p<T, V, 2, NORM>(A, p, st);
        case 3: return launch_rms_p<T, V, 3, NORM>(A, p, st);
        case 4: return launch_rms_p<T, V, 4, NORM>(A, p, st);
        case 5: return launch_rms_p<T, V, 5, NORM>(A, p, st);
        case 6: return launch_rms_p<T, V, 6, NORM>(A, p, st);
        default: return launch_rms_p<T, V, 8, NORM>(A, p, st);
    }
}
// `access`: bytes of a piece that every tensor's alignment allows: 16, 4 or the element's
template <typename T, bool NORM>
static cudaError_t launch_rms_t(const RmsArgs& A, int access, cudaStream_t st) {
    if (access == 16) return launch_rms_v<T, 16 / sizeof(T), NORM>(A, st);
    if (sizeof(T) == 2 && access == 4) return launch_rms_v<T, 4 / sizeof(T), NORM>(A, st);
    return launch_rms_v<T, 1, NORM>(A, st);
}

template <typename T, int V, int P>
static cudaError_t launch_rms_backward_p(const RmsBackwardArgs& A0, const RowsPlan& p, int64_t parts, int* ctas_out, cudaStream_t st) {
    RmsBackwardArgs A = A0;
    A.lanes = p.lanes;
    const int groups = p.lanes > 32 ? 1 : p.threads / p.lanes;
    int64_t ctas = ceil_div(A.shape.rows, groups);
    const int64_t most = 148 * (2048 / p.threads);
    ctas = ctas < most ? ctas : most;
    if (A.part && ctas > parts) ctas = parts;
    *ctas_out = (int)ctas;
    const size_t joined = A.part && groups > 1 ? (size_t)groups * A.shape.C * 4 : 0;  // 128 threads' sums: 20 KB at most
    return launch_after(rms_norm_backward_kernel<T, V, P>, dim3((unsigned)ctas), dim3(p.threads), joined, st, A);
}
template <typename T, int V>
static cudaError_t launch_rms_backward_v(const RmsBackwardArgs& A, int64_t parts, int* ctas, cudaStream_t st) {
    const RowsPlan p = rows_plan(A.shape.rows, ceil_div(A.shape.C, V), kRowsBackwardMost, [](int k) { return k * V > 16 ? 384 : kRowThreads; });
    switch (p.pieces) {
        case 0: return launch_rms_backward_p<T, V, 0>(A, p, parts, ctas, st);
        case 1: return launch_rms_backward_p<T, V, 1>(A, p, parts, ctas, st);
        case 2: return launch_rms_backward_p<T, V, 2>(A, p, parts, ctas, st);
        case 3: return launch_rms_backward_p<T, V, 3>(A, p, parts, ctas, st);
        case 4: return launch_rms_backward_p<T, V, 4>(A, p, parts, ctas, st);
        default: return launch_rms_backward_p<T, V, 5>(A, p, parts, ctas, st);
    }
}
template <typename T>
static cudaError_t launch_rms_backward_t(const RmsBackwardArgs& A, int access, int64_t parts, int* ctas, cudaStream_t st) {
    if (access == 16) return launch_rms_backward_v<T, 16 / sizeof(T)>(A, parts, ctas, st);
    if (sizeof(T) == 2 && access == 4) return launch_rms_backward_v<T, 4 / sizeof(T)>(A, parts, ctas, st);
    return launch_rms_backward_v<T, 1>(A, parts, ctas, st);
}

}  // namespace dvdq
