// What the 16-bit-float and fp32 operators around the quantized layers share (linear.cuh, rope.cuh,
// group_norm.cuh): element types, vector accesses, the activations and their slopes.
#pragma once

#include <cuda_fp16.h>

#include "dvdq_common.cuh"

namespace dvdq {

// ------------------------------------------------------------------ element types

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// the one rounding of an output: to nearest, ties to even
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }

template <typename T> struct IsBf16 { static constexpr int value = 0; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr int value = 1; };

// V elements moved by one access (V * sizeof(T) = 2, 4, 8 or 16 bytes, aligned to that).
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};
template <typename T, int V>
__device__ __forceinline__ void widen(const Vec<T, V>& v, float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_f32(v.e[i]);
}
// ------------------------------------------------------------------ activations

// 1 / (1 + exp(-u)): one ex2.approx and one rcp.approx, about 1e-6 relative for |u| < 10.
__device__ __forceinline__ float logistic(float u) {
    float t, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(-1.4426950408889634f * u));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + t));
    return r;
}

// Both activations are z f(u) with f the logistic function: u = z (SiLU), or u = sqrt(8 / pi)
// (z + 0.044715 z^3) (GELU in its tanh form, since (1 + tanh(a)) / 2 = f(2a)).
constexpr float kGeluA = 1.5957691216057308f;              // sqrt(8 / pi)
constexpr float kGeluB = kGeluA * 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == DVDQ_ACT_NONE) return z;
    const float u = ACT == DVDQ_ACT_SILU ? z : z * fmaf(kGeluB, z * z, kGeluA);
    return z * logistic(u);
}
// d/dz of it: f + z u'(z) f (1 - f).  GELU's z is held at 20, where u is 600 and f 0 or 1: no overflow of z^3.  SiLU's is not: its
// u is z, the slope still 4e-8 at -20, and f (1 + z (1 - f)) has no power of z to overflow.
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == DVDQ_ACT_NONE) return 1.0f;
    if (ACT == DVDQ_ACT_SILU) {
        const float f = logistic(z);
        return fmaf(f, fmaf(-z, f, z), f);
    }
    const float c = z != z ? z : fminf(fmaxf(z, -20.0f), 20.0f);
    const float f = logistic(c * fmaf(kGeluB, c * c, kGeluA));
    return fmaf(c * fmaf(3.0f * kGeluB, c * c, kGeluA) * f, 1.0f - f, f);
}
__device__ __forceinline__ float act_value_rt(int act, float z) {
    return act == DVDQ_ACT_GELU_TANH ? act_value<DVDQ_ACT_GELU_TANH>(z) : act == DVDQ_ACT_SILU ? act_value<DVDQ_ACT_SILU>(z) : z;
}

// ------------------------------------------------------------------ the same on pairs of channels
//
// sm_100 issues add, multiply and fma on two fp32 values at a time; the streaming kernels are bound by
// issue slots long before arithmetic, so they work on pairs.  One channel (V = 1) rides with a zero beside it.
template <int V>
struct Pairs {
    static constexpr int N = (V + 1) / 2;
    uint64_t p[N];
    __device__ __forceinline__ float get(int i) const {
        float a, b;
        f2_unpack(p[i >> 1], a, b);
        return i & 1 ? b : a;
    }
    __device__ __forceinline__ void set(const float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = f2_pack(f[2 * i], 2 * i + 1 < V ? f[2 * i + 1] : 0.f);
    }
};
template <typename T, int V>
__device__ __forceinline__ Pairs<V> widen2(const Vec<T, V>& v) {
    Pairs<V> r;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 f = unpack2<T>(reinterpret_cast<const uint32_t*>(&v)[i]);
            r.p[i] = f2_pack(f.x, f.y);
        }
    } else {
        float f[V];
        widen(v, f);
        r.set(f);
    }
    return r;
}
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> narrow2(const Pairs<V>& r) {
    Vec<T, V> v;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            float a, b;
            f2_unpack(r.p[i], a, b);
            reinterpret_cast<uint32_t*>(&v)[i] = pack2<T>(a, b);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v.e[i] = from_f32<T>(r.get(i));
    }
    return v;
}
__device__ __forceinline__ uint64_t f2_splat(float v) { return f2_pack(v, v); }
// logistic(u) of a pair, given -log2(e) u.  SHARED: one reciprocal for both, 1/a = b / (ab), for kernels that the
// special-function unit (16 a clock per SM; two per value otherwise) would bound.  The exponents are then held at
// 60, so that ab stays finite, and past that logistic(u), below 2^-60, is 0: z times 2^-60 would not be small for z = -1e20.
template <bool SHARED>
__device__ __forceinline__ uint64_t logistic2_scaled(uint64_t e) {
    float a, b;
    f2_unpack(e, a, b);
    const bool a_gone = a > 60.0f, b_gone = b > 60.0f;
    if (SHARED) {  // of NaN this makes 60: it must not reach the other value (maybe another group's); its own result is NaN by z
        asm("min.f32 %0, %0, 0f42700000;" : "+f"(a));
        asm("min.f32 %0, %0, 0f42700000;" : "+f"(b));
    }
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    f2_unpack(f2_add(f2_pack(a, b), f2_splat(1.0f)), a, b);
    if (SHARED) {
        float r = a * b;
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r));
        return f2_mul(f2_splat(r), f2_pack(a_gone ? 0.0f : b, b_gone ? 0.0f : a));
    }
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2_pack(a, b);
}
constexpr float kMinusLog2e = -1.4426950408889634f;
template <int ACT, bool SHARED = false>
__device__ __forceinline__ uint64_t act_value2(uint64_t z) {
    if (ACT == DVDQ_ACT_NONE) return z;
    const uint64_t e = ACT == DVDQ_ACT_SILU ? f2_mul(z, f2_splat(kMinusLog2e))
                                            : f2_mul(z, f2_fma(f2_splat(kGeluB * kMinusLog2e), f2_mul(z, z), f2_splat(kGeluA * kMinusLog2e)));
    return f2_mul(z, logistic2_scaled<SHARED>(e));
}
// act_slope of a pair.
template <int ACT, bool SHARED = false>
__device__ __forceinline__ uint64_t act_slope2(uint64_t z) {
    if (ACT == DVDQ_ACT_SILU) {
        const uint64_t f = logistic2_scaled<SHARED>(f2_mul(z, f2_splat(kMinusLog2e)));
        return f2_fma(f, f2_sub(z, f2_mul(z, f)), f);
    }
    if (ACT == DVDQ_ACT_GELU_TANH) {
        float a, b;
        f2_unpack(z, a, b);  // NaN stays NaN
        asm("{\n\tmax.NaN.f32 %0, %0, 0fC1A00000;\n\tmin.NaN.f32 %0, %0, 0f41A00000;\n\t}" : "+f"(a));
        asm("{\n\tmax.NaN.f32 %0, %0, 0fC1A00000;\n\tmin.NaN.f32 %0, %0, 0f41A00000;\n\t}" : "+f"(b));
        const uint64_t c = f2_pack(a, b), s = f2_mul(c, c);
        const uint64_t f = logistic2_scaled<SHARED>(f2_mul(c, f2_fma(f2_splat(kGeluB * kMinusLog2e), s, f2_splat(kGeluA * kMinusLog2e))));
        const uint64_t w = f2_mul(f2_mul(c, f2_fma(f2_splat(3.0f * kGeluB), s, f2_splat(kGeluA))), f);  // c u'(c) f
        return f2_add(f, f2_sub(w, f2_mul(w, f)));
    }
    return f2_splat(1.0f);
}

// n / d for 32-bit n by a multiplication: m = ceil(2^(32 + s) / d) with 2^s >= d, n < 2^31.
struct FastDiv {
    uint32_t d, m, s;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div), m(0), s(0) {
        while ((1u << s) < div) ++s;
        const uint64_t full = (((uint64_t)1 << (32 + s)) + div - 1) / div;  // in (2^32, 2^33]: keep the low word
        m = (uint32_t)(full - ((uint64_t)1 << 32));
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(n, m) + n) >> s); }
};

// ------------------------------------------------------------------ streams

constexpr int kStreamThreads = 256;  // threads of the CTAs that stream

template <typename T, int V> struct WholePieces { static constexpr bool value = sizeof(T) * V == 16; };

// A thread's own stream of 16-byte pieces, `count` of them from STREAMS tensors side by side, through a ring
// of D slots of its own in shared memory (cp.async): D - 1 pieces per tensor are in flight while one is
// worked on, without a register each, and no barrier is needed.  With whole batches of register loads
// a warp waits for its slowest load with nothing in flight: 3.8 instead of 5 TB/s.
// A slot is refilled only when what was read from it has been delivered: the copy's address
// depends on the words read (ANDed with a zero that the compiler does not know).
template <int D, int STREAMS, typename T, int V, int THREADS = kStreamThreads, typename Use>
__device__ __forceinline__ void thread_stream(uint32_t ring, int count, const T* from0, int64_t step0, const T* from1, int64_t step1, Use use) {
    constexpr uint32_t kSlot = THREADS * 16;
    static_assert(sizeof(Vec<T, V>) == 16, "16-byte pieces");
    uint32_t zero;
    asm volatile("mov.u32 %0, %%ntid.z;" : "=r"(zero));  // the CTAs here are one-dimensional: ntid.z == 1
    zero -= 1u;
    auto fill = [&](uint32_t slot, int k, uint32_t dep) {
        if (k < count) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + slot * STREAMS * kSlot + dep), "l"(from0) : "memory");
            from0 += step0;
            if constexpr (STREAMS == 2) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (slot * STREAMS + 1) * kSlot + dep), "l"(from1) : "memory");
                from1 += step1;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < D - 1; ++k) fill((uint32_t)k, k, 0u);
    uint32_t slot = 0, behind = D - 1, dep = 0u;  // `behind`: the slot that was read last (at first: the one not yet filled)
    for (int k = 0; k < count; ++k) {
        fill(behind, k + D - 1, dep);
        asm volatile("cp.async.wait_group %0;" ::"n"(D - 1) : "memory");
        union { uint4 w; Vec<T, V> v; } in[STREAMS];
        dep = 0u;
#pragma unroll
        for (int j = 0; j < STREAMS; ++j) {
            in[j].w = lds128(ring + (slot * STREAMS + j) * kSlot);
            dep ^= in[j].w.w;
        }
        dep &= zero;
        if constexpr (STREAMS == 1) use(in[0].v);
        else use(in[0].v, in[1].v);
        behind = slot;
        slot = slot + 1 == D ? 0u : slot + 1;
    }
}
// The same sequence with plain loads, sixteen (or twice eight) in flight, for accesses narrower than 16 bytes.
template <int STREAMS, typename T, int V, typename Use>
__device__ __forceinline__ void plain_stream(int count, const T* from0, int64_t step0, const T* from1, int64_t step1, Use use) {
    constexpr int U = STREAMS == 1 ? 16 : 8;
    for (; count > 0; count -= U) {
        Vec<T, V> a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < count) {
                a[u] = *reinterpret_cast<const Vec<T, V>*>(from0);
                from0 += step0;
                if (STREAMS == 2) {
                    b[u] = *reinterpret_cast<const Vec<T, V>*>(from1);
                    from1 += step1;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < count) {
                if constexpr (STREAMS == 1) use(a[u]);
                else use(a[u], b[u]);
            }
        }
    }
}
template <int D, int STREAMS, typename T, int V, typename Use>
__device__ __forceinline__ void walk(const uint8_t* raw, int count, const T* from0, int64_t step0, const T* from1, int64_t step1, Use use) {
    if constexpr (WholePieces<T, V>::value)
        thread_stream<D, STREAMS, T, V>(smem_u32(raw) + threadIdx.x * 16, count, from0, step0, from1, step1, use);
    else
        plain_stream<STREAMS, T, V>(count, from0, step0, from1, step1, use);
}
template <typename T, int V>
__device__ __forceinline__ void store_streaming(T* p, const Vec<T, V>& v) {  // written once, not read here again: first out of L2
    if constexpr (sizeof(Vec<T, V>) == 16) __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&v));
    else *reinterpret_cast<Vec<T, V>*>(p) = v;
}
// Both passes of one thread over its pieces.  forward(): as thread_stream, and the last D pieces stay in the ring;
// backward(): from the last piece to the first, those D from where they are, the rest through the ring again.
template <int D, int STREAMS, int THREADS, typename T, int V>
struct TwoWay {
    static constexpr int kBytes = sizeof(Vec<T, V>);
    static_assert(kBytes == 4 || kBytes == 8 || kBytes == 16, "what cp.async copies");
    static constexpr uint32_t kSlot = THREADS * kBytes, kPiece = STREAMS * kSlot;
    static constexpr size_t kRingBytes = (size_t)kPiece * D;
    uint32_t ring, zero;
    int count;
    const T *at0, *at1;      // next piece to fetch
    int64_t step0, step1;
    __device__ __forceinline__ static void copy(uint32_t to, const T* from) {
        if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(kBytes) : "memory");
    }
    __device__ __forceinline__ void fill(uint32_t slot, uint32_t dep) {
        copy(ring + slot * kPiece + dep, at0);
        if constexpr (STREAMS == 2) copy(ring + slot * kPiece + kSlot + dep, at1);
    }
    __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ static void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(D - 1) : "memory"); }
    // hands the slot's pieces to use(); the value returned is zero, but known only when they have been delivered
    template <typename Use>
    __device__ __forceinline__ uint32_t take(uint32_t slot, Use& use) {
        union Piece { uint32_t w[kBytes / 4]; Vec<T, V> v; __device__ Piece() {} } in[STREAMS];
        uint32_t dep = 0u;
#pragma unroll
        for (int j = 0; j < STREAMS; ++j) {
            const uint32_t at = ring + slot * kPiece + j * kSlot;
            if constexpr (kBytes == 16) {
                const uint4 w = lds128(at);
                in[j].w[0] = w.x; in[j].w[1] = w.y; in[j].w[2] = w.z; in[j].w[3] = w.w;
            } else if constexpr (kBytes == 8) {
                const uint2 w = lds64(at);
                in[j].w[0] = w.x; in[j].w[1] = w.y;
            } else {
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(in[j].w[0]) : "r"(at));
            }
            dep ^= in[j].w[kBytes / 4 - 1];
        }
        if constexpr (STREAMS == 1) use(in[0].v);
        else use(in[0].v, in[1].v);
        return dep & zero;
    }
    __device__ __forceinline__ TwoWay(const uint8_t* raw, int n, const T* from0, int64_t s0, const T* from1, int64_t s1)
        : ring(smem_u32(raw) + threadIdx.x * kBytes), count(n), at0(from0), at1(from1), step0(s0), step1(s1) {
        asm volatile("mov.u32 %0, %%ntid.z;" : "=r"(zero));  // the CTAs here are one-dimensional: ntid.z == 1
        zero -= 1u;
#pragma unroll
        for (int k = 0; k < D - 1; ++k) next((uint32_t)k, k, 0u);
    }
    __device__ __forceinline__ void next(uint32_t slot, int k, uint32_t dep) {
        if (k < count) {
            fill(slot, dep);
            at0 += step0;
            if (STREAMS == 2) at1 += step1;
        }
        commit();
    }
    template <typename Use>
    __device__ __forceinline__ void forward(Use use) {  // the constructor has asked for the first D - 1 pieces
        uint32_t slot = 0, behind = D - 1, dep = 0u;
        for (int k = 0; k < count; ++k) {
            next(behind, k + D - 1, dep);
            wait();
            dep = take(slot, use);
            behind = slot;
            slot = slot + 1 == D ? 0u : slot + 1;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    template <typename Use>
    __device__ __forceinline__ void backward(Use use) {
        if (count == 0) return;
        // piece k is in slot k % D; at0 stands one past the last piece
        uint32_t slot = (uint32_t)((count - 1) % D);
        at0 -= (int64_t)(D + 1) * step0;  // piece count - 1 - D
        if (STREAMS == 2) at1 -= (int64_t)(D + 1) * step1;
        for (int k = count - 1; k >= 0; --k) {
            wait();
            const uint32_t dep = take(slot, use);
            if (k >= D) {
                fill(slot, dep);
                at0 -= step0;
                if (STREAMS == 2) at1 -= step1;
            }
            commit();
            slot = slot == 0 ? D - 1 : slot - 1;
        }
    }
};

// ------------------------------------------------------------------ dependent launches

// A kernel launched with launch_after may start while its predecessor on the stream drains; it
// must not touch the predecessor's results before wait_predecessor.  It releases its own successor after that wait, not before:
// released at its start, a chain of kernels piles up on the SMs, and waiting CTAs with a whole SM's shared memory keep those in
// front of them from it (gradients of 1 token, 1536 -> 1536: 25 us, 11 this way; of 4: 20 and 12.7).
__device__ __forceinline__ void wait_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release_successor() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... Par, typename... Arg>
inline cudaError_t launch_after(void (*kern)(Par...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Arg... arg) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<Par>(arg)...);
}

// ------------------------------------------------------------------ host helpers

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int dtype_bytes(int32_t dtype) { return dtype == DVDQ_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace dvdq
