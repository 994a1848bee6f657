// Rows of C values, each held by a few lanes, a warp or a CTA: what the RMS norm (rms_norm.cuh) and its gradients
// (rms_norm_backward.cuh) share.  Pieces of a row in words, a thread's share of a row, the exchange over a row's threads, the plan.
#pragma once

#include "block_common.cuh"

namespace dvdq {

constexpr int kRowThreads = 1024;    // most threads of a row
constexpr int kSmallThreads = 128;   // of a CTA whose rows take a warp or less

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

// V neighbouring values as they lie in memory, in words: elements of 16 bits as such would be packed and unpacked at every
// turn (77 instead of 15 instructions an element, and twice the time).
template <typename T, int V>
struct Piece {
    static constexpr int kBytes = V * (int)sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* p) {
        if constexpr (kBytes == 16) {
            const uint4 v = *static_cast<const uint4*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (kBytes == 4) {
            w[0] = *static_cast<const uint32_t*>(p);
        } else {
            w[0] = *static_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void load_shared(uint32_t at) {  // (a load through a generic pointer is slower)
        if constexpr (kBytes == 16) {
            const uint4 v = lds128(at);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (kBytes == 4) {
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
        } else {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
            w[0] = v;
        }
    }
    __device__ __forceinline__ void store(void* p) const {
        if constexpr (kBytes == 16) *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (kBytes == 4) *static_cast<uint32_t*>(p) = w[0];
        else *static_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void put(int j, T v) {  // into zeros
        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(v);
        else w[j >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(&v) << (16 * (j & 1));
    }
    __device__ __forceinline__ T take(int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
        const uint16_t v = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        return *reinterpret_cast<const T*>(&v);
    }
    __device__ __forceinline__ Pairs<V> wide() const {
        Pairs<V> f;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < Pairs<V>::N; ++i) f.p[i] = f2_pack(__uint_as_float(w[2 * i]), 2 * i + 1 < V ? __uint_as_float(w[2 * i + 1]) : 0.f);
        } else if constexpr (V == 1) {
            f.p[0] = f2_pack(to_f32(take(0)), 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float2 v = unpack2<T>(w[i]);
                f.p[i] = f2_pack(v.x, v.y);
            }
        }
        return f;
    }
    __device__ __forceinline__ static Piece narrow(const Pairs<V>& f) {
        Piece r;
#pragma unroll
        for (int i = 0; i < Pairs<V>::N; ++i) {
            float a, b;
            f2_unpack(f.p[i], a, b);
            if constexpr (sizeof(T) == 4) {
                r.w[2 * i] = __float_as_uint(a);
                if (2 * i + 1 < V) r.w[2 * i + 1] = __float_as_uint(b);
            } else {
                r.w[i] = pack2<T>(a, b);
            }
        }
        return r;
    }
};
// WHOLE: all V channels from c on are in the row; else those past its end are zero, and are neither read nor written.
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ Piece<T, V> row_load(const T* p, int c, int C) {
    Piece<T, V> v;
    if constexpr (WHOLE) {
        v.load(p + c);
    } else {
        v.clear();
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < C) v.put(j, p[c + j]);
    }
    return v;
}
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ void row_store(T* p, int c, int C, const Pairs<V>& f, bool there) {
    const Piece<T, V> v = Piece<T, V>::narrow(f);
    if constexpr (WHOLE) {
        if (there) v.store(p + c);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (there && c + j < C) p[c + j] = v.take(j);
    }
}
template <typename T>
__device__ __forceinline__ float gamma_at(const void* gamma, int params_f32, int c) {
    return !gamma ? 1.0f : params_f32 ? static_cast<const float*>(gamma)[c] : to_f32(static_cast<const T*>(gamma)[c]);
}
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ Pairs<V> gamma_load(const void* gamma, int params_f32, int c, int C) {  // NULL: ones
    Pairs<V> g;
    if (!gamma) {
#pragma unroll
        for (int j = 0; j < Pairs<V>::N; ++j) g.p[j] = f2_splat(1.0f);
        return g;
    }
    if (sizeof(T) == 4 || !params_f32) return row_load<T, V, WHOLE>(static_cast<const T*>(gamma), c, C).wide();
    const float* p = static_cast<const float*>(gamma) + c;
    if constexpr (WHOLE && V == 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(p + 4 * i);
            g.p[2 * i] = f2_pack(v.x, v.y);
            g.p[2 * i + 1] = f2_pack(v.z, v.w);
        }
    } else if constexpr (WHOLE && V == 2) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        g.p[0] = f2_pack(v.x, v.y);
    } else {
        float f[2 * Pairs<V>::N];
#pragma unroll
        for (int j = 0; j < 2 * Pairs<V>::N; ++j) f[j] = j < V && c + j < C ? p[j] : 0.f;
#pragma unroll
        for (int j = 0; j < Pairs<V>::N; ++j) g.p[j] = f2_pack(f[2 * j], f[2 * j + 1]);
    }
    return g;
}
template <int V>
__device__ __forceinline__ void add_to(Pairs<V>& a, const Pairs<V>& b) {
#pragma unroll
    for (int j = 0; j < Pairs<V>::N; ++j) a.p[j] = f2_add(a.p[j], b.p[j]);
}
struct Whole { static constexpr bool value = true; };
struct Part { static constexpr bool value = false; };
__device__ __forceinline__ int64_t row_at(const RowsOf& t, uint32_t n, uint32_t s) { return (int64_t)n * t.outer + (int64_t)s * t.row; }

// ------------------------------------------------------------------ what a whole row decides

// Sum of a and max of b over the threads of a row, the same bits in each of them.  WIDE: a CTA's warps meet through shared memory;
// `turn` alternates between two sets of slots, so that one barrier a row is enough.
template <bool WIDE>
struct RowMeet {
    float2* slots;   // [2][32]
    int lanes, turn = 0;
    __device__ __forceinline__ RowMeet(float2* s, int l) : slots(s), lanes(l) {}
    __device__ __forceinline__ float2 operator()(float a, float b, bool with_max) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (WIDE || o < lanes) {
                a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
                if (with_max) b = max_nan(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
            }
        }
        if constexpr (WIDE) {
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

// The pieces of a row that a thread has: P whole ones, and, where V does not divide C, one thread the row's end.  KIND: kFull (every thread has P whole
// pieces, and that is the row), kWide (a CTA's row: each warp has 32 P neighbouring pieces, so that a thread's addresses differ by constants; with
// the CTA's width between them, odd rows of 1541 took 94 us instead of 71).
enum RowKind { kRagged = 0, kFull = 1, kWide = 2 };
template <int V, int P, int KIND>
struct RowLanes {
    static constexpr bool FULL = (KIND & kFull) != 0, WIDE = (KIND & kWide) != 0;
    int C, lanes, lane, whole;  // whole pieces of the row
    int first;                  // this thread's first
    bool tail;                  // whether this thread has its end
    __device__ __forceinline__ RowLanes(int channels, int n, int l) : C(channels), lanes(n), lane(l) {
        whole = channels / V;
        first = WIDE && P > 0 ? (l >> 5) * (32 * P) + (l & 31) : l;
        tail = !FULL && V > 1 && channels % V != 0 && whole % n == l;
    }
    __device__ __forceinline__ int piece(int i) const { return first + i * (WIDE ? 32 : lanes); }
    __device__ __forceinline__ bool has(int i) const { return FULL || piece(i) < whole; }
    __device__ __forceinline__ int channel(int i) const { return piece(i) * V; }
    __device__ __forceinline__ int end() const { return whole * V; }
};
// gamma of a thread's channels: kept (KEEP), or loaded where it is needed
template <typename T, int V, int P, int KIND, bool KEEP>
struct RowGamma {
    static constexpr int K = KEEP ? P : 0;
    using Lanes = RowLanes<V, P, KIND>;
    Pairs<V> g[K + 1], end;
    const void* p;
    int f32, C;
    __device__ __forceinline__ void init(const Lanes& L, const void* gamma, int params_f32) {
        p = gamma;
        f32 = params_f32;
        C = L.C;
#pragma unroll
        for (int i = 0; i < K; ++i) {
#pragma unroll
            for (int j = 0; j < Pairs<V>::N; ++j) g[i].p[j] = 0ull;
            if (L.has(i)) g[i] = gamma_load<T, V, true>(p, f32, L.channel(i), C);
        }
        if (KEEP && L.tail) end = gamma_load<T, V, false>(p, f32, L.end(), C);
    }
    template <bool WHOLE>
    __device__ __forceinline__ Pairs<V> get(int i, int c) const {
        if constexpr (KEEP) return WHOLE ? g[i] : end;
        else return gamma_load<T, V, WHOLE>(p, f32, WHOLE && c + V > C ? 0 : c, C);  // a piece that is not there: any
    }
};

// ------------------------------------------------------------------ host side

struct RowsPlan {
    int lanes, lanes_log2, threads, pieces;  // pieces 0: the row is read again instead of kept
    bool wide, full;
};
// Pieces a thread that the kernels are built for: 1, 2, 4, 8, and where they fill the threads 3, 5, 6, 7 too.
constexpr int rows_pieces(int64_t k) { return k <= 2 ? (int)k : k <= 4 ? 4 : 8; }
// How `rows` rows of nv pieces are laid over threads that keep up to `most` pieces each (`warp_most` in rows of a warp, ragged_most where pieces do not
// fill the threads), in CTAs of up to limit(pieces) threads.  `whole`: nothing is left of the row behind its pieces; `order`: which numbers of pieces to try
// then.
template <typename Limit>
inline RowsPlan rows_plan(int64_t rows, int64_t nv, bool whole, int warp_most, int most, int ragged_most, Limit limit, const int* order) {
    RowsPlan p = {};
    const bool few = rows < 148 * 2;
    if (nv <= 64 || (nv <= 32 * warp_most && !few && rows >= 148 * 8)) {  // a warp or part of it
        p.threads = kSmallThreads;
        // lanes that have as many pieces each, two to `warp_most` (12 pieces of 96 channels: four lanes with three; eight with up to two took 55 us for
        // 32760 x 12 heads, 16 bytes of each)
        for (p.lanes_log2 = 5; whole && p.lanes_log2 >= 0; --p.lanes_log2) {
            const int64_t k = nv >> p.lanes_log2;
            if (k << p.lanes_log2 == nv && (k >= 2 || nv == 1) && k <= (warp_most < 5 ? 5 : warp_most)) {
                p.lanes = 1 << p.lanes_log2;
                p.pieces = (int)k;
                p.full = true;
                return p;
            }
        }
        p.lanes_log2 = 5;
        while (p.lanes_log2 > 0 && nv <= 1 << p.lanes_log2) --p.lanes_log2;  // two pieces a thread, where there are two
        p.lanes = 1 << p.lanes_log2;
        p.pieces = rows_pieces(ceil_div(nv, p.lanes));
        return p;
    }
    p.wide = true;
    // a CTA whose threads all have as many pieces (few rows: as few as there can be; many: up to 256 threads if possible, so that the CTAs of an SM wait for
    // their barriers by turns: 10000 rows of 16384 202 us in 256 threads, 217 in 512)
    static const int up[] = {1, 2, 3, 4, 5, 6, 7, 8, 0};
    for (int cap = few ? kRowThreads : 256; whole && cap <= kRowThreads; cap *= 4)
        for (const int* k = few ? up : order; *k; ++k)
            if (*k <= most && nv % (32 * *k) == 0 && nv / *k >= 64 && nv / *k <= cap && nv / *k <= limit(*k)) {
                p.pieces = *k;
                p.lanes = p.threads = (int)(nv / *k);
                p.full = true;
                return p;
            }
    // otherwise as many as leave two warps
    for (int k = few ? 1 : ragged_most; k >= 1 && k <= ragged_most; k = few ? k * 2 : k / 2) {
        const int64_t threads = align_up(ceil_div(nv, k), 32);
        if (threads > limit(k) || (!few && threads < 64 && k > 1)) continue;
        p.pieces = k;
        p.lanes = p.threads = (int)(threads < 64 ? 64 : threads);
        return p;
    }
    p.lanes = p.threads = kRowThreads;
    return p;
}
// CTAs of a kernel that an SM holds, for each number of warps (asked once).
struct RowsHeld {
    int held[kRowThreads / 32 + 1];
};
template <typename Kern>
static int rows_held(PerDevice<RowsHeld>& cache, Kern kern, int threads) {
    RowsHeld* h = cache.get([&](RowsHeld& all, int) {
        cudaFuncAttributes a;
        if (cudaFuncGetAttributes(&a, kern) != cudaSuccess) return false;
        for (int w = 1; w <= kRowThreads / 32; ++w) {
            all.held[w] = 1;
            if (w * 32 <= a.maxThreadsPerBlock && cudaOccupancyMaxActiveBlocksPerMultiprocessor(&all.held[w], kern, w * 32, 0) != cudaSuccess) return false;
        }
        return true;
    });
    return h ? (h->held[threads / 32] < 1 ? 1 : h->held[threads / 32]) : 0;
}

// The widest piece, in bytes of the tensors' type, that all of them and gamma allow.
inline bool piece_ok(const RowsOf& t, int bytes, int piece) {
    return aligned_to(t.p, piece) && (t.outer * bytes) % piece == 0 && (t.row * bytes) % piece == 0;
}
inline int rows_access(const RowsOf* const* tensors, int count, const RowsOf* codes, const void* gamma, int bytes, int param_bytes) {
    for (int piece = 16; piece > bytes; piece /= 4) {
        const int v = piece / bytes, of_gamma = v * param_bytes < 16 ? v * param_bytes : 16;
        bool ok = !gamma || aligned_to(gamma, of_gamma);
        for (int i = 0; i < count; ++i) ok = ok && (!tensors[i]->p || piece_ok(*tensors[i], bytes, piece));
        if (ok && (!codes || !codes->p || piece_ok(*codes, 1, v))) return piece;
    }
    return bytes;
}
inline RowsShape rows_shape(int64_t N, int64_t S, int64_t C) {
    RowsShape r;
    r.rows = N * S;
    r.by_s = FastDiv((uint32_t)S);
    r.S = (int)S;
    r.C = (int)C;
    return r;
}

// ------------------------------------------------------------------ checks of arguments

inline bool rows_dtype_ok(int32_t t) { return t == DVDQ_BF16 || t == DVDQ_F16 || t == DVDQ_F32; }
inline bool rows_sizes_ok(int64_t N, int64_t S, int64_t C) {
    const int64_t most = 0x7FFFFFFFll;
    return N >= 0 && S >= 0 && N <= most && S <= most && N * S <= most && C > 0 && C <= (1 << 20);
}
// Whether rows of C elements that start at n * outer + s * row lie over one another (both pitches C or more).
inline bool rows_collide(int64_t N, int64_t S, int64_t C, int64_t outer, int64_t row) {
    if (N <= 1 || S <= 1) return false;
    const bool rows_inside = row <= outer;
    const int64_t inner = rows_inside ? row : outer, wide = rows_inside ? outer : row, steps = (rows_inside ? S : N) - 1;
    if (inner > ((int64_t)1 << 61) / steps) return false;  // no memory holds such rows
    const int64_t last = steps * inner;
    for (int64_t k = 1, at = wide; k < (rows_inside ? N : S) && at < last + C; ++k, at += wide) {  // at most the smaller extent's number of turns
        const int64_t below = at - at / inner * inner;
        if (at > last || below < C || inner - below < C) return true;
    }
    return false;
}
// An [N, S, C] tensor's pitches; those of an extent of one are not read.
inline dvdq_status check_rows(RowsOf* t, int64_t N, int64_t S, int64_t C, int bytes, bool written) {
    if (!t->p) return DVDQ_OK;
    if (N == 1) t->outer = 0;
    if (S == 1) t->row = 0;
    if (t->outer < 0 || t->row < 0) return DVDQ_ERR_SHAPE;
    if (written && ((S > 1 && t->row < C) || (N > 1 && t->outer < C) || rows_collide(N, S, C, t->outer, t->row))) return DVDQ_ERR_SHAPE;  // a row over another
    return aligned_to(t->p, bytes) ? DVDQ_OK : DVDQ_ERR_ALIGN;
}
// An output over the tensor that it is made from lies exactly over it (after check_rows).
inline bool in_place_ok(const RowsOf& from, const RowsOf& to) { return !to.p || from.p != to.p || (from.outer == to.outer && from.row == to.row); }

}  // namespace dvdq
