// Rotary positions: the pair (a, b) of a head at position p turns by the angle p * freq_i,
//
//   (a, b) -> (a cos - b sin, b cos + a sin),       inverse (the gradient): the same with -sin,
//
// with (a, b) = (x_2i, x_2i+1) ("pairs") or (x_i, x_{i + rot/2}) ("halves"), over the first rot
// channels of a head; the rest of the head passes through.
//
// What bounds it: reading and writing q and k once (the table's row of a token, 4 * rot bytes, is
// shared by all heads).  So the angles' cosines and sines come from a table that is made once
// (rope_table_kernel, in fp64: at position 10^5 an fp32 angle is off by 0.004), q and k go in one
// launch, and a thread keeps the table's values of its channels in registers while it walks over
// up to four heads of the token, all their loads in flight at once.
#pragma once

#include "block_common.cuh"

namespace dvdq {

constexpr int kRopeMaxPairs = 256;
constexpr int kRopeThreads = 256;

struct RopeAngles {
    double freq[kRopeMaxPairs];
    uint8_t axis[kRopeMaxPairs];
};

// table[t][i] = amplitude * (cos, sin)(positions[t][axis_i] * freq_i); positions NULL: t itself.
__global__ void __launch_bounds__(kRopeThreads)
rope_table_kernel(const __grid_constant__ RopeAngles ang, const int32_t* __restrict__ positions, int64_t total, int pairs, int axes,
                  double amplitude, float2* __restrict__ table) {
    for (int64_t i = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kRopeThreads) {
        const int64_t t = i / pairs;
        const int p = (int)(i - t * pairs);
        const double pos = positions ? (double)positions[t * axes + ang.axis[p]] : (double)t;
        double s, c;
        sincos(pos * ang.freq[p], &s, &c);
        table[i] = make_float2((float)(amplitude * c), (float)(amplitude * s));
    }
}

struct RopeSide {
    const void* x;
    void* y;
    int heads;
    int64_t xb, xs, xh, yb, ys, yh;
};

struct RopeArgs {
    RopeSide q, k;
    const float2* table;
    const int32_t* rows;
    int64_t rows_batch, table_rows;
    int64_t token0;        // first token (over batches) of this launch
    uint32_t threads;      // of this launch: tokens * groups * items
    int64_t S;             // tokens of a sequence
    int rot, head_dim;
    int q_groups;          // groups of heads, q's first; a group belongs to one of the two
    FastDiv per_token, items, seq;
    int rot_items;         // accesses per head: those that rotate, then those that pass through
    int inverse, small;    // small: token indices fit 31 bits
};

// W elements per access; a rotating item covers W pairs of a "halves" head (two accesses) or W / 2
// pairs of a "pairs" head (one access; two single elements for W = 1).
template <typename T, bool HALVES, int W, int HEADS>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs A) {
    constexpr int P = HALVES ? W : (W > 1 ? W / 2 : 1);
    constexpr bool TWO = HALVES || W == 1;  // a rotating item is two accesses
    wait_predecessor();
    release_successor();
    const uint32_t idx = blockIdx.x * (uint32_t)kRopeThreads + threadIdx.x;
    if (idx >= A.threads) return;
    const uint32_t lt = A.per_token(idx), rem = idx - lt * A.per_token.d;
    int grp = (int)A.items(rem);
    const int item = (int)(rem - (uint32_t)grp * A.items.d);
    const int64_t token = A.token0 + lt;
    const int64_t b = A.small ? (int64_t)A.seq((uint32_t)token) : token / A.S;
    const int64_t s = token - b * A.S;

    const bool turns = item < A.rot_items;
    const int c0 = turns ? item * (HALVES ? P : 2 * P) : A.rot + (item - A.rot_items) * W;  // first channel
    const int c1 = HALVES ? A.rot / 2 : W;                                                    // on to the second access's
    float2 cs[P];
    bool inside = true;
    if (turns) {
        const int64_t row = A.rows ? (int64_t)A.rows[b * A.rows_batch + s] : s;
        inside = row >= 0 && row < A.table_rows;
        const float2* t = A.table + (inside ? row : 0) * (A.rot / 2) + (HALVES ? c0 : c0 / 2);
        if constexpr (P >= 2) {
#pragma unroll
            for (int p = 0; p < P; p += 2) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(t + p));
                cs[p] = make_float2(v.x, v.y);
                cs[p + 1] = make_float2(v.z, v.w);
            }
        } else {
            cs[0] = __ldg(t);
        }
    }
    const bool is_q = grp < A.q_groups;
    if (!is_q) grp -= A.q_groups;
    const RopeSide& side = is_q ? A.q : A.k;
    const int h0 = grp * HEADS, left = side.heads - h0;  // this thread's heads: h0 .. h0 + min(HEADS, left)
    const T* src = static_cast<const T*>(side.x) + b * side.xb + s * side.xs + h0 * side.xh + c0;
    T* dst = static_cast<T*>(side.y) + b * side.yb + s * side.ys + h0 * side.yh + c0;
    if (!turns && src == dst) return;  // in place: what passes through is there already
    Vec<T, W> lo[HEADS], hi[HEADS];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        if (j < left) {
            lo[j] = *reinterpret_cast<const Vec<T, W>*>(src);
            if (TWO && turns) hi[j] = *reinterpret_cast<const Vec<T, W>*>(src + c1);
            src += side.xh;
        }
    }
    if (!turns) {
#pragma unroll
        for (int j = 0; j < HEADS; ++j) {
            if (j < left) *reinterpret_cast<Vec<T, W>*>(dst) = lo[j];
            dst += side.yh;
        }
        return;
    }
    if (!inside) {  // a row outside the table: the outputs say so, and so does the device status
        if (item == 0 && atomicCAS(&g_device_status[0], 0u, (uint32_t)DVDQ_ERR_SHAPE) == 0u) g_device_status[1] = kDetailRopeRow;
#pragma unroll
        for (int p = 0; p < P; ++p) cs[p] = make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));
    }
    if (A.inverse) {
#pragma unroll
        for (int p = 0; p < P; ++p) cs[p].y = -cs[p].y;
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        if (j < left) {
            if constexpr (TWO) {  // fp32 pairs: neighbouring channels of one half
                const Pairs<W> a = widen2<T, W>(lo[j]), bb = widen2<T, W>(hi[j]);
                Pairs<W> ya, yb;
#pragma unroll
                for (int i = 0; i < Pairs<W>::N; ++i) {
                    const int p1 = 2 * i + 1 < P ? 2 * i + 1 : 2 * i;
                    const uint64_t c = f2_pack(cs[2 * i].x, cs[p1].x), sn = f2_pack(cs[2 * i].y, cs[p1].y);
                    const uint64_t ns = f2_pack(-cs[2 * i].y, -cs[p1].y);
                    ya.p[i] = f2_fma(a.p[i], c, f2_mul(bb.p[i], ns));
                    yb.p[i] = f2_fma(bb.p[i], c, f2_mul(a.p[i], sn));
                }
                *reinterpret_cast<Vec<T, W>*>(dst) = narrow2<T, W>(ya);
                *reinterpret_cast<Vec<T, W>*>(dst + c1) = narrow2<T, W>(yb);
            } else {              // fp32 pairs: (a, b) of one rotation
                const Pairs<W> x = widen2<T, W>(lo[j]);
                Pairs<W> y;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    float a, bb;
                    f2_unpack(x.p[p], a, bb);
                    y.p[p] = f2_fma(x.p[p], f2_pack(cs[p].x, cs[p].x), f2_mul(f2_pack(bb, a), f2_pack(-cs[p].y, cs[p].y)));
                }
                *reinterpret_cast<Vec<T, W>*>(dst) = narrow2<T, W>(y);
            }
            dst += side.yh;
        }
    }
}

// ------------------------------------------------------------------ host side

// The widest access that every head's first channel, the halves' split, the rotated part and the rest allow.
inline int rope_access(const RopeSide* side, int sides, int D, int rot, bool halves, int bytes) {
    for (int w = 16 / bytes; w > 1; w /= 2) {
        bool ok = (halves ? rot / 2 : rot) % w == 0 && (D - rot) % w == 0;
        for (int i = 0; i < sides; ++i) {
            const RopeSide& s = side[i];
            ok = ok && aligned_to(s.x, (uintptr_t)w * bytes) && aligned_to(s.y, (uintptr_t)w * bytes);
            for (int64_t st : {s.xb, s.xs, s.xh, s.yb, s.ys, s.yh}) ok = ok && st % w == 0;
        }
        if (ok) return w;
    }
    return 1;
}

template <typename T, bool HALVES, int W, int HEADS>
static cudaError_t launch_rope_heads(RopeArgs A, int64_t tokens, int items, cudaStream_t st) {
    A.q_groups = (A.q.heads + HEADS - 1) / HEADS;
    const int groups = A.q_groups + (A.k.heads + HEADS - 1) / HEADS;
    const int64_t per_token = (int64_t)groups * items;
    A.per_token = FastDiv((uint32_t)per_token);
    A.items = FastDiv((uint32_t)items);
    A.small = tokens < ((int64_t)1 << 31);
    A.seq = FastDiv((uint32_t)A.S);
    const int64_t most = (((int64_t)1 << 31) - kRopeThreads) / per_token;  // a launch's thread index fits 31 bits
    for (int64_t t = 0; t < tokens; t += most) {
        A.token0 = t;
        A.threads = (uint32_t)((tokens - t < most ? tokens - t : most) * per_token);
        const cudaError_t e = launch_after(rope_kernel<T, HALVES, W, HEADS>, dim3((unsigned)ceil_div(A.threads, kRopeThreads)), dim3(kRopeThreads), 0, st, A);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, bool HALVES, int W>
static cudaError_t launch_rope_w(RopeArgs A, int64_t tokens, cudaStream_t st) {
    constexpr int P = HALVES ? W : (W > 1 ? W / 2 : 1);
    A.rot_items = A.rot / 2 / P;
    const int items = A.rot_items + (A.head_dim - A.rot) / W;
    // Few tokens: one head per thread, the shortest chain.  Many: four, which share the table's values
    // and keep four loads (eight in halves) in flight.  24 heads of 128 channels, one and four heads per thread: 100 tokens 1.6
    // and 1.8 us, 400 2.8 and 2.5, 1600 5.3 and 3.9, 32760 81 and 63 (6.4 TB/s); 32 heads of 96, halves, 65536: 148 and 121 (6.7 TB/s).
    const bool many = tokens * (A.q.heads + A.k.heads) * items >= (int64_t)148 * 1024;
    return many ? launch_rope_heads<T, HALVES, W, 4>(A, tokens, items, st) : launch_rope_heads<T, HALVES, W, 1>(A, tokens, items, st);
}

template <typename T, bool HALVES>
static cudaError_t launch_rope_t(const RopeArgs& A, int w, int64_t tokens, cudaStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (w == 8) return launch_rope_w<T, HALVES, 8>(A, tokens, st);
    }
    if (w == 4) return launch_rope_w<T, HALVES, 4>(A, tokens, st);
    if (w == 2) return launch_rope_w<T, HALVES, 2>(A, tokens, st);
    return launch_rope_w<T, HALVES, 1>(A, tokens, st);
}

}  // namespace dvdq
