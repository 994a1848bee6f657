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
// kRopeHeads heads of the token, all their loads in flight at once.
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
    int64_t token0;       // first token (over batches) of this launch
    int tokens, S;        // tokens of this launch; tokens of a sequence
    int rot, head_dim;
    int groups;           // ceil((q.heads + k.heads) / heads per thread)
    int items, rot_items; // accesses per head: those that rotate, then those that pass through
    int inverse;
};

// W elements per access; a rotating item covers W pairs of a "halves" head (two accesses) or W / 2
// pairs of a "pairs" head (one access; two single elements for W = 1).
template <typename T, bool HALVES, int W, int HEADS>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs A) {
    constexpr int P = HALVES ? W : (W > 1 ? W / 2 : 1);
    const uint32_t per_token = (uint32_t)A.groups * (uint32_t)A.items;
    const uint32_t idx = blockIdx.x * (uint32_t)kRopeThreads + threadIdx.x;
    const uint32_t lt = idx / per_token;
    if (lt >= (uint32_t)A.tokens) return;
    const uint32_t rem = idx - lt * per_token;
    const int grp = (int)(rem / (uint32_t)A.items), item = (int)(rem - (uint32_t)grp * (uint32_t)A.items);
    const int64_t token = A.token0 + lt;
    const int64_t b = A.S == 1 ? token : token / A.S;
    const int64_t s = token - b * A.S;
    const int heads = A.q.heads + A.k.heads;

    const bool turns = item < A.rot_items;
    const int c0 = turns ? item * (HALVES ? P : 2 * P) : A.rot + (item - A.rot_items) * W;  // first channel
    const int c1 = HALVES ? c0 + A.rot / 2 : c0 + W;                                          // the second access's

    const T* src[HEADS];
    T* dst[HEADS];
    Vec<T, W> lo[HEADS], hi[HEADS];
    const bool two = turns && (HALVES || W == 1);
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        const int h = grp + j * A.groups;
        src[j] = nullptr;
        if (h < heads) {
            const bool is_q = h < A.q.heads;
            const RopeSide& side = is_q ? A.q : A.k;
            const int hh = is_q ? h : h - A.q.heads;
            src[j] = static_cast<const T*>(side.x) + b * side.xb + s * side.xs + hh * side.xh;
            dst[j] = static_cast<T*>(side.y) + b * side.yb + s * side.ys + hh * side.yh;
            if (!turns && src[j] == dst[j]) src[j] = nullptr;  // in place: what passes through is there already
        }
        if (src[j]) {
            lo[j] = *reinterpret_cast<const Vec<T, W>*>(src[j] + c0);
            if (two) hi[j] = *reinterpret_cast<const Vec<T, W>*>(src[j] + c1);
        }
    }
    if (!turns) {
#pragma unroll
        for (int j = 0; j < HEADS; ++j)
            if (src[j]) *reinterpret_cast<Vec<T, W>*>(dst[j] + c0) = lo[j];
        return;
    }
    float cs[P], sn[P];
    {
        const int64_t row = A.rows ? (int64_t)A.rows[b * A.rows_batch + s] : s;
        if (row >= 0 && row < A.table_rows) {
            const float2* t = A.table + row * (A.rot / 2) + (HALVES ? c0 : c0 / 2);
            if constexpr (P >= 2) {
#pragma unroll
                for (int p = 0; p < P; p += 2) {
                    const float4 v = __ldg(reinterpret_cast<const float4*>(t + p));
                    cs[p] = v.x; sn[p] = v.y; cs[p + 1] = v.z; sn[p + 1] = v.w;
                }
            } else {
                const float2 v = __ldg(t);
                cs[0] = v.x; sn[0] = v.y;
            }
        } else {  // a row outside the table: the outputs say so, and so does the device status
            if (item == 0 && grp == 0 && atomicCAS(&g_device_status[0], 0u, (uint32_t)DVDQ_ERR_SHAPE) == 0u)
                g_device_status[1] = kDetailRopeRow;
#pragma unroll
            for (int p = 0; p < P; ++p) cs[p] = sn[p] = __int_as_float(0x7FC00000);
        }
        if (A.inverse) {
#pragma unroll
            for (int p = 0; p < P; ++p) sn[p] = -sn[p];
        }
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        if (!src[j]) continue;
        if constexpr (HALVES || W == 1) {
            float a[W], bb[W], ya[W], yb[W];
            widen(lo[j], a);
            widen(hi[j], bb);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                ya[p] = fmaf(a[p], cs[p], -(bb[p] * sn[p]));
                yb[p] = fmaf(bb[p], cs[p], a[p] * sn[p]);
            }
            *reinterpret_cast<Vec<T, W>*>(dst[j] + c0) = narrow<T, W>(ya);
            *reinterpret_cast<Vec<T, W>*>(dst[j] + c1) = narrow<T, W>(yb);
        } else {
            float a[W], y[W];
            widen(lo[j], a);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                y[2 * p] = fmaf(a[2 * p], cs[p], -(a[2 * p + 1] * sn[p]));
                y[2 * p + 1] = fmaf(a[2 * p + 1], cs[p], a[2 * p] * sn[p]);
            }
            *reinterpret_cast<Vec<T, W>*>(dst[j] + c0) = narrow<T, W>(y);
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

template <typename T, bool HALVES, int W>
static cudaError_t launch_rope_w(RopeArgs A, int64_t tokens, cudaStream_t st) {
    constexpr int P = HALVES ? W : (W > 1 ? W / 2 : 1);
    const int heads = A.q.heads + A.k.heads;
    A.rot_items = A.rot / 2 / P;
    A.items = A.rot_items + (A.head_dim - A.rot) / W;
    // Few tokens: one head per thread, the shortest chain.  Many: four, which share the table's values
    // and keep four loads (eight in halves) in flight.
    const bool many = tokens * heads * A.items >= (int64_t)148 * 2048 * 2;
    A.groups = many ? (heads + 3) / 4 : heads;
    const int64_t per_token = (int64_t)A.groups * A.items;
    const int64_t most = (((int64_t)1 << 31) - kRopeThreads) / per_token;  // the thread index is 32 bits wide
    for (int64_t t = 0; t < tokens; t += most) {
        A.token0 = t;
        A.tokens = (int)(tokens - t < most ? tokens - t : most);
        const unsigned grid = (unsigned)ceil_div((int64_t)A.tokens * per_token, kRopeThreads);
        if (many) rope_kernel<T, HALVES, W, 4><<<grid, kRopeThreads, 0, st>>>(A);
        else rope_kernel<T, HALVES, W, 1><<<grid, kRopeThreads, 0, st>>>(A);
    }
    return cudaGetLastError();
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
