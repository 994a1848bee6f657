// Rows of C values: RMS norm with the residual's addition, its output in the rows' type or in 8 bits with a scale for each
// row; and the 8-bit quantization alone (NORM = false).
//
//   h = x + r,  q = 1 / sqrt(mean h^2 + eps),  y = h q gamma,  s = max|y| / 127,  c = round(y / s)
//
// Everything between the loads and the one rounding of each output is fp32; y and c come from the unrounded h.  Both things that the
// whole row decides, sum of h^2 and max |h gamma| (max |y| is q times that), meet in one exchange.
//
// What bounds it: memory, each input read once and each output written once.  So a row is held in registers from its loads to its stores (P pieces
// of V channels a thread, 16 bytes where the tensors' alignment allows), by a few lanes, a warp or a CTA, whichever gives a thread several pieces:
// what a row costs beside its pieces (addresses, exchange, root, division) is paid by each of its threads.  CTAs go from row to row and their threads keep
// their channels, so that gamma stays in registers.  Instructions, not latency, were the next bound at each step: elements of 16 bits kept in
// words, no branch in the inner loops (kernels for what is asked for, for rows that fill the threads), addresses that differ by constants (32760 x 5120 with
// residual and codes: 538, 250, 189, 182, and 179 us since rows that are far from one have a loop of their own).  Rows beyond a CTA's registers (P = 0) are read again from L2.
// Measured: 32760 x 5120 bf16, residual, codes 179 us (1174 MB, 6.6 TB/s); residual, y 208 us; rows of 8960 in 8 bits 133 us (6.6 TB/s); 32760 x 12 heads of
// 128 in a fused projection 34.3 us (5.8 TB/s); 20000 x 1541 (odd: single elements) with residual, y 75 us (3.3 TB/s); 30000 x 2049 fp32 173 us (5.7 TB/s).
#pragma once

#include "rms_rows.cuh"

namespace dvdq {

struct RmsArgs {
    RowsShape shape;
    RowsOf x, r, h, y, codes;
    const void* gamma;
    float *scales, *rstd;  // dense [N, S]
    int params_f32;
    float eps, inv_c;
    int lanes, lanes_log2; // threads of a row: a power of two up to 32, or the CTA's
};
// What a row's unit has found: y = (f h) q gamma, top = max |y|.
struct RowScale {
    float q, f, top;
};

// 2^-e for the power of two 2^e at or below v > 0, at most 2^126: brings v to [1, 2).
__device__ __forceinline__ float bring_to_one(float v) {
    const int e = (int)(__float_as_uint(v) >> 23) - 127;  // -127 below the normal numbers
    return __uint_as_float((uint32_t)(127 - (e < -126 ? -126 : e > 126 ? 126 : e)) << 23);
}

// A row in registers (P > 0), or loaded from memory at each visit (P = 0).
template <typename T, int V, int P, int KIND>
struct RowValues {
    static constexpr int K = P > 0 ? P : 1;
    using Lanes = RowLanes<V, P, KIND>;
    Pairs<V> v[K], end;
    const T *x, *r;
    template <bool WHOLE>
    __device__ __forceinline__ Pairs<V> get(int c, int C) const {
        Pairs<V> h = row_load<T, V, WHOLE>(x, c, C).wide();
        if (r) add_to<V>(h, row_load<T, V, WHOLE>(r, c, C).wide());
        return h;
    }
    // f(piece, channel, values, Whole or Part, whether the piece is there: its values are zero otherwise)
    template <typename F>
    __device__ __forceinline__ void visit(const Lanes& L, F f) {
        if constexpr (P > 0) {
#pragma unroll
            for (int i = 0; i < P; ++i) f(i, L.channel(i), v[i], Whole(), L.has(i));
            if (!Lanes::FULL && V > 1 && L.tail) f(P, L.end(), end, Part(), true);
        } else {
#pragma unroll 4
            for (int p = L.lane; p < L.whole; p += L.lanes) f(0, p * V, get<true>(p * V, L.C), Whole(), true);
            if (V > 1 && L.tail) f(0, L.end(), get<false>(L.end(), L.C), Part(), true);
        }
    }
};
// U rows' loads, all of them before the first is used.
template <typename T, int V, int P, int KIND, int U>
__device__ __forceinline__ void rows_load(const RowLanes<V, P, KIND>& L, RowValues<T, V, P, KIND> (&rows)[U], const bool (&active)[U], bool both) {
    if constexpr (P > 0) {
        Piece<T, V> a[U][P], b[U][P];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                a[u][i].clear();
                if (active[u] && L.has(i)) a[u][i].load(rows[u].x + L.channel(i));
            }
        if (both) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    b[u][i].clear();
                    if (active[u] && L.has(i)) b[u][i].load(rows[u].r + L.channel(i));
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!L.FULL && V > 1 && L.tail) rows[u].end = rows[u].template get<false>(L.end(), active[u] ? L.C : 0);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                rows[u].v[i] = a[u][i].wide();
                if (both) add_to<V>(rows[u].v[i], b[u][i].wide());
            }
        }
    }
}

// What turns a row's values into codes, c = round_half_even(v / (top / 127)).
//
// Plain rows are multiplied by `inv`, 127 / top rounded up.  Of a row in 16 bits no value lies within 2^-19 of a border without lying on it (254 v and (2 n + 1) top
// are multiples of one number), and on it, 254 v = (2 n + 1) top, only if it is half of the largest value, n = 63, or if top is a multiple of 127.  Half of the largest
// value then lies above 63.5 steps or on them and has the even code, 64 (with 127 / top rounded to nearest it had 63 in half of all rows); rows whose top / 127 is
// exact, but not 127 / top, are divided, as are rows far from one or near the smallest numbers.  (All rows by a corrected reciprocal: 32760 x 8960 142 us, 134 this way.)
struct RowCodes {
    float scale, inv;   // as written; the factor of plain rows
    bool plain;
    __device__ __forceinline__ RowCodes(const RowScale& o) : inv(0.f), plain(false) {
        const float top = o.top;
        scale = __uint_as_float(0x7FC00000u);
        if (top <= 3.4028235e38f) scale = top / 127.0f;  // not NaN, not infinite
        plain = o.f == 1.0f && top == 0.f;               // zeros
        if (!(o.f == 1.0f && top >= kLiftBelow && top <= 3.4028235e38f)) return;
        plain = fmaf(scale, -127.0f, top) != 0.f || (__float_as_uint(scale) & 0x7FFFFFu) == 0u;
        inv = 127.0f / top;
        if (fmaf(inv, top, -127.0f) < 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1u);
    }
    static constexpr float kLiftBelow = 1e-27f;
};
// Quotients of values by top / 127 rounded down, so that half of the largest value has code 64 here too; those of a division in fp32: from the reciprocal, corrected once
// by the remainder (Markstein 1990; for the mantissa of every divisor and the values around each of its borders the codes were compared with the division's).  Zeros where
// the row has no scale.  Values near the smallest numbers are lifted first, so that the reciprocal stays finite and remainders have all their digits.  A scale below
// 2^-126 has few digits itself and is what is divided by, so that its codes count it as it is written; quotients by it may pass 127, where codes end.
struct RowDivide {
    float lift, step, recip;
    __device__ __forceinline__ RowDivide(float top) : lift(0.f), step(1.f), recip(0.f) {
        const float scale = top <= 3.4028235e38f ? top / 127.0f : 0.f;
        if (scale == 0.f) return;
        lift = top < RowCodes::kLiftBelow ? 18446744073709551616.0f : 1.0f;
        step = scale * lift;
        if (scale >= 1.17549435e-38f && fmaf(step, 127.0f, -top * lift) > 0.f) step = __uint_as_float(__float_as_uint(step) - 1u);
        recip = 1.0f / step;
    }
    __device__ __forceinline__ uint64_t operator()(uint64_t v) const {
        if (lift == 0.f) return 0ull;
        const uint64_t y = f2_mul(v, f2_splat(lift)), q = f2_mul(y, f2_splat(recip));
        float a, b;
        f2_unpack(f2_fma(f2_fma(q, f2_splat(-step), y), f2_splat(recip), q), a, b);
        return f2_pack(fminf(fmaxf(a, -127.f), 127.f), fminf(fmaxf(b, -127.f), 127.f));
    }
};

// Codes of V channels: y * inv (inv = 1: y is a quotient), rounded to a whole number in the one rounding of its addition to 1.5 * 2^23, whose last byte
// then is the code.  |y| inv is at most 127 (1 + 2^-22).
template <int V, bool WHOLE>
__device__ __forceinline__ void codes_store(int8_t* p, int c, int C, const Pairs<V>& y, float inv, bool there) {
    constexpr int N = Pairs<V>::N;
    uint32_t w[2 * N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float a, b;
        f2_unpack(f2_fma(y.p[j], f2_splat(inv), f2_splat(12582912.0f)), a, b);
        w[2 * j] = __float_as_uint(a);
        w[2 * j + 1] = __float_as_uint(b);
    }
    if constexpr (WHOLE && V == 8) {
        uint2 o;
        o.x = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
        o.y = __byte_perm(__byte_perm(w[4], w[5], 0x0040), __byte_perm(w[6], w[7], 0x0040), 0x5410);
        if (there) *reinterpret_cast<uint2*>(p + c) = o;
    } else if constexpr (WHOLE && V == 4) {
        const uint32_t o = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
        if (there) *reinterpret_cast<uint32_t*>(p + c) = o;
    } else if constexpr (WHOLE && V == 2) {
        if (there) *reinterpret_cast<uint16_t*>(p + c) = (uint16_t)__byte_perm(w[0], w[1], 0x0040);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (there && c + j < C) p[c + j] = (int8_t)(w[j] & 0xFFu);
    }
}

// 1 / sqrt(m) for 1e-30 < m < 1e30, to two units of the last place
__device__ __forceinline__ float root(float m) {
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(m));
    return r;
}

// Squares that left fp32's range, or an h gamma that did: the row once more, from memory, with f h, f a power of two that brings the largest
// |h| (or sqrt(eps), where that is larger) to 1, and with y formed as it is written.  `top`: max |h gamma| as row_decide found it; `far`: whether this row needs it.
template <bool WIDE, typename T, int V, int P, int KIND>
__device__ __forceinline__ RowScale row_far(const RmsArgs& A, const RowLanes<V, P, KIND>& L, RowValues<T, V, P, KIND>& row, RowMeet<WIDE>& meet, float top, bool far) {
    float largest = 0.f;
    row.visit(L, [&](int, int, const Pairs<V>& h, auto, bool) {
#pragma unroll
        for (int j = 0; j < Pairs<V>::N; ++j) largest = max_abs2(largest, h.p[j]);
    });
    largest = meet(0.f, largest, true).y;
    RowScale o{1.0f / sqrtf(A.eps), 1.0f, top};  // a row of zeros
    const bool zeros = largest == 0.f && A.eps > 0.f;
    if (WIDE ? zeros : __all_sync(0xFFFFFFFFu, zeros || !far)) return o;
    largest = fmaxf(largest, sqrtf(A.eps));
    o.f = largest <= 3.4028235e38f && largest > 0.f ? bring_to_one(largest) : 1.0f;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {  // sum of squares; largest |y|
        float a = 0.f;
#pragma unroll 1
        for (int c = L.lane; c < L.C; c += L.lanes) {
            float h = to_f32(row.x[c]);
            if (row.r) h += to_f32(row.r[c]);
            h *= o.f;
            if (turn == 0) a = fmaf(h, h, a);
            else a = max_nan(a, fabsf(h * o.q * gamma_at<T>(A.gamma, A.params_f32, c)));
        }
        const float2 all = meet(a, a, turn == 1);
        if (turn == 0) o.q = 1.0f / sqrtf(fmaf(all.x, A.inv_c, A.eps * o.f * o.f));
        else o.top = all.y;
    }
    return o;
}

// The row's q and top.  CODES: whether the output in 8 bits is asked for.
template <bool NORM, bool WIDE, typename T, int V, int P, int KIND, bool KEEP>
__device__ __forceinline__ RowScale row_decide(const RmsArgs& A, const RowLanes<V, P, KIND>& L, RowValues<T, V, P, KIND>& row,
                                               const RowGamma<T, V, P, KIND, KEEP>& gamma, RowMeet<WIDE>& meet, bool codes) {
    constexpr int N = Pairs<V>::N;
    uint64_t sum = 0ull;
    float top = 0.f;
    row.visit(L, [&](int i, int c, const Pairs<V>& h, auto whole, bool) {
        if (NORM) {
#pragma unroll
            for (int j = 0; j < N; ++j) sum = f2_fma(h.p[j], h.p[j], sum);
        }
        if (codes) {
            const Pairs<V> g = NORM ? gamma.template get<decltype(whole)::value>(i, c) : h;
#pragma unroll
            for (int j = 0; j < N; ++j) top = max_abs2(top, NORM ? f2_mul(h.p[j], g.p[j]) : h.p[j]);
        }
    });
    float s0, s1;
    f2_unpack(sum, s0, s1);
    const float2 all = meet(s0 + s1, top, codes);
    RowScale o{1.0f, 1.0f, all.y};
    if (!NORM) return o;
    const float m = fmaf(all.x, A.inv_c, A.eps);
    o.q = root(m);
    o.top *= o.q;
    // (An h gamma below 2^-126 has not all its digits: y, which is (h q) gamma, may be larger than q times the largest of them, or be there without one.)
    // The rows of a warp take the turn together and keep what is theirs.
    const bool far = !(m > 1e-30f && m < 1e30f && o.top < 3e38f) || (codes && all.y < 1e-30f);
    if (WIDE ? far : __any_sync(0xFFFFFFFFu, far)) {
        const RowScale again = row_far<WIDE, T>(A, L, row, meet, all.y, far);
        if (far) o = again;
    }
    return o;
}

template <bool NORM, typename T, int V, int P, int KIND, bool KEEP>
__device__ __forceinline__ void row_write(const RmsArgs& A, const RowLanes<V, P, KIND>& L, RowValues<T, V, P, KIND>& row,
                                          const RowGamma<T, V, P, KIND, KEEP>& gamma, const RowScale& o, uint32_t index, uint32_t n, uint32_t s, bool codes) {
    constexpr int N = Pairs<V>::N;
    const int C = A.shape.C;
    if (NORM && A.rstd && L.lane == 0) A.rstd[index] = o.q * o.f;
    bool plain = o.f == 1.0f;
    float inv = 0.f;
    if (codes) {
        const RowCodes k(o);
        if (L.lane == 0) A.scales[index] = k.scale;
        plain = k.plain;
        inv = k.inv;
    }
    T* to_h = NORM && A.h.p ? static_cast<T*>(A.h.p) + row_at(A.h, n, s) : nullptr;
    T* to_y = NORM && A.y.p ? static_cast<T*>(A.y.p) + row_at(A.y, n, s) : nullptr;
    int8_t* to_c = codes ? static_cast<int8_t*>(A.codes.p) + row_at(A.codes, n, s) : nullptr;
    if constexpr (P > 0) {  // a row in registers; one that is read again may lie where h goes, and is stored with y below
        if (to_h) row.visit(L, [&](int, int c, const Pairs<V>& h, auto whole, bool there) { row_store<T, V, decltype(whole)::value>(to_h, c, C, h, there); });
        if (!to_y && !codes) return;
    }
    auto write = [&](auto is_plain, const auto& divide) {
        constexpr bool PLAIN = decltype(is_plain)::value;
        row.visit(L, [&](int i, int c, const Pairs<V>& h, auto whole, bool there) {
            constexpr bool W = decltype(whole)::value;
            if (P == 0 && to_h) row_store<T, V, W>(to_h, c, C, h, there);
            Pairs<V> y = h;
            if (NORM) {
                if (!PLAIN) {
#pragma unroll
                    for (int j = 0; j < N; ++j) y.p[j] = f2_mul(y.p[j], f2_splat(o.f));
                }
                const Pairs<V> g = gamma.template get<W>(i, c);
#pragma unroll
                for (int j = 0; j < N; ++j) y.p[j] = f2_mul(f2_mul(y.p[j], f2_splat(o.q)), g.p[j]);
            }
            if (to_y) row_store<T, V, W>(to_y, c, C, y, there);
            if (codes) {
                if constexpr (!PLAIN) {
#pragma unroll
                    for (int j = 0; j < N; ++j) y.p[j] = divide(y.p[j]);
                }
                codes_store<V, W>(to_c, c, C, y, PLAIN ? inv : 1.0f, there);
            }
        });
    };
    if constexpr (!NORM && P > 0) {
        if (plain) {
            write(Whole(), 0);
            return;
        }
        // read again, piece by piece (from registers: up to 34 more of them, 32760 x 8960 190 us, for the values are kept in their own type until here)
        const RowDivide divide(o.top);
        auto again = [&](int c, auto whole) {
            constexpr bool W = decltype(whole)::value;
            Pairs<V> y = row.template get<W>(c, C);
#pragma unroll
            for (int j = 0; j < N; ++j) y.p[j] = divide(y.p[j]);
            codes_store<V, W>(to_c, c, C, y, 1.0f, true);
        };
#pragma unroll 1
        for (int i = 0; i < P; ++i)
            if (L.has(i)) again(L.channel(i), Whole());
        if (!L.FULL && V > 1 && L.tail) again(L.end(), Part());
    } else if (plain) {
        write(Whole(), 0);
    } else {
        write(Part(), RowDivide(o.top));
    }
}

// Rows that a thread has in hand at once (more warps are worth more than more rows a warp: 32760 x 12 heads of 128 channels, two pieces a thread, 1, 2, 4 rows: 34.6, 38.8, 37.1 us).
__host__ __device__ constexpr int rows_at_once(int P) { return P == 1 ? 2 : 1; }
// Registers of a thread of a wide row, and with them threads of a CTA at most.  (Given a number of threads instead, the compiler spills to 80 registers for an occupancy
// that is of no use: 32760 x 5120 with residual and y 228 us.)
__host__ __device__ constexpr int rows_registers(int V, int P) { return P * V > 40 ? 128 : P * V > 24 ? 112 : P * V > 8 ? 96 : 64; }
__host__ __device__ constexpr int rows_threads(int V, int P) { return 65536 / rows_registers(V, P) / 32 * 32; }

// What a call asks for, as far as kernels are built for it (each branch of an inner loop costs as much as a piece's arithmetic): a
// residual, codes; else all is looked up at run time.
enum RowsAsk { kAskAny = 0, kAskPlain = 1, kAskResidual = 2, kAskCodes = 3, kAskBoth = 4 };

// WIDE: a row has the CTA to itself.
template <typename T, int V, int P, bool NORM, bool WIDE, bool FULL, int ASK>
__device__ __forceinline__ void rms_norm_rows(const RmsArgs& A) {
    constexpr int U = WIDE ? 1 : rows_at_once(P);
    constexpr bool KEEP = NORM && P > 0 && P * V <= 40;
    constexpr int KIND = (FULL ? kFull : 0) | (WIDE ? kWide : 0);
    const bool both = ASK == kAskAny ? A.r.p != nullptr : ASK == kAskResidual || ASK == kAskBoth;
    const bool codes = !NORM || (ASK == kAskAny ? A.scales != nullptr : ASK == kAskCodes || ASK == kAskBoth);
    __shared__ float2 slots[64];
    const int lanes = WIDE ? (int)blockDim.x : A.lanes, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    const int groups = WIDE ? 1 : kSmallThreads >> A.lanes_log2, group = WIDE ? 0 : (int)threadIdx.x >> A.lanes_log2;
    const RowLanes<V, P, KIND> L(A.shape.C, lanes, lane);
    RowMeet<WIDE> meet(slots, lanes);
    wait_predecessor();
    release_successor();
    RowGamma<T, V, P, KIND, KEEP> gamma;
    if (NORM) gamma.init(L, A.gamma, A.params_f32);
    for (int64_t at = (int64_t)blockIdx.x * (groups * U); at < A.shape.rows; at += (int64_t)gridDim.x * (groups * U)) {
        RowValues<T, V, P, KIND> rows[U];
        uint32_t index[U], n[U], s[U];
        bool active[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = at + u * groups + group;
            active[u] = WIDE || row < A.shape.rows;
            index[u] = (uint32_t)(active[u] ? row : at);  // threads without a row of their own take part in the exchanges
            n[u] = A.shape.by_s(index[u]);
            s[u] = index[u] - n[u] * (uint32_t)A.shape.S;
            rows[u].x = static_cast<const T*>(A.x.p) + row_at(A.x, n[u], s[u]);
            rows[u].r = both ? static_cast<const T*>(A.r.p) + row_at(A.r, n[u], s[u]) : nullptr;
        }
        rows_load<T, V, P, KIND, U>(L, rows, active, both);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const RowScale o = row_decide<NORM>(A, L, rows[u], gamma, meet, codes);
            if (active[u]) row_write<NORM>(A, L, rows[u], gamma, o, index[u], n[u], s[u], codes);
        }
    }
}

template <typename T, int V, int P, bool NORM, bool FULL, int ASK>
__global__ void __maxnreg__(rows_registers(V, P))
rms_norm_wide_kernel(const __grid_constant__ RmsArgs A) {
    rms_norm_rows<T, V, P, NORM, true, FULL, ASK>(A);
}
template <typename T, int V, int P, bool NORM, bool FULL, int ASK>
__global__ void __launch_bounds__(kSmallThreads)
rms_norm_kernel(const __grid_constant__ RmsArgs A) {
    rms_norm_rows<T, V, P, NORM, false, FULL, ASK>(A);
}

// ------------------------------------------------------------------ launches

template <typename T, int V, int P, bool NORM, bool WIDE, bool FULL, int ASK>
static cudaError_t launch_rms_p(const RmsArgs& A0, const RowsPlan& p, cudaStream_t st) {
    RmsArgs A = A0;
    A.lanes = p.lanes;
    A.lanes_log2 = p.lanes_log2;
    void (*kern)(RmsArgs);
    if constexpr (WIDE) kern = rms_norm_wide_kernel<T, V, P, NORM, FULL, ASK>;
    else kern = rms_norm_kernel<T, V, P, NORM, FULL, ASK>;
    static PerDevice<RowsHeld> cache;
    const int held = rows_held(cache, kern, p.threads);
    if (held == 0) return cudaErrorInvalidValue;
    const int64_t at_once = WIDE ? 1 : (int64_t)(kSmallThreads / p.lanes) * rows_at_once(P), ctas = ceil_div(A.shape.rows, at_once);
    return launch_after(kern, dim3((unsigned)(ctas < 148 * held ? ctas : 148 * held)), dim3(p.threads), 0, st, A);
}
template <typename T, int V, int P, bool NORM, bool FULL, int ASK>
static cudaError_t launch_rms_w(const RmsArgs& A, const RowsPlan& p, cudaStream_t st) {
    return p.wide ? launch_rms_p<T, V, P, NORM, true, FULL, ASK>(A, p, st) : launch_rms_p<T, V, P, NORM, false, FULL, ASK>(A, p, st);
}
template <typename T, int V, int P, bool NORM, bool FULL>
static cudaError_t launch_rms_ask(const RmsArgs& A, const RowsPlan& p, cudaStream_t st) {
    if constexpr (NORM) {
        if (A.r.p && A.scales) return launch_rms_w<T, V, P, NORM, FULL, kAskBoth>(A, p, st);
        if (A.r.p) return launch_rms_w<T, V, P, NORM, FULL, kAskResidual>(A, p, st);
        if (A.scales) return launch_rms_w<T, V, P, NORM, FULL, kAskCodes>(A, p, st);
        return launch_rms_w<T, V, P, NORM, FULL, kAskPlain>(A, p, st);
    }
    return launch_rms_w<T, V, P, NORM, FULL, kAskCodes>(A, p, st);
}
template <typename T, int V, bool NORM>
static cudaError_t launch_rms_v(const RmsArgs& A, cudaStream_t st) {
    constexpr bool kPieces16 = V * sizeof(T) == 16;
    // Pieces a thread, 4 and 5, 32760 x 5120: residual and codes 190 and 181 us, residual and y 209 and 225, y alone 144 and 118; 6 and more leave too few warps
    // (267).  Rows whose pieces do not fill the threads: 8 (20000 x 1541, odd: 1, 2, 4, 8, 16 pieces 389, 183, 119, 94, 91 us).
    static const int five[] = {5, 4, 6, 7, 8, 3, 2, 1, 0}, four[] = {4, 5, 6, 7, 8, 3, 2, 1, 0};
    const RowsPlan p = rows_plan(A.shape.rows, ceil_div(A.shape.C, V), kPieces16 && A.shape.C % V == 0, 8, 8, 8, [](int k) { return rows_threads(V, k); },
                                 A.r.p && !A.scales ? four : five);
    if constexpr (kPieces16) {
        if (p.full) {
            switch (p.pieces) {
                case 1: return launch_rms_ask<T, V, 1, NORM, true>(A, p, st);
                case 2: return launch_rms_ask<T, V, 2, NORM, true>(A, p, st);
                case 3: return launch_rms_ask<T, V, 3, NORM, true>(A, p, st);
                case 4: return launch_rms_ask<T, V, 4, NORM, true>(A, p, st);
                case 5: return launch_rms_ask<T, V, 5, NORM, true>(A, p, st);
                case 6: return launch_rms_ask<T, V, 6, NORM, true>(A, p, st);
                case 7: return launch_rms_ask<T, V, 7, NORM, true>(A, p, st);
                default: return launch_rms_ask<T, V, 8, NORM, true>(A, p, st);
            }
        }
    }
    constexpr int ask = NORM ? kAskAny : kAskCodes;
    switch (p.pieces) {
        case 0: return launch_rms_p<T, V, 0, NORM, true, false, ask>(A, p, st);
        case 1: return launch_rms_w<T, V, 1, NORM, false, ask>(A, p, st);
        case 2: return launch_rms_w<T, V, 2, NORM, false, ask>(A, p, st);
        case 4: return launch_rms_ask<T, V, 4, NORM, false>(A, p, st);
        default: return launch_rms_ask<T, V, 8, NORM, false>(A, p, st);
    }
}
// `access`: bytes of a piece that every tensor's alignment allows: 16, 4 or the element's
template <typename T, bool NORM>
static cudaError_t launch_rms_t(const RmsArgs& A, int access, cudaStream_t st) {
    if (access == 16) return launch_rms_v<T, 16 / sizeof(T), NORM>(A, st);
    if (sizeof(T) == 2 && access == 4) return launch_rms_v<T, 4 / sizeof(T), NORM>(A, st);
    return launch_rms_v<T, 1, NORM>(A, st);
}

}  // namespace dvdq
