// The linear layer on 8-bit integers with a scale for each token and each output channel:
//
//   acc[m, n] = sum_k a[m, k] w[n, k]  (int32, exact),   y = act(acc s_m t_n + bias_n) + residual
//
// The tiling, the rings, the roles of the warps and the walk over tiles are those of the 16-bit layer (linear.cuh); what differs: stages
// of 128 along k (the same 128-byte rows), tcgen05.mma.cta_group::2.kind::i8 256 x bn x 32 into int32 accumulators, and an epilogue that
// multiplies by the two scales in fp32: acc (below 2^31) is rounded to fp32 once, the product of the scales once, their product is added to the
// bias in one fma, and the output is rounded once.  Pieces of k are joined as integers, so that the result does not depend on how many there are.
//
// What bounds it: the tensor pipe on layers of thousands of tokens, and with it the power cap: 32760 x 5120 -> 13824 with GELU takes 1037 us (4.47 PTOPS, the issue
// loop's 4.43) when all codes are zero, and 1400-1840 (2.5-3.3 PTOPS) with codes of normal values, by the clock (the vendor library's bare product in the same
// run 1670-1990).  8192 x 5120 -> 5120: tensor pipe 91 % active.  Short contractions: the epilogue (a tile of 256 x 256 outputs takes a pair 2.9 us, 4.6
// with an activation, 4.3 with a residual in wide blocks; 12 k-blocks of products 3.4).  Few tokens: streaming W (1 token 5120 -> 13824 15.2 us, 4.7 TB/s).
#pragma once

#include "linear.cuh"

namespace dvdq {

constexpr int kL8BK = 128;  // elements of k per stage: one 128-byte swizzle row

template <int OUT, bool WIDE>
struct L8Smem {
    // a residual that comes early takes two more blocks per epilogue warp (one, where they are wide), and 32 KB of the ring
    static constexpr int kRing = (OUT == kLinFinalMore ? (WIDE ? 4 : 5) : (WIDE ? 5 : 6)) * 32768;
    static constexpr int kMaxStages = OUT == kLinFinalMore ? 12 : 16;  // a stage is 32 KB at most; narrow tiles and few rows take less
    static constexpr int kBufs = OUT == kLinFinalMore ? (WIDE ? 3 : 4) : 2;
    static constexpr int kCols = WIDE ? 64 : 32;            // of an epilogue block
    static constexpr int kBuf = 32 * kCols * 2;             // 32 x kCols outputs; int32 pieces use two as one
    static constexpr int kBufOff = kRing;
    static constexpr int kScaleOff = kBufOff + kLinEpiWarps * kBufs * kBuf;   // per warp: 32 scales, 32 biases as they come
    static constexpr int kBarOff = kScaleOff + kLinEpiWarps * 32 * (4 + 2);
    static constexpr int kResBars = OUT == kLinFinalMore ? 4 * kLinEpiWarps : 0;
    static constexpr int kNumBars = 2 * kMaxStages + 5 + kResBars;
    static constexpr int kMiscOff = kBarOff + kNumBars * 8;
    static constexpr int kTotal = kMiscOff + 16 + 1024;
    static_assert(kTotal <= 232448, "more than the 227 KB of shared memory a CTA can have");
};

struct L8Args {
    LinArgs t;
    const float *a_scales, *w_scales;
};

template <typename T, int OUT, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinThreads, 1)
linear_int8_kernel(const __grid_constant__ LinMaps maps, const __grid_constant__ CUtensorMap tmR, const __grid_constant__ L8Args args) {
    const LinArgs& A = args.t;
    const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    const int items = A.num_m * A.num_n * A.splits;
    using S = L8Smem<OUT, WIDE>;
    constexpr int MS = S::kMaxStages;
    const uint32_t ST = (uint32_t)A.stages, stage = (uint32_t)A.stage;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();

    const uint32_t bar0 = sbase + S::kBarOff;
    auto full = [&](int s) { return bar0 + 8u * s; };                    // leader's copy: both CTAs' operands are in place
    auto empty = [&](int s) { return bar0 + 8u * (MS + s); };            // one per CTA
    auto acc_full = [&](int s) { return bar0 + 8u * (2 * MS + s); };     // one per CTA
    auto acc_empty = [&](int s) { return bar0 + 8u * (2 * MS + 2 + s); };  // leader's copy
    const uint32_t drain_bar = bar0 + 8u * (2 * MS + 4);
    auto res_full = [&](int w, int b) { return bar0 + 8u * (2 * MS + 5 + 4 * w + b); };  // a warp's residual block has landed
    volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + S::kMiscOff);  // [0] tmem base, [1] abort
    volatile uint32_t* abort_flag = misc + 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < MS; ++s) { mbar_init(full(s), 2); mbar_init(empty(s), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(acc_full(s), 1); mbar_init(acc_empty(s), 2 * kLinEpiWarps); }
        mbar_init(drain_bar, 1);
        for (int w = 0; w < S::kResBars; ++w) mbar_init(res_full(0, w), 1);
        misc[1] = 0u;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(sbase + S::kMiscOff, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = misc[0];
    wait_predecessor();
    release_successor();

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------ TMA producers: warp 0 of A, warp 2 of W
        if (elect_one()) {
            const bool of_a = warp == 0;
            const CUtensorMap* map = of_a ? &maps.a : &maps.b;
            tma_prefetch_desc(map);
            const int bw = A.bn / 2;  // columns per CTA
            const uint32_t leader_full = map_to_cta(full(0), 0);
            LinRing ring(empty(0), ST, 1u);
            const uint32_t dst = sbase + (of_a ? 0 : A.b_off);
            bool ok = true;
            for (int item = pair; ok && item < items; item += num_pairs) {
                int tm, tn, piece;
                lin_item(A, item, tm, tn, piece);
                const int2 kr = lin_range(A, piece);
                const int r0 = of_a ? tm * kLinTile + (int)rank * 128 : tn * A.bn + (int)rank * bw;
                // rows past the last token need no operand: whatever lies in their stage reaches only rows that are not stored
                const bool needed = !of_a || r0 < A.Md;
                const uint32_t bytes = of_a ? A.a_bytes * (tm * kLinTile + 128 < A.Md ? 2u : 1u) : 2u * (uint32_t)(bw * kL8BK);
                int k0 = kr.x * kL8BK;
                ok = ring.walk(kr.y - kr.x, abort_flag, kWaitWideEmpty, [&](uint32_t st) {
                    if (rank == 0) mbar_arrive_expect_tx(full(st), bytes);
                    if (needed) tma_load_2d_pair(dst + st * stage, map, leader_full + 8u * st, k0, r0);
                    k0 += kL8BK;
                });
            }
            if (!ok)  // giving up after seconds of waiting: a bounded pause covers the last copies
                for (int it = 0; it < 64; ++it) __nanosleep(1000);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products (leader CTA only)
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = umma_idesc_s8s8s32(kLinTile, A.bn);
            const uint64_t ad0 = umma_desc_sw128_kmajor(sbase), bd0 = umma_desc_sw128_kmajor(sbase + A.b_off);
            LinRing ring(full(0), ST, 0u);
            uint32_t lt = 0;
            bool ok = true;
            for (int item = pair; ok && item < items; item += num_pairs, ++lt) {
                int tm, tn, piece;
                lin_item(A, item, tm, tn, piece);
                const int2 kr = lin_range(A, piece);
                const uint32_t a = lt & 1u, aph = (lt >> 1) & 1u;
                if (!mbar_wait(acc_empty(a), aph ^ 1u, abort_flag, kWaitAccEmpty)) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + a * kLinTile;
                uint32_t add = 0u;
                ok = ring.walk(kr.y - kr.x, abort_flag, kWaitWideFull, [&](uint32_t st) {
                    tc_fence_after();
                    const uint32_t off = st * (stage >> 4);  // in the descriptors' 16-byte units
#pragma unroll
                    for (int k = 0; k < kL8BK / 32; ++k) {   // 32 codes along k: 32 bytes inside a swizzle row
                        tc_mma_i8_ss_pair(d_tmem, ad0 + (off + 2u * k), bd0 + (off + 2u * k), idesc, add);
                        add = 1u;
                    }
                    tc_commit_pair(empty(st), 3);
                });
                if (ok) tc_commit_pair(acc_full(a), 3);
            }
            tc_commit_pair(drain_bar, 1);
            mbar_wait(drain_bar, 0u, abort_flag, kWaitDrain);
        }
        __syncwarp();
    } else if (warp >= kLinFirstEpi) {
        // ------------------------------------------------------------ epilogue
        const int ew = warp - kLinFirstEpi;
        const int q = warp & 3, half = ew >> 2;  // tensor-memory lane quarter; which of every two blocks of columns
        const uint32_t buf0 = sbase + S::kBufOff + ew * (S::kBufs * S::kBuf);
        const uint32_t c_scale = sbase + S::kScaleOff + ew * (32 * 6), c_bias = c_scale + 128;
        const bool residual = OUT == kLinFinalMore;
        const bool with_bias = OUT != kLinPartial && A.bias != nullptr;
        const uint16_t* bias = static_cast<const uint16_t*>(A.bias);
        constexpr uint32_t turns = S::kBufs;  // output blocks take turns in so many buffers
        if (lane == 0) tma_prefetch_desc(&maps.y);
        const int rows_from = (int)rank * 128 + q * 32;
        uint32_t lt = 0;
        uint32_t buf_i = 0;               // the next block's buffer
        uint32_t rask = 0, rphase = 0;    // the next residual's buffer; the parity to wait for, a bit per buffer
        uint32_t pending = 0;             // residual blocks asked for and not taken
        bool ok = true;
        // Asks for the residual of the next block ahead, into the buffer whose turn it is (as linear.cuh)
        LinBlocks<S::kCols> ahead;
        ahead.item = pair;
        auto ask = [&]() {
            ahead.next(A, items, num_pairs, rows_from, half);
            if (!ahead.more) return;
            if (lane == 0) {
                tma_store_wait_read<1>();
                mbar_arrive_expect_tx(res_full(ew, rask), S::kBuf);
                tma_load_2d(buf0 + rask * S::kBuf, &tmR, res_full(ew, rask), ahead.col0 + ahead.c * (2 * S::kCols), ahead.row0);
            }
            rask = rask + 1 == turns ? 0u : rask + 1;
            ++pending;
        };
        if (residual)
            for (uint32_t i = 1; i < turns; ++i) ask();
        LinBlocks<S::kCols> b;
        for (b.item = pair; ok && b.item < items; b.item += num_pairs, ++lt) {
            b.tile(A, rows_from, half);
            const uint32_t a = lt & 1u, aph = (lt >> 1) & 1u;
            const int row0 = b.row0, col0 = b.col0, blocks = b.blocks, piece = b.piece;
            // the next 32 columns' scales and biases, a lane each: asked for a block ahead
            float t_next = 0.f, s_m = 0.f;
            uint16_t b_next = 0;
            auto ask_columns = [&](int from) {
                const bool in = from + lane < A.Nd;
                t_next = in ? args.w_scales[from + lane] : 0.f;
                if (with_bias) b_next = in ? bias[from + lane] : (uint16_t)0;
            };
            if (OUT != kLinPartial && blocks > 0) {
                ask_columns(col0);
                if (row0 + lane < A.Md) s_m = args.a_scales[row0 + lane];
            }
            const uint64_t s2 = f2_pack(s_m, s_m);
            __syncwarp();
            ok = mbar_wait_one_lane(acc_full(a), aph, abort_flag, kWaitAccFull);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < blocks; ++c) {
                if constexpr (OUT == kLinPartial) {
                    uint32_t r[32];
                    __syncwarp();
                    tmem_ld_32x32(tmem_base + a * kLinTile + half * 32 + c * 64 + ((uint32_t)(q * 32) << 16), r);
                    if (lane == 0) tma_store_wait_read<0>();
                    __syncwarp();
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 8; ++j)  // rows of 128 bytes, 16-byte chunk index XORed with row % 8
                        sts128(buf0 + lane * 128 + ((j ^ (lane & 7)) << 4), r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&maps.y, buf0, col0 + c * 64, piece * A.part_rows + row0);
                        tma_store_commit();
                    }
                } else {
                    const uint32_t buf = buf0 + buf_i * S::kBuf;
                    const int block_col = col0 + c * (2 * S::kCols);
#pragma unroll
                    for (int h = 0; h < S::kCols / 32; ++h) {  // 32 columns at a time
                        uint32_t r[32];
                        __syncwarp();
                        tmem_ld_32x32(tmem_base + a * kLinTile + half * S::kCols + c * (2 * S::kCols) + h * 32 + ((uint32_t)(q * 32) << 16), r);
                        // the block's output buffer (without a residual: else ask() has waited for it): free once all but the newest store have been read
                        if (h == 0 && !residual && lane == 0) tma_store_wait_read<1>();
                        sts32f(c_scale + 4 * lane, t_next);
                        if (with_bias) asm volatile("st.shared.u16 [%0], %1;" ::"r"(c_bias + 2 * lane), "h"(b_next) : "memory");
                        __syncwarp();
                        ask_columns(h + 1 < S::kCols / 32 ? block_col + (h + 1) * 32 : c + 1 < blocks ? block_col + 2 * S::kCols : A.Nd);
                        if (residual && h == 0) {
                            ok = mbar_wait_one_lane(res_full(ew, buf_i), (rphase >> buf_i) & 1u, abort_flag, kWaitPackedFull);
                            if (!ok) break;
                            rphase ^= 1u << buf_i;
                            --pending;
                        }
                        tmem_ld_wait();
                        uint64_t v[16];  // pairs of columns
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = f2_pack((float)(int)r[2 * j], (float)(int)r[2 * j + 1]);
                        if (with_bias) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint4 w = lds128(c_bias + 16 * j);
                                const float4 t0 = lds128f(c_scale + 32 * j), t1 = lds128f(c_scale + 32 * j + 16);
                                const Pairs<8> f = widen2<T, 8>(*reinterpret_cast<const Vec<T, 8>*>(&w));
                                v[4 * j] = f2_fma(v[4 * j], f2_mul(s2, f2_pack(t0.x, t0.y)), f.p[0]);
                                v[4 * j + 1] = f2_fma(v[4 * j + 1], f2_mul(s2, f2_pack(t0.z, t0.w)), f.p[1]);
                                v[4 * j + 2] = f2_fma(v[4 * j + 2], f2_mul(s2, f2_pack(t1.x, t1.y)), f.p[2]);
                                v[4 * j + 3] = f2_fma(v[4 * j + 3], f2_mul(s2, f2_pack(t1.z, t1.w)), f.p[3]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float4 t0 = lds128f(c_scale + 16 * j);
                                v[2 * j] = f2_mul(v[2 * j], f2_mul(s2, f2_pack(t0.x, t0.y)));
                                v[2 * j + 1] = f2_mul(v[2 * j + 1], f2_mul(s2, f2_pack(t0.z, t0.w)));
                            }
                        }
                        if (A.act == DVDQ_ACT_GELU_TANH) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = act_value2<DVDQ_ACT_GELU_TANH>(v[j]);
                        } else if (A.act == DVDQ_ACT_SILU) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = act_value2<DVDQ_ACT_SILU>(v[j]);
                        }
                        // what the swizzled TMA copies use: rows of 64 bytes, 16-byte chunk index XORed with (row / 2) % 4, or of
                        // 128 bytes, with row % 8
                        auto at = [&](int j) {
                            return WIDE ? buf + lane * 128 + (((h * 4 + j) ^ (lane & 7)) << 4) : buf + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4);
                        };
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (residual) {
                                const uint4 w = lds128(at(j));
                                const Pairs<8> f = widen2<T, 8>(*reinterpret_cast<const Vec<T, 8>*>(&w));
#pragma unroll
                                for (int t = 0; t < 4; ++t) v[4 * j + t] = f2_add(v[4 * j + t], f.p[t]);
                            }
                            uint32_t w[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                float lo, hi;
                                f2_unpack(v[4 * j + t], lo, hi);
                                w[t] = pack2<T>(lo, hi);
                            }
                            sts128(at(j), w[0], w[1], w[2], w[3]);
                        }
                    }
                    if (!ok) break;
                    buf_i = buf_i + 1 == turns ? 0u : buf_i + 1;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&maps.y, buf, block_col, row0);
                        tma_store_commit();
                    }
                    if (residual) ask();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty(a), 0));
        }
        if (lane == 0) {
            tma_store_wait_all();
            // gave up with residual blocks in flight: let them land (bounded) before the CTA exits
            for (; pending > 0; --pending) {
                for (int it = 0; it < (1 << 16) && !mbar_try_wait(res_full(ew, buf_i), (rphase >> buf_i) & 1u); ++it) {}
                buf_i = buf_i + 1 == turns ? 0u : buf_i + 1;
            }
        }
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) tmem_dealloc(tmem_base, 512);
}

// ------------------------------------------------------------------ joining the pieces

// One output before the residual, from its accumulator: the operations of the epilogue above, so that an output's bits do not depend on which kernel
// or how many pieces it comes from.
template <typename T>
__device__ __forceinline__ float l8_value(int acc, float s, float t, const T* bias, int n, int act) {
    const float f = (float)acc, st = s * t;
    float z = bias ? fmaf(f, st, to_f32(bias[n])) : f * st, other;
    if (act == DVDQ_ACT_GELU_TANH) f2_unpack(act_value2<DVDQ_ACT_GELU_TANH>(f2_splat(z)), z, other);
    else if (act == DVDQ_ACT_SILU) f2_unpack(act_value2<DVDQ_ACT_SILU>(f2_splat(z)), z, other);
    return z;
}

// y from the sum of the pieces, four columns per thread.
template <typename T>
__global__ void __launch_bounds__(256)
linear_int8_join_kernel(const int32_t* __restrict__ part, int64_t piece_ints, int pitch, int splits, int64_t Md, int Nd, const float* __restrict__ a_scales,
                        const float* __restrict__ w_scales, const T* __restrict__ bias, const T* residual, int64_t ldr, int act, T* y, int64_t ldy) {
    wait_predecessor();
    release_successor();
    const int quads = (Nd + 3) >> 2;
    const int64_t total = Md * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int n = (int)(i - m * quads) * 4;
        const int32_t* p = part + m * pitch + n;
        int4 s = *reinterpret_cast<const int4*>(p);
#pragma unroll 4
        for (int k = 1; k < splits; ++k) {
            const int4 t = *reinterpret_cast<const int4*>(p + k * piece_ints);
            s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
        }
        const int acc[4] = {s.x, s.y, s.z, s.w}, here = Nd - n < 4 ? Nd - n : 4;
        const float s_m = a_scales[m];
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < here) v[j] = l8_value(acc[j], s_m, w_scales[n + j], bias, n + j, act);
        if (here == 4) {  // rows start on 16 bytes and n is a multiple of 4: 8-byte accesses
            if (residual) {
                const uint2 w = *reinterpret_cast<const uint2*>(residual + m * ldr + n);
                const float2 f0 = unpack2<T>(w.x), f1 = unpack2<T>(w.y);
                v[0] += f0.x; v[1] += f0.y; v[2] += f1.x; v[3] += f1.y;
            }
            *reinterpret_cast<uint2*>(y + m * ldy + n) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
        } else {
            for (int j = 0; j < here; ++j) {
                float o = v[j];
                if (residual) o += to_f32(residual[m * ldr + n + j]);
                y[m * ldy + n + j] = from_f32<T>(o);
            }
        }
    }
}

// ------------------------------------------------------------------ a few tokens

// 16 warps to a group of 16 channels where an SM has two groups at most.
inline bool l8_long_few(int64_t N, int64_t K) { return ceil_div(N, 16) <= 148 * 2 && K >= 1024; }

// Which calls: up to 8 tokens all.  With 16 warps a group also up to 16 tokens, unless the rows are very long, and up to 32 where an SM has one group at
// most (the kernel then takes its registers), unless they are long for so few groups: tiles cut them over all SMs.  Here and in tiles, in us: 16 tokens
// 1536 -> 1536 2.7, 4.8; 2049 -> 4101 5.7, 6.2; 8192 -> 4096 11.0, 13.5; 13824 -> 512 7.7, 8.0; 20000 -> 1536 16.4, 13.5; other warps: 1024 -> 20000 10.8, 9.2,
// 5120 -> 5120 11.0, 10.2.  32 tokens 1536 -> 1536 3.4, 4.9; 5120 -> 2304 6.6, 9.9; 8960 -> 1536 9.6, 10.7; 8960 -> 512 7.8, 7.1; two groups:
// 3584 -> 3584 10.2, 7.8; fewer warps: 300 -> 300 4.8, 3.4.
inline bool l8_few(int64_t M, int64_t N, int64_t K) {
    return M <= 8 || (l8_long_few(N, K) && ((M <= 16 && K <= 16384) || (M <= 32 && N <= 148 * 16 && K <= 6 * N)));
}

// As linear_few_kernel: mma.sync m16n8k32 with 16 rows of W as its A operand and 8 tokens as B, NT times.  A dot product does not care for the order
// of k, so a lane's 16 consecutive codes of a row fill its A slots of two MMAs, and the same 16 codes of a token its B slots.
__device__ __forceinline__ void mma_16x8x32_i8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 codes of a row from column k on; those past K are zero (and are not read).
__device__ __forceinline__ uint4 l8_few_load(const int8_t* row, int k, int K) {
    if (k + 16 <= K) return *reinterpret_cast<const uint4*>(row + k);
    Vec<int8_t, 16> v;
#pragma unroll
    for (int j = 0; j < 16; ++j) v.e[j] = k + j < K ? row[k + j] : (int8_t)0;
    return *reinterpret_cast<const uint4*>(&v);
}

// Asks L2 for the first 512 bytes of a warp's 16 rows of W while the predecessor still runs: nothing is read, so it does not matter who writes W.
// (Behind dvdq_quantize_rows, 1 token: 5120 -> 13824 17.6 and 16.6 us for both, 5120 -> 5120 10.2 and 9.4.  The kernel above gained nothing, and lost
// 1.5 us where rows start off a line.)
__device__ __forceinline__ void l8_few_ahead(const int8_t* W, int64_t ldw, int n0, int N, int k0, int k1) {
    const int lane = threadIdx.x & 31, k = k0 + (lane & 3) * 128;
#pragma unroll
    for (int r = lane >> 2; r < 16; r += 8)
        if (n0 + r < N && k < k1) asm volatile("prefetch.global.L2 [%0];" ::"l"(W + (int64_t)(n0 + r) * ldw + k));
}

constexpr int kL8FewDepth = 6;
template <typename T, int WARPS, int KS, int NT>
__global__ void __launch_bounds__(WARPS * 32, NT <= 2 ? 32 / WARPS : 1)  // the CTAs that an SM holds where WARPS and KS are chosen
linear_int8_few_kernel(const int8_t* __restrict__ X, int64_t ldx, const int8_t* __restrict__ W, int64_t ldw, int M, int N, int K, int k_per_warp,
                       const float* __restrict__ a_scales, const float* __restrict__ w_scales, const T* __restrict__ bias, const T* R, int64_t ldr,
                       int act, T* Y, int64_t ldy) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int piece = warp % KS, group = warp / KS;
    const int n0 = (blockIdx.x * (WARPS / KS) + group) * 16;
    l8_few_ahead(W, ldw, n0, N, piece * k_per_warp, min(K, (piece + 1) * k_per_warp));
    wait_predecessor();
    release_successor();
    int c[NT][4] = {};
    if (n0 < N) {
        // rows past N repeat the last one: their results are not stored
        const int8_t* w0 = W + (int64_t)min(n0 + g, N - 1) * ldw;
        const int8_t* w1 = W + (int64_t)min(n0 + g + 8, N - 1) * ldw;
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        int k = piece * k_per_warp + t * 16;
        const int k1 = min(K, (piece + 1) * k_per_warp);  // k_per_warp is a multiple of 64
        uint4 x[NT];  // the tokens' codes of the next step: asked for a step ahead (5120 -> 2304 8 tokens 4.8 -> 4.3 us, 8960 -> 1536 7.4 -> 6.5)
        auto ask = [&]() {
#pragma unroll
            for (int j = 0; j < NT; ++j) x[j] = 8 * j + g < M && k < k1 ? l8_few_load(X + (8 * j + g) * ldx, k, K) : none;
        };
        ask();
        auto step = [&](const uint4& a, const uint4& b) {
            uint4 now[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) now[j] = x[j];
            k += 64;
            ask();
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                mma_16x8x32_i8(c[j], a.x, b.x, a.y, b.y, now[j].x, now[j].y);
                mma_16x8x32_i8(c[j], a.z, b.z, a.w, b.w, now[j].z, now[j].w);
            }
        };
        const int whole = k1 > k - t * 16 ? (k1 - (k - t * 16)) / 64 : 0;  // steps of 64 that lie in the rows
        thread_stream<kL8FewDepth, 2, int8_t, 16, WARPS * 32>(smem_u32(raw) + threadIdx.x * 16, whole, w0 + k, 64, w1 + k, 64,
            [&](const Vec<int8_t, 16>& a, const Vec<int8_t, 16>& b) { step(*reinterpret_cast<const uint4*>(&a), *reinterpret_cast<const uint4*>(&b)); });
        if (k - t * 16 < k1) {  // the end of the rows
            const bool in = k < K;
            step(in ? l8_few_load(w0, k, K) : none, in ? l8_few_load(w1, k, K) : none);
        }
    }
    __syncthreads();  // the ring's memory becomes the sums'
    int* sh = reinterpret_cast<int*>(raw);  // [warp][token][16]
    constexpr int kTile = NT * 8 * 16;
    int* mine = sh + warp * kTile + 2 * t * 16 + g;  // c = (row g, tokens 2t, 2t + 1), (row g + 8, the same)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        mine[j * 128] = c[j][0];
        mine[j * 128 + 16] = c[j][1];
        mine[j * 128 + 8] = c[j][2];
        mine[j * 128 + 24] = c[j][3];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < (WARPS / KS) * kTile; o += WARPS * 32) {
        const int gr = o / kTile, r = o - gr * kTile, m = r >> 4, n = (blockIdx.x * (WARPS / KS) + gr) * 16 + (r & 15);
        if (m >= M || n >= N) continue;
        int acc = 0;
#pragma unroll
        for (int w = 0; w < KS; ++w) acc += sh[(gr * KS + w) * kTile + r];
        float v = l8_value(acc, a_scales[m], w_scales[n], bias, n, act);
        if (R) v += to_f32(R[m * ldr + n]);
        Y[m * ldy + n] = from_f32<T>(v);
    }
}

// ------------------------------------------------------------------ host side

// Epilogue blocks of 32 x 64 instead of 32 x 32 outputs with a residual, up to this many k-blocks (half the copies, one operand stage less): 32760 x K ->
// 1536, K = 512, 1024, 1536, 2048, 5120, 8960: 52-56, 58-70, 74-83, 90-102, 196-212, 360-365 us, in narrow blocks 60-66, 75-77, 86-88, 91-115, 198-224,
// 292-355 (ranges: the power cap's).  Without a residual narrow ones are the faster from 512 on (35 us, 38).
constexpr int kL8WideMore = 12;

struct L8Scales {
    const float *a, *w;
};

// Tile width and pieces along k: lin_plan's estimate, with k-blocks of 128 codes that take as long as its 64 16-bit values.  Joining integer pieces
// costs more than it says by about 0.3 us a piece (16 x 5120 -> 5120: 12.8 us in 3 pieces of 224-column tiles, 10.0 whole in 96-column ones; 100 x 8960 -> 1536:
// 12.4 in 7 pieces, 10.4 in 3 or 4).
inline LinPlan l8_plan(int64_t M, int64_t N, int64_t K) { return lin_plan(M, N, ceil_div(K, 2), 32, nullptr, 0.3); }

inline bool l8_map(CUtensorMap* tm, CUtensorMapDataType type, const void* base, int64_t rows, int64_t cols, int64_t pitch_bytes, uint32_t box_cols,
                   uint32_t box_rows) {
    PFN_encodeTiled enc = get_encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch_bytes};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(tm, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               type == CU_TENSOR_MAP_DATA_TYPE_UINT8 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int OUT, bool WIDE>
static dvdq_status launch_linear_int8_out(const LinMatrix& a, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinPlan& plan,
                                          const L8Scales& sc, const LinEpilogue& e, const LinMatrix& y, int32_t* part, cudaStream_t st) {
    constexpr bool bf = IsBf16<T>::value != 0;
    using S = L8Smem<OUT, WIDE>;
    LinMaps maps;
    L8Args args;
    const int a_rows = lin_a_rows(M);
    if (!l8_map(&maps.a, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.p, M, K, a.ld, kL8BK, (uint32_t)a_rows) ||
        !l8_map(&maps.b, CU_TENSOR_MAP_DATA_TYPE_UINT8, w.p, N, K, w.ld, kL8BK, (uint32_t)(plan.bn / 2)))
        return DVDQ_ERR_CUDA;
    if (OUT == kLinPartial ? !l8_map(&maps.y, CU_TENSOR_MAP_DATA_TYPE_INT32, part, plan.splits * plan.part_rows, N, plan.part_pitch * 4, 32, 32)
                           : !make_map_out<WIDE>(&maps.y, bf, y, M, N))
        return DVDQ_ERR_CUDA;
    CUtensorMap tmR = maps.y;  // where unused
    if (OUT == kLinFinalMore && !make_map_out<WIDE>(&tmR, bf, e.residual, M, N)) return DVDQ_ERR_CUDA;
    LinArgs& A = args.t;
    A = LinArgs{};
    A.Md = (int)M;
    A.Nd = (int)N;
    A.num_m = (int)ceil_div(M, kLinTile);
    A.bn = plan.bn;
    A.num_n = (int)ceil_div(N, plan.bn);
    A.kblocks = (int)ceil_div(K, kL8BK);
    A.splits = plan.splits;
    A.panel = 2048 / plan.bn < A.num_n ? 2048 / plan.bn : A.num_n;
    A.by_splits = FastDiv((uint32_t)A.splits);
    A.by_panel_tiles = FastDiv((uint32_t)(A.num_m * A.panel));
    A.by_panel = FastDiv((uint32_t)A.panel);
    A.by_last = FastDiv((uint32_t)(A.num_n - (A.num_n - 1) / A.panel * A.panel));
    A.part_rows = (int)plan.part_rows;
    A.a_bytes = a_rows * kL8BK;
    A.b_off = (int)align_up(A.a_bytes, 1024);  // swizzle atoms are 1024 bytes
    A.stage = A.b_off + (int)align_up(plan.bn / 2 * kL8BK, 1024);
    A.stages = S::kRing / A.stage < S::kMaxStages ? S::kRing / A.stage : S::kMaxStages;
    A.act = e.act;
    A.bias = OUT != kLinPartial ? e.bias : nullptr;
    args.a_scales = sc.a;
    args.w_scales = sc.w;
    auto kern = linear_int8_kernel<T, OUT, WIDE>;
    static PerDevice<int> cache;
    const int max_pairs = resident_pairs(cache, kern, kLinThreads, S::kTotal);
    if (max_pairs == 0) return DVDQ_ERR_CUDA;
    const int64_t items = (int64_t)A.num_m * A.num_n * A.splits;
    const unsigned pairs = (unsigned)(items < max_pairs ? items : max_pairs);
    return cuda_status(launch_after(kern, dim3(2 * pairs), dim3(kLinThreads), S::kTotal, st, maps, tmR, args));
}

template <typename T, int WARPS, int KS, int NT>
static cudaError_t launch_linear_int8_few_w(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const L8Scales& sc,
                                            const LinEpilogue& e, const LinMatrix& y, cudaStream_t st) {
    static_assert(NT * 8 * 16 * 4 <= 32 * 32 * kL8FewDepth, "the sums of a warp fit its rings");
    constexpr int smem = WARPS * 32 * 32 * kL8FewDepth;  // the rings; the sums take their place
    auto kern = linear_int8_few_kernel<T, WARPS, KS, NT>;
    static PerDevice<int> ready;
    if (smem > 48 * 1024 &&
        !ready.get([&](int&, int) { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess; }))
        return cudaErrorInvalidValue;
    const int per_warp = (int)align_up(ceil_div(K, KS), 64);
    return launch_after(kern, dim3((unsigned)ceil_div(N, 16 * (WARPS / KS))), dim3(WARPS * 32), smem, st, static_cast<const int8_t*>(x.p), x.ld,
                        static_cast<const int8_t*>(w.p), w.ld, (int)M, (int)N, (int)K, per_warp, sc.a, sc.w, static_cast<const T*>(e.bias),
                        static_cast<const T*>(e.residual.p), e.residual.ld, e.act, static_cast<T*>(const_cast<void*>(y.p)), y.ld);
}
// Warps that share 16 channels, as launch_linear_few chooses them.  In us, KS = 2, 4, 8, 16: 1 token 5120 -> 13824 22.9, 16.0, 18.3, 17.8 (71 MB: 10.8 at the copy
// rate); 5120 -> 5120 20.5, 12.0, 9.0, 10.2; 8960 -> 1536 34.6, 18.7, 10.8, 6.9; 3 tokens 1536 -> 1536 7.5, 4.3, 3.2, 3.0
// (since then the tokens' codes are asked for a step ahead: 15.2, 8.8, 5.9 and 2.2 with the KS chosen).
template <typename T>
static dvdq_status launch_linear_int8_few(const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const L8Scales& sc,
                                          const LinEpilogue& e, const LinMatrix& y, cudaStream_t st) {
    const int64_t groups = ceil_div(N, 16), wave = 148 * 4 * 8;
    if (M > 16) return cuda_status(launch_linear_int8_few_w<T, 16, 16, 4>(x, w, M, N, K, sc, e, y, st));
    if (M > 8) return cuda_status(launch_linear_int8_few_w<T, 16, 16, 2>(x, w, M, N, K, sc, e, y, st));
    if (l8_long_few(N, K)) return cuda_status(launch_linear_int8_few_w<T, 16, 16, 1>(x, w, M, N, K, sc, e, y, st));
    if (groups * 8 <= wave) return cuda_status(launch_linear_int8_few_w<T, 8, 8, 1>(x, w, M, N, K, sc, e, y, st));
    if (groups * 4 <= wave) return cuda_status(launch_linear_int8_few_w<T, 8, 4, 1>(x, w, M, N, K, sc, e, y, st));
    if (groups * 2 <= wave) return cuda_status(launch_linear_int8_few_w<T, 8, 2, 1>(x, w, M, N, K, sc, e, y, st));
    return cuda_status(launch_linear_int8_few_w<T, 8, 1, 1>(x, w, M, N, K, sc, e, y, st));
}

template <typename T>
static dvdq_status launch_linear_int8(const LinMatrix& a, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinPlan& plan,
                                      const L8Scales& sc, const LinEpilogue& e, const LinMatrix& y, int32_t* part, cudaStream_t st) {
    if (l8_few(M, N, K)) return launch_linear_int8_few<T>(a, w, M, N, K, sc, e, y, st);
    if (plan.splits == 1) {
        // a tile is whole blocks for both warps
        if (e.residual.p && plan.bn % 128 == 0 && ceil_div(K, kL8BK) <= kL8WideMore) return launch_linear_int8_out<T, kLinFinalMore, true>(a, w, M, N, K, plan, sc, e, y, part, st);
        if (e.residual.p) return launch_linear_int8_out<T, kLinFinalMore, false>(a, w, M, N, K, plan, sc, e, y, part, st);
        return launch_linear_int8_out<T, kLinFinal, false>(a, w, M, N, K, plan, sc, e, y, part, st);
    }
    const dvdq_status s = launch_linear_int8_out<T, kLinPartial, false>(a, w, M, N, K, plan, sc, e, y, part, st);
    if (s != DVDQ_OK) return s;
    const int64_t ctas = ceil_div(M * ((N + 3) / 4), 256);
    return cuda_status(launch_after(linear_int8_join_kernel<T>, dim3((unsigned)(ctas < 148 * 8 ? ctas : 148 * 8)), dim3(256), 0, st, part,
                                    plan.part_rows * plan.part_pitch, (int)plan.part_pitch, plan.splits, M, (int)N, sc.a, sc.w,
                                    static_cast<const T*>(e.bias), static_cast<const T*>(e.residual.p), e.residual.ld, e.act,
                                    static_cast<T*>(const_cast<void*>(y.p)), y.ld));
}

}  // namespace dvdq
