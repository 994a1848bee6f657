// The linear layer in 16-bit floating point and its gradients, as one kernel of matrix products
//
//   D[m, n] = sum_k A[m, k] B[n, k]     forward   D = z = X W^T      A = X  [M, K],    B = W [N, K]
//                                       dX = dZ W                    A = dZ [M, N],    B = W^T
//                                       dW = dZ^T X                  A = dZ^T,         B = X^T
//
// A transposed operand is read where it lies: tcgen05 takes shared-memory tiles whose contiguous
// axis is the contracted one ("K-major") or the other one ("MN-major"), so nothing is transposed in memory.
//
// A CTA pair owns a tile of 256 rows x `bn` columns of D (bn = 32 .. 256, chosen per call: the smaller
// it is, the more tiles a small product has for the 74 pairs): tcgen05.mma.cta_group::2.kind::f16 256 x bn x 16,
// operands in shared memory (128-byte swizzle) in a ring of TMA-filled stages of 64 along k, two fp32
// accumulators in tensor memory, so that the epilogue of a tile runs under the next tile's products.
// Roles per CTA: warps 0 and 2 TMA producers of A and B; warp 1 (leader CTA) issues the products; warps 4-11 epilogue, two
// per tensor-memory lane quarter, every other block of 32 (or 64) columns each: bias, activation, residual in fp32, ONE
// rounding (fp32 outputs would double what is written), and TMA stores; the residual's blocks come by TMA, up to three ahead.
//
// What bounds it: the tensor pipe on layers of thousands of tokens (32760 x 5120 -> 13824 with GELU: 3.1-3.5 ms, 1.32-1.5
// PFLOP/s under the power cap; cold 3.3-3.8 ms, 2.9-4.3 the bare product of the vendor's library in the same run; tensor pipe
// 98 % active in the gradients, 84 % at 32760 x 1536 -> 1536, where it takes 105-145 us with the clock); with few tokens, streaming
// W; with a contraction of a few k-blocks, the copies of outputs and residuals (32760 x 64 -> 1536: 27 us, with a residual 50 for 205 MB).
// Products with fewer tiles than CTA pairs are cut along k (`splits`): each piece writes its fp32 sums,
// and a second kernel adds the pieces in a fixed order and does the epilogue (no atomics).
#pragma once

#include "block_common.cuh"
#include "host_setup.cuh"

namespace dvdq {

constexpr int kLinBK = 64;                    // elements of k per stage: one 128-byte swizzle row
constexpr int kLinTile = 256;                 // rows of a pair's tile, and most columns
constexpr int kLinEpiWarps = 8, kLinFirstEpi = 4;
constexpr int kLinThreads = (kLinFirstEpi + kLinEpiWarps) * 32;
constexpr int kLinPairs = 74;                 // CTA pairs of a B200 (148 SMs): what the split along k is planned for

// What the kernel writes: the output; the output from a residual, or z as well; fp32 pieces.
enum LinOut { kLinFinal = 0, kLinFinalMore = 1, kLinPartial = 2 };

template <int OUT, bool WIDE>
struct LinSmem {
    // a residual that comes early, and z, take two more blocks per epilogue warp, and 32 KB of the ring
    static constexpr int kRing = (OUT == kLinFinalMore ? (WIDE ? 3 : 5) : (WIDE ? 5 : 6)) * 32768;
    static constexpr int kMaxStages = 16;                   // a stage is 32 KB at most; narrow tiles and few rows take less
    static constexpr int kBufs = OUT == kLinFinalMore ? 4 : 2;
    static constexpr int kCols = WIDE ? 64 : 32;            // of an epilogue block
    static constexpr int kBuf = 32 * kCols * 2;             // 32 x kCols outputs; fp32 partials use two as one
    static constexpr int kBufOff = kRing;
    static constexpr int kBiasOff = kBufOff + kLinEpiWarps * kBufs * kBuf;
    static constexpr int kBarOff = kBiasOff + kLinEpiWarps * 32 * 4;
    static constexpr int kNumBars = 2 * kMaxStages + 5 + 4 * kLinEpiWarps;
    static constexpr int kMiscOff = kBarOff + kNumBars * 8;
    static constexpr int kTotal = kMiscOff + 16 + 1024;
    static_assert(kTotal <= 232448, "more than the 227 KB of shared memory a CTA can have");
};

struct LinArgs {
    int Md, Nd;             // rows and columns of D
    int bn;                 // columns of a tile: a multiple of 32 (of 64 where B is MN-major)
    int num_m, num_n;       // tiles
    int kblocks, splits;    // k-blocks of the contraction, pieces it is cut into
    int panel;              // column tiles walked together
    FastDiv by_splits, by_panel_tiles, by_panel, by_last;  // pieces; tiles of a panel; columns of a panel, of the last one
    int part_rows;          // rows of one piece in the partial buffer
    int a_bytes;            // of one CTA's half of A's stage
    int low;                // dz as A in two parts that add up: row m + low of dz is the second part of row m (0: one part)
    int stages, stage, b_off;  // of the operand ring: how many, bytes per CTA of each, where B's half begins in it
    int act, has_residual, has_z;
    const void* bias;
};

// mbar_wait by a converged warp of which one lane polls (32 polling lanes of eight warps keep the shared memory's
// barrier unit busy, and the producer and the issuer of products wait for it); the others look once, when it is over.
__device__ __forceinline__ bool mbar_wait_one_lane(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t wait_id) {
    bool ok = true;
    if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, abort_flag, wait_id);
    ok = __shfl_sync(0xFFFFFFFFu, (int)ok, 0) != 0;
    return ok && __all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity));
}

// A walk through a ring of stages by one thread: visit(stage) for `n` stages in turn, after their barriers' phases.  The
// barriers of a deep ring (narrow tiles) are looked at in pairs, which overlaps their latencies: with one look per stage
// these loops, not the tensor pipe, were the bound of tiles narrower than 192 columns (0.19 us a k-block; 0.145 in
// pairs).  A ring of six 32 KB stages has none to spare for pairs (4096^3: 95 us with, 93 without).
constexpr int kLinPairStages = 7;
struct LinRing {
    uint32_t bars, stages, st = 0, parity;
    __device__ __forceinline__ LinRing(uint32_t first_bar, uint32_t n, uint32_t p) : bars(first_bar), stages(n), parity(p) {}
    __device__ __forceinline__ void step() {
        if (++st == stages) { st = 0; parity ^= 1u; }
    }
    template <typename Visit>
    __device__ __forceinline__ bool walk(int n, volatile uint32_t* abort_flag, uint32_t wait_id, Visit visit) {
        for (const bool pairs = stages > kLinPairStages; n > 0;) {
            const bool two = pairs && n > 1, wraps = st + 1 == stages;
            const uint32_t bar0 = bars + 8u * st, bar1 = wraps ? bars : bar0 + 8u, parity1 = wraps ? parity ^ 1u : parity;
            const bool first = mbar_try_wait(bar0, parity), second = !two || mbar_try_wait(bar1, parity1);
            if (!first && !mbar_wait(bar0, parity, abort_flag, wait_id)) return false;
            if (!second && !mbar_wait(bar1, parity1, abort_flag, wait_id)) return false;
            visit(st);
            step();
            if (two) {
                visit(st);
                step();
            }
            n -= two ? 2 : 1;
        }
        return true;
    }
};

// Item -> tile and piece.  Tiles are walked in panels of `panel` column tiles, columns fastest, so that the
// tiles in flight together share rows and columns of the operands in L2; the pieces of a tile are neighbours.
__device__ __forceinline__ void lin_item(const LinArgs& A, int item, int& tm, int& tn, int& piece) {
    const int tile = (int)A.by_splits((uint32_t)item);
    piece = item - tile * A.splits;
    const int p = (int)A.by_panel_tiles((uint32_t)tile), r = tile - p * A.num_m * A.panel;
    const bool last = (p + 1) * A.panel >= A.num_n;
    const int w = last ? A.num_n - p * A.panel : A.panel;
    tm = (int)(last ? A.by_last((uint32_t)r) : A.by_panel((uint32_t)r));
    tn = p * A.panel + (r - tm * w);
}
__device__ __forceinline__ int2 lin_range(const LinArgs& A, int piece) {  // k-blocks of a piece: never empty
    const int q = A.kblocks / A.splits, rest = A.kblocks - q * A.splits;
    const int b = piece * q + min(piece, rest);
    return make_int2(b, b + q + (piece < rest ? 1 : 0));
}

// Descriptor of a 64-wide MN-major tile with the 128-byte swizzle: rows of k are 128 bytes, eight of
// them (1024 bytes) a swizzle atom; the next 64 columns are kLinBK rows = 8192 bytes further on.
__device__ __forceinline__ uint64_t umma_desc_sw128_mnmajor(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
    d |= (uint64_t)((kLinBK * 128) >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1u << 46;
    d |= (uint64_t)2u << 61;
    return d;
}
// Instruction descriptor for kind::f16: fp32 accumulator, both operands bf16 (or both fp16), which of them
// are MN-major, and the shape; n is added at run time.
__host__ __device__ constexpr uint32_t umma_idesc_f16(bool bf16, bool a_mn, bool b_mn, int m) {
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void tc_mma_f16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// This CTA's `width` rows (or columns) of an operand's stage: one box of 64 x width, or boxes of 64 columns x 64
// rows of k (the last one may be wider than needed); all count their bytes on the leader's barrier.
__device__ __forceinline__ void lin_load(bool mn, uint32_t dst, const CUtensorMap* m, uint32_t bar, int k0, int r0, int width) {
    if (!mn) {
        tma_load_2d_pair(dst, m, bar, k0, r0);
    } else {
        tma_load_2d_pair(dst, m, bar, r0, k0);
        if (width > 64) tma_load_2d_pair(dst + kLinBK * 128, m, bar, r0 + 64, k0);
    }
}
__host__ __device__ constexpr uint32_t lin_bytes(bool mn, int width) { return (uint32_t)(mn ? (width + 63) / 64 * (kLinBK * 128) : width * kLinBK * 2); }

// One product's operands and where it goes.
struct LinMaps {
    CUtensorMap a, b, y;
};

// Walks the 32 x COLS blocks of one epilogue warp, tile after tile.
template <int COLS>
struct LinBlocks {
    int item, c = -1, blocks = 0, row0 = 0, col0 = 0, piece = 0;
    bool more = true;
    __device__ __forceinline__ void tile(const LinArgs& A, int rows_from, int half) {
        int tm, tn;
        lin_item(A, item, tm, tn, piece);
        row0 = tm * kLinTile + rows_from;
        col0 = tn * A.bn + half * COLS;
        const int width = min(A.bn, A.Nd - tn * A.bn) - half * COLS;
        blocks = row0 < A.Md && width > 0 ? (width + 2 * COLS - 1) / (2 * COLS) : 0;  // those that lie in D: columns col0, col0 + 2 COLS, ...
    }
    // to the next block that lies in D
    __device__ __forceinline__ void next(const LinArgs& A, int items, int step, int rows_from, int half) {
        if (!more || (c >= 0 && ++c < blocks)) return;
        if (c < 0) c = 0;
        else item += step;
        for (; item < items; item += step) {
            tile(A, rows_from, half);
            c = 0;
            if (blocks > 0) return;
        }
        more = false;
    }
};

// TWO: dX and dW of a small layer in one launch: neither fills the pairs, so the first items of the grid are the tiles of
// one, the rest those of the other (each pair has one tile).  The first product's A is then K-major, the second's MN-major.
template <typename T, bool AMN_, bool BMN, int OUT, bool TWO, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinThreads, 1)
linear_kernel(const __grid_constant__ LinMaps maps1, const __grid_constant__ CUtensorMap tmR, const __grid_constant__ CUtensorMap tmZ,
              const __grid_constant__ LinArgs args1, const __grid_constant__ LinMaps maps2, const __grid_constant__ LinArgs args2) {
    const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    const int items1 = args1.num_m * args1.num_n * args1.splits;
    const bool second = TWO && pair >= items1;
    const LinMaps& maps = second ? maps2 : maps1;
    const LinArgs& A = second ? args2 : args1;
    const bool AMN = TWO ? second : AMN_;
    const int items = second ? args2.num_m * args2.num_n : items1;
    const int first_item = second ? pair - items1 : pair, item_step = TWO ? 1 << 30 : num_pairs;
    using S = LinSmem<OUT, WIDE>;
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
        for (int w = 0; w < 4 * kLinEpiWarps; ++w) mbar_init(res_full(0, w), 1);
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
        // ------------------------------------------------------------ TMA producers: warp 0 of A, warp 2 of B
        // (one thread that asks for both takes 460 clocks a k-block, as long as the products of a 256-wide tile)
        if (elect_one()) {
            const bool of_a = warp == 0;
            const CUtensorMap* map = of_a ? &maps.a : &maps.b;
            tma_prefetch_desc(map);
            const int bw = A.bn / 2;  // columns per CTA
            const uint32_t leader_full = map_to_cta(full(0), 0);
            LinRing ring(empty(0), ST, 1u);
            const uint32_t dst = sbase + (of_a ? 0 : A.b_off);
            bool ok = true;
            for (int item = first_item; ok && item < items; item += item_step) {
                int tm, tn, piece;
                lin_item(A, item, tm, tn, piece);
                const int2 kr = lin_range(A, piece);
                const int r0 = of_a ? tm * kLinTile + (int)rank * 128 : tn * A.bn + (int)rank * bw;
                // rows past D's last need no operand: whatever lies in their stage reaches only rows that are not stored
                const bool needed = !of_a || r0 < A.Md;
                const uint32_t bytes = of_a ? A.a_bytes * (tm * kLinTile + 128 < A.Md ? 2u : 1u) : 2 * lin_bytes(BMN, bw);
                int k0 = kr.x * kLinBK;
                ok = ring.walk(kr.y - kr.x, abort_flag, kWaitWideEmpty, [&](uint32_t st) {
                    if (rank == 0) mbar_arrive_expect_tx(full(st), bytes);
                    if (needed) {
                        lin_load(of_a ? AMN : BMN, dst + st * stage, map, leader_full + 8u * st, k0, r0, of_a ? 128 : bw);
                        if (BMN && of_a && A.low > 0)
                            lin_load(AMN, dst + st * stage + A.a_bytes / 2, map, leader_full + 8u * st, AMN ? k0 + A.low : k0, AMN ? r0 : r0 + A.low, 128);
                    }
                    k0 += kLinBK;
                });
            }
            if (!ok)  // giving up after seconds of waiting: a bounded pause covers the last copies
                for (int it = 0; it < 64; ++it) __nanosleep(1000);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products (leader CTA only)
        // One thread runs the whole loop: a warp-wide wait for every k-block costs more than the products of a narrow tile.
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = umma_idesc_f16(IsBf16<T>::value, AMN, BMN, kLinTile) | ((uint32_t)(A.bn >> 3) << 17);
            // 16 elements along k: 32 bytes inside a K-major swizzle row, two atoms of an MN-major tile
            const uint32_t step_a = AMN ? 2048 / 16 : 2;
            constexpr uint32_t kStepB = BMN ? 2048 / 16 : 2;
            const uint64_t ad0 = AMN ? umma_desc_sw128_mnmajor(sbase) : umma_desc_sw128_kmajor(sbase);
            const uint64_t ad1 = ad0 + (uint32_t)(A.a_bytes / 2 >> 4);  // the second part
            const uint64_t bd0 = BMN ? umma_desc_sw128_mnmajor(sbase + A.b_off) : umma_desc_sw128_kmajor(sbase + A.b_off);
            LinRing ring(full(0), ST, 0u);
            uint32_t lt = 0;
            bool ok = true;
            for (int item = first_item; ok && item < items; item += item_step, ++lt) {
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
                    for (int k = 0; k < kLinBK / 16; ++k) {
                        tc_mma_f16_pair(d_tmem, ad0 + (off + step_a * k), bd0 + (off + kStepB * k), idesc, add);
                        add = 1u;
                    }
                    if (BMN && A.low > 0) {
#pragma unroll
                        for (int k = 0; k < kLinBK / 16; ++k)
                            tc_mma_f16_pair(d_tmem, ad1 + (off + step_a * k), bd0 + (off + kStepB * k), idesc, 1u);
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
        const int q = warp & 3, half = ew >> 2;  // tensor-memory lane quarter; which of every two 32-column blocks
        const uint32_t buf0 = sbase + S::kBufOff + ew * (S::kBufs * S::kBuf);
        const uint32_t c_bias = sbase + S::kBiasOff + ew * 128;
        const bool residual = OUT == kLinFinalMore && A.has_residual, with_z = OUT == kLinFinalMore && A.has_z;
        const bool with_bias = OUT != kLinPartial && A.bias != nullptr;
        const T* bias = static_cast<const T*>(A.bias);
        // output blocks take turns in `turns` buffers; z has the last one to itself
        const uint32_t turns = OUT == kLinFinalMore ? (with_z ? 3u : 4u) : 2u;
        if (lane == 0) tma_prefetch_desc(&maps.y);
        const int rows_from = (int)rank * 128 + q * 32;
        uint32_t lt = 0;
        uint32_t buf_i = 0;               // the next block's buffer
        uint32_t rask = 0, rphase = 0;    // the next residual's buffer; the parity to wait for, a bit per buffer
        uint32_t pending = 0;             // residual blocks asked for and not taken
        bool ok = true;
        // Asks for the residual of the next block ahead, into the buffer whose turn it is: at the start all but one, then one after
        // each block, when that block's store is the newest and the store that used the buffer is the one before it.
        LinBlocks<S::kCols> ahead;
        ahead.item = first_item;
        auto ask = [&]() {
            ahead.next(A, items, item_step, rows_from, half);
            if (!ahead.more) return;
            if (lane == 0) {
                if (with_z) tma_store_wait_read<2>();
                else tma_store_wait_read<1>();
                mbar_arrive_expect_tx(res_full(ew, rask), S::kBuf);
                tma_load_2d(buf0 + rask * S::kBuf, &tmR, res_full(ew, rask), ahead.col0 + ahead.c * (2 * S::kCols), ahead.row0);
            }
            rask = rask + 1 == turns ? 0u : rask + 1;
            ++pending;
        };
        if (residual)
            for (uint32_t i = 1; i < turns; ++i) ask();
        LinBlocks<S::kCols> b;
        for (b.item = first_item; ok && b.item < items; b.item += item_step, ++lt) {
            b.tile(A, rows_from, half);
            const uint32_t a = lt & 1u, aph = (lt >> 1) & 1u;
            const int row0 = b.row0, col0 = b.col0, blocks = b.blocks, piece = b.piece;
            float b_next = 0.f;
            if (with_bias && blocks > 0 && col0 + lane < A.Nd) b_next = to_f32(bias[col0 + lane]);
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
                    const uint32_t buf = buf0 + buf_i * S::kBuf, zb = buf0 + 3 * S::kBuf;
                    const int block_col = col0 + c * (2 * S::kCols);
#pragma unroll
                    for (int h = 0; h < S::kCols / 32; ++h) {  // 32 columns at a time
                        uint32_t r[32];
                        __syncwarp();
                        tmem_ld_32x32(tmem_base + a * kLinTile + half * S::kCols + c * (2 * S::kCols) + h * 32 + ((uint32_t)(q * 32) << 16), r);
                        // the block's output buffer (without a residual: else ask() has waited for it) and z's: free once all but the
                        // newest store have been read
                        if (h == 0 && (!residual || with_z) && lane == 0) tma_store_wait_read<1>();
                        if (with_bias) sts32f(c_bias + 4 * lane, b_next);
                        __syncwarp();
                        if (with_bias) {
                            const int next = h + 1 < S::kCols / 32 ? block_col + (h + 1) * 32 : c + 1 < blocks ? block_col + 2 * S::kCols : A.Nd;
                            b_next = next + lane < A.Nd ? to_f32(bias[next + lane]) : 0.f;
                        }
                        if (residual && h == 0) {
                            ok = mbar_wait_one_lane(res_full(ew, buf_i), (rphase >> buf_i) & 1u, abort_flag, kWaitPackedFull);
                            if (!ok) break;
                            rphase ^= 1u << buf_i;
                            --pending;
                        }
                        tmem_ld_wait();
                        uint64_t v[16];  // pairs of columns
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = f2_pack(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        if (with_bias) {
#pragma unroll
                            for (int j = 0; j < 16; j += 2) {
                                const float4 f = lds128f(c_bias + 8 * j);
                                v[j] = f2_add(v[j], f2_pack(f.x, f.y));
                                v[j + 1] = f2_add(v[j + 1], f2_pack(f.z, f.w));
                            }
                        }
                        // what the swizzled TMA copies use: rows of 64 bytes, 16-byte chunk index XORed with (row / 2) % 4, or of
                        // 128 bytes, with row % 8
                        auto at = [&](uint32_t base, int j) {
                            return WIDE ? base + lane * 128 + (((h * 4 + j) ^ (lane & 7)) << 4) : base + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4);
                        };
                        auto put = [&](uint32_t base, int j) {  // columns 8 j .. 8 j + 7
                            uint32_t w[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                float lo, hi;
                                f2_unpack(v[4 * j + t], lo, hi);
                                w[t] = pack2<T>(lo, hi);
                            }
                            sts128(at(base, j), w[0], w[1], w[2], w[3]);
                        };
                        if (with_z) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) put(zb, j);
                            if (h + 1 == S::kCols / 32) {
                                fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0) {
                                    tma_store_2d(&tmZ, zb, block_col, row0);
                                    tma_store_commit();
                                }
                            }
                        }
                        if (A.act == DVDQ_ACT_GELU_TANH) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = act_value2<DVDQ_ACT_GELU_TANH>(v[j]);
                        } else if (A.act == DVDQ_ACT_SILU) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = act_value2<DVDQ_ACT_SILU>(v[j]);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (residual) {
                                const uint4 w = lds128(at(buf, j));
                                const Pairs<8> f = widen2<T, 8>(*reinterpret_cast<const Vec<T, 8>*>(&w));
#pragma unroll
                                for (int t = 0; t < 4; ++t) v[4 * j + t] = f2_add(v[4 * j + t], f.p[t]);
                            }
                            put(buf, j);
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

// y = act(sum of the pieces + bias) + residual, four columns per thread; pieces are added in order.
template <typename T>
__global__ void __launch_bounds__(256)
linear_join_kernel(const float* __restrict__ part, int64_t piece_floats, int pitch, int splits, int64_t Md, int Nd, const T* __restrict__ bias,
                   const T* residual, int64_t ldr, int act, T* y, int64_t ldy, T* z, int64_t ldz) {
    wait_predecessor();
    release_successor();
    const int quads = (Nd + 3) >> 2;
    const int64_t total = Md * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int n = (int)(i - m * quads) * 4;
        const float* p = part + m * pitch + n;
        float4 s = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
        for (int k = 1; k < splits; ++k) {
            const float4 t = *reinterpret_cast<const float4*>(p + k * piece_floats);
            s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
        }
        float v[4] = {s.x, s.y, s.z, s.w};
        const int here = Nd - n < 4 ? Nd - n : 4;
        if (bias) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < here) v[j] += to_f32(bias[n + j]);
        }
        if (here == 4) {  // rows start on 16 bytes and n is a multiple of 4: 8-byte accesses
            if (z) *reinterpret_cast<uint2*>(z + m * ldz + n) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = act_value_rt(act, v[j]);
            if (residual) {
                const uint2 w = *reinterpret_cast<const uint2*>(residual + m * ldr + n);
                const float2 f0 = unpack2<T>(w.x), f1 = unpack2<T>(w.y);
                v[0] += f0.x; v[1] += f0.y; v[2] += f1.x; v[3] += f1.y;
            }
            *reinterpret_cast<uint2*>(y + m * ldy + n) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
        } else {
            for (int j = 0; j < here; ++j) {
                if (z) z[m * ldz + n + j] = from_f32<T>(v[j]);
                float o = act_value_rt(act, v[j]);
                if (residual) o += to_f32(residual[m * ldr + n + j]);
                y[m * ldy + n + j] = from_f32<T>(o);
            }
        }
    }
}

// ------------------------------------------------------------------ backward: dz and its column sums

// dz = dy act'(z) in fp32, rounded once to the operands' type for the tensor cores (an fp32 dz would cost
// the two products half of their rate or more); the bias's gradient sums the unrounded values.
// low > 0 (so few values that their roundings would not average out): dz goes into two parts (split_in_two), the second to row
// m + low, and dX and dW are formed from both, in one accumulator.  Where dW's last k-block reaches past row M it meets rows
// of the second part, but x has zeros there and a second part is finite.
// A CTA takes 256 columns (8 per thread, 32 threads side by side, 8 rows at a time) of one chunk of
// rows and writes their sums; linear_colsum_kernel adds the chunks.  Bound by its bytes: 32760 x 8960 with GELU 276 us, 6.4 TB/s.  act = none: dz is dy itself, only sums.
constexpr int kLinDzCols = 256, kLinDzDepth = 5;

__device__ __forceinline__ __nv_bfloat16 toward_zero(float d, __nv_bfloat16) { return __float2bfloat16_rz(d); }
__device__ __forceinline__ __half toward_zero(float d, __half) { return __float2half_rz(d); }
// d = first + second up to the rounding of `second`.  Both have d's sign and neither is zero (unless d is zero, or the type's smallest
// number or less), so that beside an infinity in the other operand the two products are the same infinity, not NaN: `first` is d
// toward zero, and one step further where that is d itself.  An infinite d: the second part is 1 of its sign.
template <typename T>
__device__ __forceinline__ void split_in_two(float d, T& first, T& second) {
    first = toward_zero(d, T());
    second = from_f32<T>(isfinite(d) ? d - to_f32(first) : d != d ? 0.0f : copysignf(1.0f, d));
    uint16_t bits;
    memcpy(&bits, &first, 2);
    if (to_f32(second) == 0.0f && (bits & 0x7FFF) > 1 && isfinite(d)) {
        --bits;
        memcpy(&first, &bits, 2);
        second = from_f32<T>(d - to_f32(first));
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kStreamThreads, 4)
linear_dz_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ z, int64_t ldz, int64_t M, int N, int64_t rows,
                 T* __restrict__ dz, int64_t lddz, int low, float* __restrict__ sums) {
    constexpr bool kAct = ACT != DVDQ_ACT_NONE;
    wait_predecessor();
    release_successor();
    __shared__ __align__(16) uint8_t raw[kStreamThreads * 16 * kLinDzDepth * (kAct ? 2 : 1)];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int n = blockIdx.x * kLinDzCols + tx * 8;
    const int64_t m0 = (int64_t)blockIdx.y * rows, m1 = m0 + rows < M ? m0 + rows : M;
    Pairs<8> s;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.p[i] = 0ull;
    const int here = N - n < 8 ? N - n : 8;
    const int64_t mt = m0 + ty;
    const int count = here > 0 && mt < m1 ? (int)((m1 - mt + 7) / 8) : 0;
    if (count > 0) {
        T* out = dz + mt * lddz + n;
        auto row = [&](const Vec<T, 8>& dv, const Vec<T, 8>& zv) {
            Pairs<8> d = widen2<T, 8>(dv);
            const Pairs<8> zz = widen2<T, 8>(zv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (kAct) d.p[i] = f2_mul(d.p[i], act_slope2<ACT>(zz.p[i]));
                s.p[i] = f2_add(s.p[i], d.p[i]);
            }
            if (kAct) {
                if (low > 0) {
                    Vec<T, 8> first, second;
#pragma unroll
                    for (int i = 0; i < 8; ++i) split_in_two(d.get(i), first.e[i], second.e[i]);
                    *reinterpret_cast<Vec<T, 8>*>(out) = first;
                    *reinterpret_cast<Vec<T, 8>*>(out + low * lddz) = second;
                } else {
                    *reinterpret_cast<Vec<T, 8>*>(out) = narrow2<T, 8>(d);
                }
                out += 8 * lddz;
            }
        };
        const T *pd = dy + mt * lddy + n, *pz = z + mt * ldz + n;
        // Past the last column a row's 16 bytes hold what lies between it and the next row: read, but used by nobody (dz
        // is the workspace's, whole groups may be written).  The matrix's very last row has no next row: element by element.
        const int streamed = here < 8 && mt + (int64_t)(count - 1) * 8 == M - 1 ? count - 1 : count;
        if constexpr (kAct) walk<kLinDzDepth, 2, T, 8>(raw, streamed, pd, 8 * lddy, pz, 8 * ldz, row);
        else walk<kLinDzDepth, 1, T, 8>(raw, streamed, pd, 8 * lddy, pd, 0, [&](const Vec<T, 8>& dv) { row(dv, dv); });
        if (streamed < count) {
            Vec<T, 8> d, zz;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d.e[j] = j < here ? dy[(M - 1) * lddy + n + j] : from_f32<T>(0.f);
                zz.e[j] = kAct && j < here ? z[(M - 1) * ldz + n + j] : from_f32<T>(0.f);
            }
            row(d, zz);
        }
    }
    if (sums) {
        __syncthreads();  // the ring's memory becomes the sums'
        float* sh = reinterpret_cast<float*>(raw);
#pragma unroll
        for (int j = 0; j < 8; ++j) sh[ty * kLinDzCols + tx * 8 + j] = s.get(j);
        __syncthreads();
        const int c = blockIdx.x * kLinDzCols + threadIdx.x;
        if (c < N) {
            float t = 0.f;
#pragma unroll
            for (int y = 0; y < 8; ++y) t += sh[y * kLinDzCols + threadIdx.x];
            sums[(int64_t)blockIdx.y * N + c] = t;
        }
    }
}

static __global__ void __launch_bounds__(256) linear_colsum_kernel(const float* __restrict__ sums, int chunks, int N, float* __restrict__ out) {
    wait_predecessor();
    release_successor();
    __shared__ double sh[8][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    double t = 0.0;
    if (c < N)
        for (int i = w; i < chunks; i += 8) t += sums[(int64_t)i * N + c];
    sh[w][lane] = t;
    __syncthreads();
    if (w == 0 && c < N) {
#pragma unroll
        for (int y = 1; y < 8; ++y) t += sh[y][lane];
        out[c] = (float)t;
    }
}

// ------------------------------------------------------------------ host side

// Epilogue blocks of 32 x 64 instead of 32 x 32 outputs: half as many TMA copies, at the price of operand stages.  Worth it where
// a tile has few products to hide its copies under: up to 4 k-blocks (32760 x 256 -> 1536: 30.9 us, 32.5 in narrow blocks; 512:
// 46.5 and 44.5), and 8 with a residual or z (512 -> 1536 with residual: 63 us, 72 in narrow blocks; 256: 54 and 66; 768: 82 and 80).
constexpr int kLinWide = 4, kLinWideMore = 8;

struct LinPlan {
    int bn, splits;
    int64_t part_rows, part_pitch, part_bytes;
};

// Tile width and pieces along k, from the sizes alone, by an estimate in microseconds fitted to measurements
// (M x N x K = 509 x 5120 x 4096, 32760 x 1536 x 1536, 4096^3, 200 x 3072 x 3072, 16 x 5120 x 5120, every width, 1 to 8
// pieces): a k-block of a 256-row tile takes a pair 0.345 us per 256 columns of products, but at least what the
// loops around it take: 0.15 us + 0.6 ns per column with a deep ring, 0.135 us + 0.83 ns with a shallow one; all of it
// at least the time of reading both operands at 6 TB/s; a tile's epilogue 0.5 + 2 us per 256 columns, hidden under the
// next tile's products if there is one; 2 us to fill the ring.  Pieces cost a second launch (2.5 us) and writing and
// reading their fp32 sums in L2 (about 8 TB/s).  The estimate knows nothing of the row pitch or of L2's traffic; it compares plans
// and does not predict: 509 x 5120 x 4096 is 18 us to it and 24-27 in fact, 34 with rows of 8208 bytes.
// `step`: 32, or 64 where B is MN-major (its shared-memory tiles are 64 columns wide).
// Rows of A that a CTA loads for its half of a tile: all 128, or (one tile, one CTA with rows) those that exist.
inline int lin_a_rows(int64_t Md) { return Md < 128 ? (int)align_up(Md, 8) : 128; }

// The estimate for one wave (or `waves`) of pieces of `kblocks`.
inline double lin_cost(int64_t Md, int bn, int64_t kblocks, int64_t waves, double memory) {
    const bool deep = LinSmem<kLinFinal, false>::kRing / ((lin_a_rows(Md) + bn / 2) * kLinBK * 2) > kLinPairStages;
    const double products = 0.345 * bn / 256.0, loops = deep ? 0.15 + 0.0006 * bn : 0.135 + 0.00083 * bn;
    const double t_epi = 0.5 + 2.0 * bn / 256.0, item = (double)kblocks * (products > loops ? products : loops);
    const double cost = (double)waves * (item > t_epi ? item : t_epi);
    return (cost < memory ? memory : cost) + 2.0 + t_epi;
}
inline double lin_memory_time(int64_t Md, int64_t Nd, int64_t Kc) { return ((double)Md + Nd) * Kc * 2.0 / 6.0e6; }

// per_piece: what each piece costs beyond that.
inline LinPlan lin_plan(int64_t Md, int64_t Nd, int64_t Kc, int step, double* estimate = nullptr, double per_piece = 0.0) {
    const int64_t kb = ceil_div(Kc, kLinBK), num_m = ceil_div(Md, kLinTile);
    LinPlan p;
    p.bn = kLinTile;
    p.splits = 1;
    p.part_rows = align_up(Md, 32);
    p.part_pitch = align_up(Nd, 4);
    double best = 1e300;
    for (int bn = kLinTile; bn >= 32 && bn % step == 0; bn -= step) {
        const int64_t tiles = num_m * ceil_div(Nd, bn);
        for (int64_t s = 1; s <= 32 && s <= kb; ++s) {
            if (s > 1 && (tiles * s > 4 * kLinPairs || s * p.part_rows * p.part_pitch * 4 > ((int64_t)256 << 20))) break;
            double cost = lin_cost(Md, bn, ceil_div(kb, s), ceil_div(tiles * s, kLinPairs), lin_memory_time(Md, Nd, Kc));
            if (s > 1) cost += 2.5 + s * per_piece + (double)s * Md * Nd * 8.0 / 8.0e6;
            if (cost < best * 0.97) { best = cost; p.bn = bn; p.splits = (int)s; }  // a wider tile reads less: prefer it when near
        }
    }
    if (estimate) *estimate = best;
    p.part_bytes = p.splits > 1 ? align_up(p.splits * p.part_rows * p.part_pitch * 4, 256) : 0;
    return p;
}

// dX [M, K] (contraction N) and dW [N, K] (contraction M) side by side: the plans, or false where their tiles do not fit the
// pairs together or one after the other (estimates e1 and e2) is estimated to be as fast (a launch of its own: 2 us).
inline bool lin_plan_two(int64_t M, int64_t N, int64_t K, double e1, double e2, LinPlan* dx, LinPlan* dw) {
    double best = 1e300;
    for (int b1 = kLinTile; b1 >= 64; b1 -= 64)
        for (int b2 = kLinTile; b2 >= 64; b2 -= 64) {
            if (ceil_div(M, kLinTile) * ceil_div(K, b1) + ceil_div(N, kLinTile) * ceil_div(K, b2) > kLinPairs) continue;
            const double c1 = lin_cost(M, b1, ceil_div(N, kLinBK), 1, lin_memory_time(M, K, N)), c2 = lin_cost(N, b2, ceil_div(M, kLinBK), 1, lin_memory_time(N, K, M));
            const double cost = c1 > c2 ? c1 : c2;
            if (cost < best) { best = cost; dx->bn = b1; dw->bn = b2; }
        }
    dx->splits = dw->splits = 1;
    dx->part_rows = dx->part_pitch = dx->part_bytes = dw->part_rows = dw->part_pitch = dw->part_bytes = 0;  // no pieces
    return best < e1 + e2 + 2.0;
}

// A 16-bit matrix [rows, cols] with row pitch ld elements, tiles of box_rows x box_cols.
inline bool make_map16(CUtensorMap* tm, bool bf16, const void* base, int64_t rows, int64_t cols, int64_t ld, uint32_t box_cols,
                       uint32_t box_rows, CUtensorMapSwizzle swizzle) {
    PFN_encodeTiled enc = get_encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(tm, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(base), dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
           CUDA_SUCCESS;
}
inline bool make_map_f32(CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld) {
    PFN_encodeTiled enc = get_encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 4};
    const cuuint32_t box[2] = {32, 32};
    const cuuint32_t estr[2] = {1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct LinMatrix {
    const void* p;
    int64_t ld;
};
// The blocks in which the epilogue writes an output or reads the residual.
template <bool WIDE>
inline bool make_map_out(CUtensorMap* tm, bool bf16, const LinMatrix& y, int64_t rows, int64_t cols) {
    return make_map16(tm, bf16, y.p, rows, cols, y.ld, WIDE ? 64 : 32, 32, WIDE ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}
struct LinEpilogue {
    const void* bias;
    LinMatrix residual, z;
    int act;
};

// Tensor maps and arguments of one product; false if a map cannot be made.
template <typename T, bool AMN, bool BMN, int OUT, bool WIDE = false>
static bool make_linear(const LinMatrix& a, const LinMatrix& b, int64_t Md, int64_t Nd, int64_t Kc, const LinPlan& plan, const LinEpilogue& e,
                        const LinMatrix& y, float* part, int low, LinMaps* maps, LinArgs* A) {
    constexpr bool bf = IsBf16<T>::value != 0;
    using S = LinSmem<OUT, WIDE>;
    auto operand = [&](CUtensorMap* m, bool mn, const LinMatrix& x, int64_t rows, int64_t k, int more, int box) {  // `more` rows in memory
        return mn ? make_map16(m, bf, x.p, k + more, rows, x.ld, 64, kLinBK, CU_TENSOR_MAP_SWIZZLE_128B)
                  : make_map16(m, bf, x.p, rows + more, k, x.ld, kLinBK, (uint32_t)box, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    const int a_rows = AMN ? 128 : lin_a_rows(Md);
    if (!operand(&maps->a, AMN, a, Md, Kc, low, a_rows) || !operand(&maps->b, BMN, b, Nd, Kc, 0, plan.bn / 2)) return false;
    if (OUT == kLinPartial ? !make_map_f32(&maps->y, part, plan.splits * plan.part_rows, Nd, plan.part_pitch)
                           : !make_map_out<WIDE>(&maps->y, bf, y, Md, Nd))
        return false;
    A->Md = (int)Md;
    A->Nd = (int)Nd;
    A->num_m = (int)ceil_div(Md, kLinTile);
    A->bn = plan.bn;
    A->num_n = (int)ceil_div(Nd, plan.bn);
    A->kblocks = (int)ceil_div(Kc, kLinBK);
    A->splits = plan.splits;
    A->panel = 2048 / plan.bn < A->num_n ? 2048 / plan.bn : A->num_n;
    A->by_splits = FastDiv((uint32_t)A->splits);
    A->by_panel_tiles = FastDiv((uint32_t)(A->num_m * A->panel));
    A->by_panel = FastDiv((uint32_t)A->panel);
    A->by_last = FastDiv((uint32_t)(A->num_n - (A->num_n - 1) / A->panel * A->panel));
    A->part_rows = (int)plan.part_rows;
    A->low = low;
    A->a_bytes = (int)lin_bytes(AMN, a_rows) * (low > 0 ? 2 : 1);
    A->b_off = (int)align_up(A->a_bytes, 1024);  // swizzle atoms are 1024 bytes
    A->stage = A->b_off + (int)align_up(lin_bytes(BMN, plan.bn / 2), 1024);
    A->stages = S::kRing / A->stage < S::kMaxStages ? S::kRing / A->stage : S::kMaxStages;
    A->act = e.act;
    A->has_residual = OUT == kLinFinalMore && e.residual.p != nullptr;
    A->has_z = OUT == kLinFinalMore && e.z.p != nullptr;
    A->bias = OUT != kLinPartial ? e.bias : nullptr;
    return true;
}

template <typename T, bool AMN, bool BMN, int OUT, bool WIDE = false>
static dvdq_status launch_linear_out(const LinMatrix& a, const LinMatrix& b, int64_t Md, int64_t Nd, int64_t Kc, const LinPlan& plan,
                                     const LinEpilogue& e, const LinMatrix& y, float* part, int low, cudaStream_t st) {
    constexpr bool bf = IsBf16<T>::value != 0;
    using S = LinSmem<OUT, WIDE>;
    LinMaps maps;
    LinArgs A;
    if (!make_linear<T, AMN, BMN, OUT, WIDE>(a, b, Md, Nd, Kc, plan, e, y, part, low, &maps, &A)) return DVDQ_ERR_CUDA;
    CUtensorMap tmR = maps.y, tmZ = maps.y;  // where unused
    const bool fin = OUT == kLinFinalMore;
    if (fin && e.residual.p && !make_map_out<WIDE>(&tmR, bf, e.residual, Md, Nd)) return DVDQ_ERR_CUDA;
    if (fin && e.z.p && !make_map_out<WIDE>(&tmZ, bf, e.z, Md, Nd)) return DVDQ_ERR_CUDA;
    auto kern = linear_kernel<T, AMN, BMN, OUT, false, WIDE>;
    static PerDevice<int> cache;
    const int max_pairs = resident_pairs(cache, kern, kLinThreads, S::kTotal);
    if (max_pairs == 0) return DVDQ_ERR_CUDA;
    const int64_t items = (int64_t)A.num_m * A.num_n * A.splits;
    const unsigned pairs = (unsigned)(items < max_pairs ? items : max_pairs);
    return cuda_status(launch_after(kern, dim3(2 * pairs), dim3(kLinThreads), S::kTotal, st, maps, tmR, tmZ, A, maps, A));
}

template <typename T>
static dvdq_status launch_linear_join(const LinPlan& plan, int64_t Md, int64_t Nd, const LinEpilogue& e, const LinMatrix& y,
                                      const float* part, cudaStream_t st) {
    const int64_t ctas = ceil_div(Md * ((Nd + 3) / 4), 256);
    return cuda_status(launch_after(linear_join_kernel<T>, dim3((unsigned)(ctas < 148 * 8 ? ctas : 148 * 8)), dim3(256), 0, st, part,
                                    plan.part_rows * plan.part_pitch, (int)plan.part_pitch, plan.splits, Md, (int)Nd,
                                    static_cast<const T*>(e.bias), static_cast<const T*>(e.residual.p), e.residual.ld, e.act,
                                    static_cast<T*>(const_cast<void*>(y.p)), y.ld, static_cast<T*>(const_cast<void*>(e.z.p)), e.z.ld));
}

// D = A B^T with the epilogue e, into y; `part` holds plan.part_bytes.  low > 0: dz, which is A, comes in two parts.
template <typename T, bool AMN, bool BMN>
static dvdq_status launch_linear(const LinMatrix& a, const LinMatrix& b, int64_t Md, int64_t Nd, int64_t Kc, const LinPlan& plan,
                                 const LinEpilogue& e, const LinMatrix& y, float* part, int low, cudaStream_t st) {
    if (plan.splits == 1) {
        // only the forward product has a residual or stores its pre-activation
        const int64_t wide_kb = plan.bn % 128 == 0 ? ceil_div(Kc, kLinBK) : kLinWideMore + 1;  // a tile is whole blocks for both warps
        if constexpr (!AMN && !BMN) {
            if (e.z.p || e.residual.p)
                return wide_kb <= kLinWideMore ? launch_linear_out<T, AMN, BMN, kLinFinalMore, true>(a, b, Md, Nd, Kc, plan, e, y, part, low, st)
                                               : launch_linear_out<T, AMN, BMN, kLinFinalMore>(a, b, Md, Nd, Kc, plan, e, y, part, low, st);
        }
        if (wide_kb <= kLinWide) return launch_linear_out<T, AMN, BMN, kLinFinal, true>(a, b, Md, Nd, Kc, plan, e, y, part, low, st);
        return launch_linear_out<T, AMN, BMN, kLinFinal>(a, b, Md, Nd, Kc, plan, e, y, part, low, st);
    }
    const dvdq_status s = launch_linear_out<T, AMN, BMN, kLinPartial>(a, b, Md, Nd, Kc, plan, e, y, part, low, st);
    return s != DVDQ_OK ? s : launch_linear_join<T>(plan, Md, Nd, e, y, part, st);
}

// dX = dZ W and dW = dZ^T X of a small layer in one launch.
template <typename T>
static dvdq_status launch_linear_two(const LinMatrix& dz, const LinMatrix& x, const LinMatrix& w, int64_t M, int64_t N, int64_t K, const LinPlan& p1,
                                     const LinPlan& p2, const LinMatrix& dx, const LinMatrix& dw, int low, cudaStream_t st) {
    using S = LinSmem<kLinFinal, false>;
    LinMaps m1, m2;
    LinArgs a1, a2;
    const LinEpilogue none = {};
    if (!make_linear<T, false, true, kLinFinal>(dz, w, M, K, N, p1, none, dx, nullptr, low, &m1, &a1) ||
        !make_linear<T, true, true, kLinFinal>(dz, x, N, K, M, p2, none, dw, nullptr, low, &m2, &a2))
        return DVDQ_ERR_CUDA;
    auto kern = linear_kernel<T, false, true, kLinFinal, true, false>;
    static PerDevice<int> cache;
    if (resident_pairs(cache, kern, kLinThreads, S::kTotal) == 0) return DVDQ_ERR_CUDA;
    // each pair of the grid has one tile; pairs need not be resident together
    const unsigned pairs = (unsigned)(a1.num_m * a1.num_n + a2.num_m * a2.num_n);
    return cuda_status(launch_after(kern, dim3(2 * pairs), dim3(kLinThreads), S::kTotal, st, m1, m1.y, m1.y, a1, m2, a2));
}

}  // namespace dvdq
