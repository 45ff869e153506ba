// The token layers' product on the 5th-generation tensor cores: for every row r
// of a group and every output channel n
//   y[r][n] = (sum_k x[r][k] w[n][k]) s_w[n] s_x[r] + bias[n],
// x and w integers of 8 bits and the sum an exact integer. The groups are the
// experts of a mixture (row ranges read from device offsets) or one dense layer.
//
// sm_103a has no 8-bit integer tensor-core kind, so codes enter as fp16 (exact)
// and fp32 accumulators hold exact integers as long as no partial sum passes
// 2^24. The layout pass measured, per expert, up to which window length
// 128 sum |w| stays below that (trained weights: usually 4096 codes and more,
// where the blind bound allows 1024); past a window the epilogue warps add the
// accumulator into int32 registers while the next window fills the other one.
//
// The WEIGHTS are the M side (128 channels, the tensor-memory lanes) and the
// tokens the N side. So the weights stay one byte in memory - what a decode step
// is bound by - and are widened on their way into tensor memory, and a tile of
// few tokens wastes no lanes. The tokens' codes are fp16 in memory (few bytes
// next to the weights, or next to the arithmetic when there are many) and go
// from the copy engine to the tensor cores untouched.
//
// Roles of a CTA's 20 warps: 0 copies (8 KB weight blocks by bulk copy, token
// boxes by TMA), 1 issues the MMAs, 4-11 widen weights (two warpgroups, every
// other 64-code block: prmt puts code + 128 into the mantissa of 1024.0, one
// subtraction leaves the code), 12-19 are the epilogue (half of the tile's
// tokens per warpgroup). Two accumulators alternate, so the epilogue of one
// window or tile runs under the MMAs of the next.
//
// PAIR: two CTAs (one cluster) compute 256 channels x T tokens with
// cta_group::2; each widens its own 128 channels and holds half of the tokens,
// which halves the shared-memory traffic per product. The peer's token copies
// complete on the leader's barriers, whose MMAs read them. split > 1: the CTAs of a
// cluster share one tile's reduction and add their int32 sums through
// distributed shared memory (integers: the order does not matter). LOOSE: token
// codes of any format, pitch and alignment, brought in and widened by the
// widening warps (their next stage's pieces on the way while one is worked on)
// instead of by TMA.
//
// Bound by the tensor cores where rows are many (8192 x 4096 -> 16384: 557 us at
// 2070 MHz, 600 us once the power cap takes clocks away, the tensor pipe 0.89
// active), by the weights' bytes where they are few per expert (256 rows, 61
// experts of 2048 x 2048: 45.5 us, 5.7 TB/s), by latency in between (48 rows,
// 4096 -> 8192: 11.8 us against 5.1 us of bytes).
// Every wait is bounded, as in the other tensor-core kernels.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hatq_tc.h"
#include "hatq_tokens.h"

namespace hatq {
namespace {

using namespace tc;

constexpr int kThreads = 640;
// registers per thread of the five warpgroups: copies and MMAs, two of converters, two of the epilogue
constexpr int kLaunchRegs = 96;         // what __launch_bounds__ gives 640 threads
constexpr int kRegsIssue = 40;
constexpr int kRegShares = 472;         // of 5 * 96
constexpr int kMaxSplit = 4;           // CTAs that share a reduction at most
constexpr int kRasterN = 8;            // channel tiles that share a sweep over the token tiles

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_shared(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// The peer's arrival at the pair leader's barrier. What it announces is tensor memory alone, ordered by the tcgen05
// fences on both sides. A release at cluster scope here, which would speak for shared memory as well, costs a memory
// barrier per hand-off: 8192 x 4096 -> 16384 1142 us a call instead of 620.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// arrival at the leader's barrier that announces copies of `bytes` on their way to the peer's shared memory
__device__ __forceinline__ void mbar_expect_tx_remote(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// a box into this CTA's shared memory whose bytes complete on a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *tm, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
        "[%2];" ::"r"(dst),
        "l"(tm), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
// Whether the phase is over, without a wait. PAIR: with an acquire of what the other CTA of the pair (or its copies)
// announced.
template <bool PAIR>
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    return ok != 0;
}
// mbar_wait; PAIR: with that acquire, made when the phase is known to be over
template <bool PAIR>
__device__ __forceinline__ bool wait_acquire(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *err) {
    if (!mbar_wait(bar, parity, abort_flag, err)) return false;
    return !PAIR || mbar_test<PAIR>(bar, parity);
}
// without regard to the abort flag: before the CTA leaves, what it has in flight has to land
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - t0 < kWaitLimitCycles) {
    }
}

__device__ __forceinline__ int4 load_cluster(uint32_t addr) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
            "r"(a), "l"(b), "r"(idesc), "r"(acc)
            : "memory");
    else
        umma_f16_ts(d, a, b, idesc, acc);
}
// arrives at the barrier of this CTA (of a pair's CTAs in `ctas`) when the MMAs issued so far are done
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar, uint16_t ctas = 3) {
    if (PAIR)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"(ctas)
            : "memory");
    else
        umma_commit(bar);
}

__device__ __forceinline__ uint32_t prmt(uint32_t x, uint32_t y, uint32_t sel) {
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(y), "r"(sel));
    return d;
}
__device__ __forceinline__ uint32_t hsub2(uint32_t x, uint32_t y) {
    uint32_t d;
    asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y));
    return d;
}

// 16 codes of row r from k0 < k on as bytes, zeros behind k
__device__ __forceinline__ uint4 loose_codes(const LinearArgs &a, int r, int k0) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (a.format == HATQ_CODES_I8) {
        const int8_t *p = reinterpret_cast<const int8_t *>(a.x) + (long long)r * a.ldx + k0;
        if (k0 + 16 <= a.k) {
            const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p);
            if ((off & 15) == 0) return *reinterpret_cast<const uint4 *>(p);
            if ((off & 7) == 0) {
                const uint2 lo = reinterpret_cast<const uint2 *>(p)[0], hi = reinterpret_cast<const uint2 *>(p)[1];
                return make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
            if ((off & 3) == 0) {
                const uint32_t *q = reinterpret_cast<const uint32_t *>(p);
                return make_uint4(q[0], q[1], q[2], q[3]);
            }
        }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k0 + i < a.k) w[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    const __half *p = reinterpret_cast<const __half *>(a.x) + (long long)r * a.ldx + k0;
    uint32_t h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k0 + 16 <= a.k && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = reinterpret_cast<const uint32_t *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k0 + i < a.k) h[i >> 1] |= (uint32_t)__half_as_ushort(p[i]) << (16 * (i & 1));
    }
    v.x = narrow_codes(h[0], h[1]);
    v.y = narrow_codes(h[2], h[3]);
    v.z = narrow_codes(h[4], h[5]);
    v.w = narrow_codes(h[6], h[7]);
    return v;
}

// a warpgroup's share, from the launch's: fewer or more, each has its own instruction
template <int REGS> __device__ __forceinline__ void set_regs() {
    static_assert(REGS != kLaunchRegs && REGS % 8 == 0, "register share");
    if constexpr (REGS < kLaunchRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS));
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS));
}

__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
    uint32_t r;
    if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void put(void *y, int type, long long at, float v) {
    if (type == HATQ_BF16) reinterpret_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
    else if (type == HATQ_F16) reinterpret_cast<__half *>(y)[at] = __float2half_rn(v);
    else reinterpret_cast<float *>(y)[at] = v;
}

template <int T, bool PAIR, bool LOOSE>
struct Config {
    static constexpr int kCtas = PAIR ? 2 : 1;
    static constexpr int kRegsWiden = LOOSE ? 104 : 72, kRegsOut = LOOSE ? 112 : 144;
    static_assert(kRegsIssue + 2 * kRegsWiden + 2 * kRegsOut <= kRegShares && kRegShares <= 5 * kLaunchRegs, "register shares");
    static_assert(!(LOOSE && PAIR), "loose codes: single CTAs");
    // 64-code blocks per pipeline stage. The MMA warp's wait, fence and commit take about 300 cycles, so a stage
    // holds enough blocks for its MMAs to take longer: one block per stage cost 480 cycles a block at any tile width.
    static constexpr int kSub = T <= 64 ? 4 : 2;
    static constexpr int kXBytes = T / kCtas * 128;                    // one block's token codes
    static constexpr int kWOffset = kSub * kXBytes;
    static constexpr int kChunks = T * kSub * 4 / 256;                 // LOOSE: 16-code pieces of a stage per widening thread
    static constexpr int kStageBytes = kSub * (kXBytes + kBlockBytes);
    static constexpr int kStages = 202 * 1024 / kStageBytes;
    // Blocks per hand-off from the widening warps to the MMA warp and back: all of a stage, or one where the
    // accumulators leave room for four blocks only. Widening takes about 1000 cycles from a freed slot to the MMAs:
    // the MMAs of three other blocks cover that, those of one other stage (770 cycles) do not.
    static constexpr int kGroup = T > 128 ? 1 : kSub;
    static constexpr int kHands = kSub / kGroup;                       // hand-offs per stage
    static constexpr int kSlotCols = 32 * kGroup;                      // a widened block takes 32 columns
    static constexpr int kFree = (512 - 2 * T) / kSlotCols;
    static constexpr int kSlots = kFree < 8 ? kFree : 8;
    static constexpr int kWideWarps = (kGroup == 1 ? 4 : 8) * kCtas;   // one set widens a hand-off, or both
    static constexpr int kTables = ((4 * kMaxExperts + 1) * 4 + 15) & ~15;   // the experts' tables
    static constexpr int kSmem = 1024 + kStages * kStageBytes + 1024 + kTables + 8 * (T / 2) * 4;
    static_assert(T % 32 == 0 && T / kCtas % 8 == 0, "token tile");
    static_assert(kSlots >= 2 && (kGroup > 1 || kSlots % 2 == 0), "slots of a hand-off");
    static_assert(8 * (kStages * (3 + kHands) + kSlots + 5) + 12 <= 1024, "barriers");
    static_assert(kStages * kStageBytes >= T * 512, "the int32 sums of a split tile reuse the stages");
};

struct Tile {
    int e, row, rows, ch;              // expert, first row, rows of the tile, first channel tile
    // columns that are multiplied: an expert's last tile may hold few rows
    __device__ __forceinline__ int columns() const { return (rows + 31) & ~31; }
};

template <int T, bool PAIR, bool LOOSE>
__global__ void __launch_bounds__(kThreads, 1)
    linear_tc_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ LinearArgs a) {
    using C = Config<T, PAIR, LOOSE>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *bar_area = smem + C::kStages * C::kStageBytes;
    const uint32_t bar0 = smem_addr(bar_area);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (C::kStages + s); };
    auto wide = [&](int s, int h) { return bar0 + 8u * (2 * C::kStages + s * C::kHands + h); };
    auto slot_free = [&](int q) { return bar0 + 8u * (C::kStages * (2 + C::kHands) + q); };
    auto dfull = [&](int d) { return bar0 + 8u * (C::kStages * (2 + C::kHands) + C::kSlots + d); };
    auto dempty = [&](int d) { return bar0 + 8u * (C::kStages * (2 + C::kHands) + C::kSlots + 2 + d); };
    const uint32_t tail = bar0 + 8u * (C::kStages * (2 + C::kHands) + C::kSlots + 4);
    auto peer_full = [&](int s) { return tail + 8u * (1 + s); };        // in a pair's leader: the peer's token codes
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(bar_area + 8 * (C::kStages * (3 + C::kHands) + C::kSlots + 5));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    uint32_t *peer_issued = tmem_holder + 2;                            // in a pair's leader: stages that the peer asked for, plus one
    // per expert: token tiles before it, its rows, its exact window
    int *tile_start = reinterpret_cast<int *>(bar_area + 1024), *first_row = tile_start + kMaxExperts + 1,
        *end_row = first_row + kMaxExperts, *window_of = end_row + kMaxExperts;
    __shared__ int warp_sums[kThreads / 32], warp_tops[kThreads / 32];
    __shared__ int s_skip;

    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const bool clustered = PAIR || a.split > 1;
    const uint32_t rank = clustered ? cluster_rank() : 0u;
    const uint32_t in_pair = PAIR ? rank : 0u;
    const int part = PAIR ? 0 : (int)rank, parts = PAIR ? 1 : a.split;

    if (threadIdx.x == 0) {
        if (!LOOSE) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmX) : "memory");
        *abort_flag = 0;
        *peer_issued = 0;
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
            for (int h = 0; h < C::kHands; ++h) mbar_init(wide(s, h), C::kWideWarps + (PAIR && h == 0 ? 1 : 0));
            if (PAIR) mbar_init(peer_full(s), 1);
        }
        for (int q = 0; q < C::kSlots; ++q) mbar_init(slot_free(q), 1);
        mbar_init(tail, 1);
        for (int d = 0; d < 2; ++d) {
            mbar_init(dfull(d), 1);
            mbar_init(dempty(d), 8 * C::kCtas);
        }
        fence_barrier_init();
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_holder)),
                         "r"(512)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_holder)),
                         "r"(512)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    // a pair's barriers and tensor memory are there once every thread of both CTAs has come by
    if (PAIR) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const int pairs_n = (a.n_tiles + C::kCtas - 1) / C::kCtas;          // channel tiles of a cluster
    const int per = PAIR ? 2 : a.split;
    const int first = (int)blockIdx.x / per, step = (int)gridDim.x / per;
    // this CTA's blocks of the reduction, whole stages but for the last
    const int units = (a.kb + C::kSub - 1) / C::kSub;
    const int kb0 = (int)((long long)units * part / parts) * C::kSub;
    const int kb1 = min((int)((long long)units * (part + 1) / parts) * C::kSub, a.kb);

    // A CTA's tiles come in order, so each role walks the experts along with them. Within an expert: all its token
    // tiles under kRasterN channel tiles, then the next channel tiles, so that weights and codes are taken from L2.
    int expert = 0;
    auto decode = [&](int t) {
        while (tile_start[expert + 1] * pairs_n <= t) ++expert;
        const int tokens = tile_start[expert + 1] - tile_start[expert];
        const int local = t - tile_start[expert] * pairs_n;
        const int sweep = local / (kRasterN * tokens), rest = local - sweep * kRasterN * tokens;
        const int width = min(kRasterN, pairs_n - sweep * kRasterN);
        const int mt = rest / width;
        Tile tile;
        tile.e = expert;
        tile.row = first_row[expert] + mt * T;
        tile.ch = (sweep * kRasterN + rest - mt * width) * C::kCtas;
        tile.rows = min(T, end_row[expert] - tile.row);
        return tile;
    };
    // copies of the stage that begins at block b
    const uint32_t stage0 = smem_addr(smem);
    auto copy_stage = [&](const Tile &tile, int b, int s) {
        // a pair's second half may lie behind the last channel tile: any block does, nothing of it is stored
        const int ct = min(tile.ch + (int)in_pair, a.n_tiles - 1);
        const uint8_t *w = a.w + (((long long)tile.e * a.n_tiles + ct) * a.kb + b) * kBlockBytes;
        const int row = tile.row + (int)in_pair * (tile.columns() / 2);              // a pair's second half of the tokens
        if (elect_one()) {
            const uint32_t st = stage0 + (uint32_t)(s * C::kStageBytes);
            const int blocks = min(C::kSub, kb1 - b);
            // The leader's MMAs read the peer's token codes, so those complete on the leader's barrier.
            const bool here = !LOOSE && in_pair == 0;
            mbar_expect_tx(full(s), (uint32_t)(blocks * (here ? C::kXBytes + kBlockBytes : kBlockBytes)));
            bulk_load(st + C::kWOffset, w, (uint32_t)(blocks * kBlockBytes), full(s));
            if (here) {
#pragma unroll
                for (int q = 0; q < C::kSub; ++q)
                    if (q < blocks) tma_load_2d(st + q * C::kXBytes, &tmX, full(s), (b + q) * 64, row);
            } else if (PAIR) {
                const uint32_t bar = map_shared(peer_full(s), 0);
                mbar_expect_tx_remote(bar, (uint32_t)(blocks * C::kXBytes));
#pragma unroll
                for (int q = 0; q < C::kSub; ++q)
                    if (q < blocks) tma_load_2d_pair(st + q * C::kXBytes, &tmX, bar, (b + q) * 64, row);
            }
        }
        __syncwarp();
    };

    after_prior_kernels();
    int issued = 0;                                                     // stages that warp 0 asked for
    if (!a.offsets && warp == 0) {
        // one group: its table needs no memory, and the first copies wait for no other warp
        if (lane == 0) {
            tile_start[0] = first_row[0] = 0;
            tile_start[1] = (a.rows + T - 1) / T;
            end_row[0] = a.rows;
        }
        __syncwarp();
        if (PAIR && in_pair != 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");   // the leader's barriers are set up
        if (first < tile_start[1] * pairs_n) {
            const Tile tile = decode(first);
            for (int b = kb0; b < kb1 && issued < C::kStages; b += C::kSub) copy_stage(tile, b, issued++);
        }
    }
    if (threadIdx.x == 0) s_skip = *reinterpret_cast<volatile int *>(a.err);
    // two experts per thread, then the warps' sums
    if (2 * threadIdx.x < a.experts) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 2 * threadIdx.x + i;
            if (e < a.experts) {
                // 64-code blocks of the longest window length that no channel's weights pass 2^24 in
                const int bits = a.windows[e];
                int j = 6;
                while (j > 0 && (bits >> j & 1)) --j;
                window_of[e] = 16 << j;
            }
        }
    }
    if (a.offsets) {
        // An expert's rows begin at the largest offset up to its own, so that no offsets, ascending or not, give a row
        // to two experts: first the running maximum, then the running sum of the token tiles.
        const int e0 = 2 * threadIdx.x;
        int o[3], top = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) o[i] = e0 + i <= a.experts ? min(max(a.offsets[e0 + i], 0), a.rows) : 0;
        top = max(o[0], o[1]);
        for (int m = 1; m < 32; m <<= 1) {
            const int other = __shfl_up_sync(0xffffffffu, top, m);
            if (lane >= m) top = max(top, other);
        }
        if (lane == 31) warp_tops[warp] = top;
        top = __shfl_up_sync(0xffffffffu, top, 1);
        if (lane == 0) top = 0;
        __syncthreads();
        for (int w = 0; w < warp; ++w) top = max(top, warp_tops[w]);
        int c[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int lo = max(top, o[i]), hi = max(lo, o[i + 1]);
            top = lo;
            if (e0 + i < a.experts) {
                first_row[e0 + i] = lo;
                end_row[e0 + i] = hi;
                c[i] = (hi - lo + T - 1) / T;
            }
        }
        int sum = c[0] + c[1];
        for (int m = 1; m < 32; m <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += o;
        }
        if (lane == 31) warp_sums[warp] = sum;
        __syncthreads();
        int before = sum - c[0] - c[1];
        for (int w = 0; w < warp; ++w) before += warp_sums[w];
        if (2 * threadIdx.x < a.experts) tile_start[2 * threadIdx.x + 1] = before + c[0];
        if (2 * threadIdx.x + 1 < a.experts) tile_start[2 * threadIdx.x + 2] = before + c[0] + c[1];
        if (threadIdx.x == 0) tile_start[0] = 0;
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR && (a.offsets || warp != 0 || in_pair == 0)) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;
    const bool skip = s_skip != 0;

    const int total = skip ? 0 : tile_start[a.experts] * pairs_n;
    bool ok = true;
    if (warp < 4) {
        set_regs<kRegsIssue>();
        if (warp == 0) {
            // what was asked for before the roles began: the first stages of the first tile
            int s = issued % C::kStages, done = issued;
            uint32_t ph = issued == C::kStages ? 0u : 1u;               // parity of the stage's previous release
            for (int t = first; t < total && ok; t += step) {
                const Tile tile = decode(t);
                for (int b = kb0 + done * C::kSub; b < kb1; b += C::kSub) {
                    ok = mbar_wait(empty(s), ph, abort_flag, a.err);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    copy_stage(tile, b, s);
                    ++issued;
                    if (++s == C::kStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                done = 0;
            }
            // The last MMAs' arrivals come to this CTA's shared memory, from a pair's leader too: it does not leave before.
            if (ok && !skip) {
                const int hands = issued * C::kHands;
                for (int i = max(0, issued - C::kStages); i < issued && ok; ++i)
                    ok = mbar_wait(empty(i % C::kStages), (uint32_t)((i / C::kStages) & 1), abort_flag, a.err);
                for (int i = max(0, hands - C::kSlots); i < hands && ok; ++i)
                    ok = mbar_wait(slot_free(i % C::kSlots), (uint32_t)((i / C::kSlots) & 1), abort_flag, a.err);
                ok = __all_sync(0xffffffffu, ok);
            }
            // nor before its copies have landed: those that no one waited for, where a wait expired
            if (!ok || skip)
                for (int i = max(0, issued - C::kStages); i < issued; ++i)
                    mbar_drain(full(i % C::kStages), (uint32_t)((i / C::kStages) & 1));
            // Only the leader's barriers know of the peer's token copies, so where it gave up it asks the peer how many
            // stages it has asked for and waits for those; the peer stays until the leader is done. (A second cluster
            // barrier instead, for every launch: 512 rows, 4096 x 4096 18.5 us instead of 17.0.)
            if (PAIR && in_pair != 0) {
                if (lane == 0)
                    asm volatile("st.release.cluster.shared::cluster.u32 [%0], %1;" ::"r"(map_shared(smem_addr(peer_issued), 0)),
                                 "r"(issued + 1)
                                 : "memory");
            } else if (PAIR && (!ok || skip)) {
                int asked = 0;                                          // plus one
                const long long t0 = clock64();
                while (asked == 0 && clock64() - t0 < 2 * kWaitLimitCycles)
                    asm volatile("ld.acquire.cluster.shared::cta.u32 %0, [%1];" : "=r"(asked) : "r"(smem_addr(peer_issued)) : "memory");
                for (int i = max(0, asked - 1 - C::kStages); i < asked - 1; ++i)
                    mbar_drain(peer_full(i % C::kStages), (uint32_t)((i / C::kStages) & 1));
            }
        } else if (warp == 1 && in_pair == 0) {
            const uint64_t bd0 = sdesc_sw128(stage0);
            int s = 0, slot = 0, cc = 0;
            uint32_t ph = 0;
            bool ready = false;
            for (int t = first; t < total && ok; t += step) {
                const Tile tile = decode(t);
                const int win = window_of[tile.e];
                const uint32_t idesc =
                    (1u << 4) | ((uint32_t)(tile.columns() >> 3) << 17) | ((uint32_t)(C::kCtas * 128 >> 4) << 24);
                for (int b = kb0; b < kb1 && ok;) {
                    const int end = min(kb1, (b / win + 1) * win);      // one exact window, one accumulator
                    const int d = cc & 1;
                    ok = wait_acquire<PAIR>(dempty(d), (uint32_t)((cc >> 1) & 1) ^ 1u, abort_flag, a.err);
                    ok = __all_sync(0xffffffffu, ok);
                    uint32_t acc = 0;
                    for (; b < end && ok; b += C::kSub) {
                        // The widening warps waited for this CTA's copies, and warp 2 for the peer's, so their arrival
                        // speaks for both operands.
                        const int now = s;
                        const uint32_t now_ph = ph;
                        if (++s == C::kStages) {
                            s = 0;
                            ph ^= 1u;
                        }
                        const uint64_t bd = bd0 + (uint64_t)(now * (C::kStageBytes >> 4));
#pragma unroll
                        for (int h = 0; h < C::kHands; ++h) {
                            if (!ready) {
                                ok = wait_acquire<PAIR>(wide(now, h), now_ph, abort_flag, a.err);
                                ok = __all_sync(0xffffffffu, ok);
                                if (!ok) break;
                            }
                            // the next hand-off is looked at early: the answer takes a while
                            const bool next = h + 1 < C::kHands ? mbar_test<PAIR>(wide(now, h + 1), now_ph)
                                                                : mbar_test<PAIR>(wide(s, 0), ph);
                            tc_fence_after();
                            if (elect_one()) {
                                const uint32_t at = tmem + (uint32_t)(2 * T + slot * C::kSlotCols);
#pragma unroll
                                for (int j = 0; j < C::kGroup; ++j) {
                                    const int block = h * C::kGroup + j;
                                    if (block > 0 && b + block >= end) break;
#pragma unroll
                                    for (int q = 0; q < 4; ++q)
                                        mma_ts<PAIR>(tmem + (uint32_t)(d * T), at + 32 * j + 8 * q,
                                                     bd + (uint64_t)(block * (C::kXBytes >> 4) + 2 * q), idesc,
                                                     acc | (uint32_t)(block + q));
                                }
                                commit<PAIR>(slot_free(slot));
                                if (h + 1 == C::kHands) {
                                    commit<PAIR>(empty(now));
                                    if (b + C::kSub >= end) commit<PAIR>(dfull(d));
                                }
                            }
                            ready = __all_sync(0xffffffffu, next);
                            if (++slot == C::kSlots) slot = 0;
                        }
                        if (!ok) break;
                        acc = 1;
                    }
                    ++cc;
                }
            }
            // all MMAs that are on their way, whether or not another role gave up, before tensor memory is handed back
            if (elect_one()) commit<PAIR>(tail, 1);
            __syncwarp();
            mbar_drain(tail, 0);
        } else if (PAIR && warp == 2 && in_pair == 0) {
            // The peer's token codes of each stage: this idle warp waits for them and joins the arrivals of the stage's
            // first hand-off, so that the MMA warp has no second barrier to wait for.
            const int tiles = total > first ? (total - first + step - 1) / step : 0;
            const long long stages = (long long)tiles * ((kb1 - kb0 + C::kSub - 1) / C::kSub);
            int s = 0;
            uint32_t ph = 0;
            for (long long it = 0; it < stages; ++it) {
                ok = wait_acquire<PAIR>(peer_full(s), ph, abort_flag, a.err);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) mbar_arrive(wide(s, 0));
                if (++s == C::kStages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
        __syncwarp();
        if (!PAIR && parts > 1) {
            cluster_sync();
            cluster_sync();
        }
    } else if (warp < 12) {
        set_regs<C::kRegsWiden>();
        const int set = (warp >> 2) - 1;                                // takes every other block of a stage
        const int m = (warp & 3) * 32 + lane;                           // channel of the tile = tensor-memory lane
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16) + 2 * T;
        const int tiles = total > first ? (total - first + step - 1) / step : 0;
        const int per_tile = (kb1 - kb0 + C::kSub - 1) / C::kSub, last = kb1 - kb0 - (per_tile - 1) * C::kSub;
        const long long stages = (long long)tiles * per_tile;
        // LOOSE: this thread's pieces of the next stage (block xb of tile xtile)
        uint4 x[C::kChunks];
        Tile xtile{};
        int xt = first, xb = kb0;
        const int u = (int)threadIdx.x - 128;
        auto fetch = [&] {
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i) {
                const int c = u + 256 * i, row = c / (4 * C::kSub), piece = c % (4 * C::kSub), k0 = xb * 64 + piece * 16;
                x[i] = make_uint4(0, 0, 0, 0);
                if (row < xtile.rows && k0 < a.k) x[i] = loose_codes(a, xtile.row + row, k0);
            }
            xb += C::kSub;
            if (xb >= kb1) {
                xb = kb0;
                xt += step;
                if (xt < total) xtile = decode(xt);
            }
        };
        if (LOOSE && first < total) {
            xtile = decode(first);
            fetch();
        }
        // hand-offs are numbered it * kHands + h, their slots in turn; with one block each, a set takes every other one
        int s = 0, left = per_tile, slot = C::kGroup == 1 ? set : 0;
        uint32_t ph = 0, slot_ph = 1;                                   // the first use of a slot waits for nothing
        for (long long it = 0; it < stages; ++it) {
            int blocks = C::kSub;
            if (--left == 0) {
                left = per_tile;
                blocks = last;
            }
            ok = mbar_wait(full(s), ph, abort_flag, a.err) && mbar_wait(slot_free(slot), slot_ph, abort_flag, a.err);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (LOOSE) {
                // into the layout that TMA leaves: rows of 128 bytes, 16-byte pieces swizzled by the row
                uint8_t *xs = smem + s * C::kStageBytes;
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i) {
                    const int c = u + 256 * i, row = c / (4 * C::kSub), piece = c % (4 * C::kSub);
                    uint8_t *to = xs + (piece >> 2) * C::kXBytes + row * 128;
                    const int at = (piece & 3) * 2;
                    const uint32_t w[4] = {x[i].x ^ 0x80808080u, x[i].y ^ 0x80808080u, x[i].z ^ 0x80808080u, x[i].w ^ 0x80808080u};
                    uint32_t h[8];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        h[2 * q] = hsub2(prmt(w[q], 0x64646464u, 0x4140u), 0x64806480u);
                        h[2 * q + 1] = hsub2(prmt(w[q], 0x64646464u, 0x4342u), 0x64806480u);
                    }
                    *reinterpret_cast<uint4 *>(to + ((at ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                    *reinterpret_cast<uint4 *>(to + (((at + 1) ^ (row & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                if (it + 1 < stages) fetch();
            }
#pragma unroll
            for (int j = 0; j < (C::kGroup == 1 ? 1 : C::kGroup / 2); ++j) {
                const int block = 2 * j + set;
                if (block >= blocks) break;                             // a tile's last stage may hold fewer
                const uint8_t *src = smem + s * C::kStageBytes + C::kWOffset + block * kBlockBytes + m * 16;
                uint32_t h[32];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(src + i * 2048);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        h[8 * i + 2 * q] = hsub2(prmt(w[q], 0x64646464u, 0x4140u), 0x64806480u);
                        h[8 * i + 2 * q + 1] = hsub2(prmt(w[q], 0x64646464u, 0x4342u), 0x64806480u);
                    }
                }
                tmem_st32(t_lane + (uint32_t)(slot * C::kSlotCols + (C::kGroup == 1 ? 0 : block * 32)), h);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = wide(s, C::kGroup == 1 ? set : 0);
                if (PAIR && in_pair != 0) mbar_arrive_remote(map_shared(bar, 0));
                else mbar_arrive(bar);                                  // a release: speaks for the token codes, too
            }
            slot += C::kGroup == 1 ? 2 : 1;
            if (slot >= C::kSlots) {
                slot -= C::kSlots;
                slot_ph ^= 1u;
            }
            if (++s == C::kStages) {
                s = 0;
                ph ^= 1u;
            }
        }
        __syncwarp();
        if (!PAIR && parts > 1) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        set_regs<C::kRegsOut>();
        constexpr int kHalf = T / 2;
        const int half = (warp >> 2) - 3;
        const int m = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * kHalf);
        float *scales = reinterpret_cast<float *>(bar_area + 1024 + C::kTables) + (warp - 12) * kHalf;
        int cc = 0;
        auto release = [&](int d) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_remote(map_shared(dempty(d), 0));
                else mbar_arrive(dempty(d));
            }
        };
        for (int t = first; t < total && ok; t += step) {
            const Tile tile = decode(t);
            const int win = window_of[tile.e];
            const int ch = (tile.ch + (int)in_pair) * kRowTile + m;
            const bool live = ch < a.n;
            const float sw = live ? a.s_w[(long long)tile.e * a.n + ch] : 0.0f;
            const float bias = live && a.bias ? a.bias[(long long)tile.e * a.n + ch] : 0.0f;
            const int chunks = (kb1 - 1) / win - kb0 / win + 1;
            // the tokens' scales of this warpgroup's columns, the warp's own copy
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kHalf; i += 32) {
                const int c = half * kHalf + i + lane;
                if (i + lane < kHalf) scales[i + lane] = c < tile.rows ? a.s_x[tile.row + c] : 0.0f;
            }
            __syncwarp();
            const bool warp_live = (tile.ch + (int)in_pair) * kRowTile + (int)(warp & 3) * 32 + 32 <= a.n;
            // 16 tokens' sums of this channel, from column half * kHalf + g
            auto emit = [&](float (&v)[16], int g) {
                const int c0 = half * kHalf + g;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 sx = reinterpret_cast<const float4 *>(scales + g)[i];
                    v[4 * i] = v[4 * i] * sw * sx.x;
                    v[4 * i + 1] = v[4 * i + 1] * sw * sx.y;
                    v[4 * i + 2] = v[4 * i + 2] * sw * sx.z;
                    v[4 * i + 3] = v[4 * i + 3] * sw * sx.w;
                }
                if (a.bias) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] += bias;
                }
                if (warp_live && c0 + 16 <= tile.rows && (a.y_type == HATQ_F32 || a.y_even)) {
                    const long long row = tile.row + c0;
                    if (a.y_type == HATQ_F32) {
                        float *y = reinterpret_cast<float *>(a.y) + row * a.ldy + ch;
#pragma unroll
                        for (int i = 0; i < 16; ++i, y += a.ldy) *y = v[i];
                        return;
                    }
                    // Lanes 2i and 2i + 1 swap halves: the even one then has both channels of the first eight tokens,
                    // the odd one of the others, and 16 stores of 2 bytes become 8 of 4.
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], a.y_type == HATQ_BF16);
                    const bool odd = (lane & 1) != 0;
                    char *y = reinterpret_cast<char *>(a.y) + ((row + (odd ? 8 : 0)) * a.ldy + (ch & ~1)) * 2;
                    const long long pitch = a.ldy * 2;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t mine = odd ? w[4 + i] : w[i];
                        const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? w[i] : w[4 + i], 1);
                        const uint32_t lo = odd ? other : mine, hi = odd ? mine : other;
                        *reinterpret_cast<uint32_t *>(y) = prmt(lo, hi, 0x5410u);
                        *reinterpret_cast<uint32_t *>(y + pitch) = prmt(lo, hi, 0x7632u);
                        y += 2 * pitch;
                    }
                    return;
                }
                long long at = (long long)(tile.row + c0) * a.ldy + ch;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (live && c0 + i < tile.rows) put(a.y, a.y_type, at, v[i]);
                    at += a.ldy;
                }
            };
            if (chunks == 1 && parts == 1) {
                ok = mbar_wait(dfull(cc & 1), (uint32_t)((cc >> 1) & 1), abort_flag, a.err);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = t_lane + (uint32_t)((cc & 1) * T);
                const int end = min(kHalf, tile.rows - half * kHalf);
                uint32_t r[16];
                if (end > 0) tmem_ld16(from, r);
#pragma unroll 1
                for (int g = 0; g < end; g += 16) {
                    tmem_wait_ld();
                    float v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
                    if (g + 16 < end) tmem_ld16(from + (uint32_t)(g + 16), r);    // while these are stored
                    emit(v, g);
                }
                release(cc & 1);
                ++cc;
            } else {
                int acc[kHalf];
#pragma unroll
                for (int i = 0; i < kHalf; ++i) acc[i] = 0;
                for (int q = 0; q < chunks; ++q, ++cc) {
                    ok = mbar_wait(dfull(cc & 1), (uint32_t)((cc >> 1) & 1), abort_flag, a.err);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int g = 0; g < kHalf; g += 16) {
                        uint32_t r[16];
                        tmem_ld16(t_lane + (uint32_t)((cc & 1) * T + g), r);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[g + i] += __float2int_rn(__uint_as_float(r[i]));
                    }
                    release(cc & 1);
                }
                if (!ok) break;
                if (parts == 1) {
#pragma unroll
                    for (int g = 0; g < kHalf; g += 16) {
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = (float)acc[g + i];
                        emit(v, g);
                    }
                } else {
                    // every MMA of this CTA is done: the stages hold its sums, [token][channel]
                    int *sums = reinterpret_cast<int *>(smem);
#pragma unroll
                    for (int i = 0; i < kHalf; ++i) sums[(half * kHalf + i) * kRowTile + m] = acc[i];
                }
            }
        }
        __syncwarp();
        if (!PAIR && parts > 1) {
            // this CTA finishes every parts-th token: a warp takes a token, a lane four channels; scales are on their way
            // while the others' sums are waited for, and the parts' sums all loaded before the first is added
            constexpr int kOwn = T / 16 < 8 ? T / 16 : 8;               // tokens of a warp, at two parts
            float sw[4], bias[4], sx[kOwn];
            Tile tile{};
            if (first < total) tile = decode(first);
            const int ch = tile.ch * kRowTile + 4 * lane, c0 = part + parts * (warp - 12);
            if (first < total) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool live = ch + i < a.n;
                    sw[i] = live ? a.s_w[(long long)tile.e * a.n + ch + i] : 0.0f;
                    bias[i] = live && a.bias ? a.bias[(long long)tile.e * a.n + ch + i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int c = c0 + 8 * parts * i;
                    sx[i] = c < tile.rows ? a.s_x[tile.row + c] : 0.0f;
                }
            }
            cluster_sync();
            // the parts' sums are all asked for before the first is used, and the others may leave once they are here:
            // the second barrier completes while the outputs are written
            constexpr int kBatch = kOwn < 4 ? kOwn : 4;
            const bool finish = ok && first < total;
            const uint32_t mine = smem_addr(smem) + 16u * (uint32_t)lane;
#pragma unroll
            for (int i0 = 0; i0 < kOwn; i0 += kBatch) {
                int4 v[kBatch][kMaxSplit];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int c = c0 + 8 * parts * (i0 + i);
#pragma unroll
                    for (int q = 0; q < kMaxSplit; ++q)
                        if (finish && c < tile.rows && q < parts)
                            v[i][q] = load_cluster(map_shared(mine + (uint32_t)c * (kRowTile * 4), (uint32_t)q));
                        else v[i][q] = make_int4(0, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
#pragma unroll
                    for (int q = 1; q < kMaxSplit; ++q) {
                        v[i][0].x += v[i][q].x;
                        v[i][0].y += v[i][q].y;
                        v[i][0].z += v[i][q].z;
                        v[i][0].w += v[i][q].w;
                    }
                if (i0 + kBatch >= kOwn) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int c = c0 + 8 * parts * (i0 + i);
                    if (!finish || c >= tile.rows) break;
                    const int part4[4] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w};
                    const long long at = (long long)(tile.row + c) * a.ldy + ch;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float r = (float)part4[q] * sw[q] * sx[i0 + i];
                        if (ch + q < a.n) put(a.y, a.y_type, at + q, a.bias ? r + bias[q] : r);
                    }
                }
            }
            asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();
    tc_fence_after();
    if (warp == 1) {
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

template <int T, bool PAIR, bool LOOSE = false>
cudaError_t launch(const CUtensorMap &tm, const LinearArgs &a, int clusters, cudaStream_t s) {
    using C = Config<T, PAIR, LOOSE>;
    // the roles' shares go by what the launch brings: a decrease below it, increases that fit its sum
    static const int regs = [] {
        cudaFuncAttributes fa{};
        return cudaFuncGetAttributes(&fa, linear_tc_kernel<T, PAIR, LOOSE>) == cudaSuccess ? fa.numRegs : 0;
    }();
    if (regs != kLaunchRegs) return cudaErrorInvalidConfiguration;
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(linear_tc_kernel<T, PAIR, LOOSE>), C::kSmem, allowed);
    if (e != cudaSuccess) return e;
    const int width = PAIR ? 2 : a.split;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * width));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0] = early_start();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)width;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = width > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, linear_tc_kernel<T, PAIR, LOOSE>, tm, a);
}

}  // namespace

cudaError_t launch_linear_tc(const CUtensorMap &tm, const LinearArgs &a, int tile, bool pair, bool loose, int clusters,
                             cudaStream_t s) {
    if (loose)
        return tile == 32   ? launch<32, false, true>(tm, a, clusters, s)
               : tile == 64 ? launch<64, false, true>(tm, a, clusters, s)
                            : launch<128, false, true>(tm, a, clusters, s);
    if (pair) return tile == 128 ? launch<128, true>(tm, a, clusters, s) : launch<192, true>(tm, a, clusters, s);
    switch (tile) {
        case 32: return launch<32, false>(tm, a, clusters, s);
        case 64: return launch<64, false>(tm, a, clusters, s);
        default: return launch<128, false>(tm, a, clusters, s);
    }
}

}  // namespace hatq
