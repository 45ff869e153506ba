// Products with 4-bit weights that have one scale per group of inputs.
#include <climits>
#include <type_traits>

#include "hatq_linear4.h"
#include "hatq_mma4.h"
#include "hatq_tc.h"

namespace hatq {
namespace {

// y[r][n] = s_x[r] sum_g s[n][g] sum_{k in g} c[n][k] x[r][k] + bias[n].
//
// The inner sums run on the tensor cores as W x^T in m16n8k16 steps, 16 channels by 8 rows of x: codes are exact in
// both 16-bit types, so 16-bit x go in as they are and fp32 x as the sum of three bf16 numbers, which is exact. A
// group's sum is scaled in fp32 and added to the total.
//
// Layout: strips of 16 channels, in each units of 128 inputs (64 where a group is no multiple of 128) one after the
// other: 16 bytes of codes a lane and 64 inputs, then the unit's 16 or 2 x 16 scales, so that one bulk copy brings in a
// warp's next units whole. The order of inputs within a step is free: lane t of four has inputs 8 t .. 8 t + 7 of each
// 32, the first four in the first step, so that x is read 16 bytes a lane from rows as they lie.
//
// Two kernels. A few rows (linear4_few): memory-bound by the weights. x lies in shared memory whole; a CTA's warps share
// the inputs of a strip, each with its own ring of bulk copies that runs on from strip to strip, and add up at the
// strip's end. More rows, or x too large for that (linear4_many): a strip a warp, x streamed through shared memory for
// all of a CTA's strips; CTAs of a cluster share the inputs where there are few strips.
//
// Measured: 4096 -> 4096, one row 5.8 us; 4096 -> 16384, one row 11 us (3.3 TB/s), 16 rows 15.5 us: bound by the instructions
// that widen codes and fill the steps; 8192 -> 4096, 64 rows 21.4 us, of which the warp-level MMAs alone take 7.3.

constexpr int kCtaStrips = 8, kMostWarps = 16;
constexpr int kFewStages = 3;          // of a warp's ring, at most; each two units of 128, or four of 64

template <typename T> constexpr int kParts = std::is_same<T, float>::value ? 3 : 1;

// a word's codes as the A operand of a step
template <typename T>
__device__ __forceinline__ void widen(uint32_t w, uint32_t (&A)[4]) {
    if constexpr (std::is_same<T, __half>::value) {
        const uint32_t u = w >> 8;
        A[0] = codes_f16<true, false>(w);
        A[1] = codes_f16<true, true>(w);
        A[2] = codes_f16<true, false>(u);
        A[3] = codes_f16<true, true>(u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) A[i] = codes_bf16(w >> 4 * i);
    }
}

// 8 inputs of a row in 16-bit parts: the upper 16 bits of a fp32 number are a bf16 number, and what is left has 16, then
// 8 bits; nothing is left of an infinity
template <typename T>
__device__ __forceinline__ void load8(const Linear4Args &a, const T *row, bool live, int k, uint4 (&out)[kParts<T>]) {
    if constexpr (std::is_same<T, float>::value) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (live && a.vec && k + 8 <= a.k) {
            const float4 x = __ldg(reinterpret_cast<const float4 *>(row + k)), y = __ldg(reinterpret_cast<const float4 *>(row + k) + 1);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
            v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else if (live) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < a.k) v[i] = row[k + i];
        }
        // (a NaN may have no bit of it in its upper half, which would be an infinity; a sum's has all)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fadd_rn(v[i], 0.0f);
#pragma unroll
        for (int part = 0; part < 3; ++part) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t x = __float_as_uint(v[i]), y = __float_as_uint(v[i + 1]);
                w[i / 2] = __byte_perm(x, y, 0x7632);
                v[i] = (x & 0x7f800000u) == 0x7f800000u ? 0.0f : v[i] - __uint_as_float(x & 0xffff0000u);
                v[i + 1] = (y & 0x7f800000u) == 0x7f800000u ? 0.0f : v[i + 1] - __uint_as_float(y & 0xffff0000u);
            }
            out[part] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
        out[0] = make_uint4(0, 0, 0, 0);
        if (live && a.vec && k + 8 <= a.k) {
            out[0] = __ldg(reinterpret_cast<const uint4 *>(row + k));
        } else if (live) {
            const unsigned short *p = reinterpret_cast<const unsigned short *>(row) + k;
            unsigned short v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < a.k ? p[i] : 0;
            out[0] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
// 16 bytes, the first `bytes` of them from src (16-byte aligned, unless bytes is 0), zeros behind
__device__ __forceinline__ void async_copy(uint32_t dst, const void *src, int bytes) {
    const void *from = bytes ? src : reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)15);
    asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void store_y(const Linear4Args &a, int row, int n, float v) {
    if (a.s_x) v *= __ldg(a.s_x + row);
    if (a.bias) v += __ldg(a.bias + n);
    const long long at = (long long)row * a.ldy + n;
    if (a.y_type == HATQ_F32) static_cast<float *>(a.y)[at] = v;
    else if (a.y_type == HATQ_F16) static_cast<__half *>(a.y)[at] = from_f32<__half>(v);
    else static_cast<__nv_bfloat16 *>(a.y)[at] = from_f32<__nv_bfloat16>(v);
}

// A unit's products with NT tiles of 8 rows, added to the totals: BLOCKS x 64 inputs, SCALES scales a channel, of STRIPS
// strips (strip_pitch bytes on) that share what is read of x. x: lane
// (g, t)'s row of the first tile at the unit's first input (8 t on); `next` bytes on the row of the next tile, part_pitch
// on the next part. (Columns of rows that are none may hold anything.) Two sums at a time where tiles are few: steps
// that add to one wait for each other.
template <typename T, int NT, int BLOCKS, int SCALES, int STRIPS>
__device__ __forceinline__ void unit_products(const uint8_t *unit, int strip_pitch, const uint8_t *x, int next, int part_pitch, int lane,
                                              float (&total)[STRIPS][NT][4]) {
    constexpr bool kHalf = std::is_same<T, __half>::value;
    constexpr int SUMS = SCALES == 2 || NT <= 2 ? 2 : 1;
    uint4 w[STRIPS][BLOCKS];
    float s[STRIPS][SCALES][2], sum[SUMS][STRIPS][NT][4];
#pragma unroll
    for (int z = 0; z < STRIPS; ++z) {
        const uint8_t *of = unit + z * strip_pitch;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) w[z][i] = *reinterpret_cast<const uint4 *>(of + 512 * i + 16 * lane);
        const float *scales = reinterpret_cast<const float *>(of + 512 * BLOCKS) + (lane >> 2);
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            s[z][i][0] = scales[kStrip * i];
            s[z][i][1] = scales[kStrip * i + 8];
        }
    }
#pragma unroll
    for (int h = 0; h < 2 * BLOCKS; ++h) {                   // 32 inputs
        const int of = SUMS == 1 ? 0 : BLOCKS == 2 ? h >> 1 : h;
        const bool first = SUMS == 1 || BLOCKS == 1 ? h == 0 || SUMS == 2 : (h & 1) == 0;
        uint32_t A[STRIPS][2][4];
#pragma unroll
        for (int z = 0; z < STRIPS; ++z) {
            widen<T>(h & 1 ? w[z][h >> 1].z : w[z][h >> 1].x, A[z][0]);
            widen<T>(h & 1 ? w[z][h >> 1].w : w[z][h >> 1].y, A[z][1]);
        }
#pragma unroll
        for (int part = kParts<T> - 1; part >= 0; --part) {
            uint4 b[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) b[nt] = *reinterpret_cast<const uint4 *>(x + nt * next + part * part_pitch + 64 * h);
#pragma unroll
            for (int z = 0; z < STRIPS; ++z)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (first && part == kParts<T> - 1) mma_first<kHalf>(sum[of][z][nt], A[z][0], b[nt].x, b[nt].y);
                    else mma_more<kHalf>(sum[of][z][nt], A[z][0], b[nt].x, b[nt].y);
                }
#pragma unroll
            for (int z = 0; z < STRIPS; ++z)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_more<kHalf>(sum[of][z][nt], A[z][1], b[nt].z, b[nt].w);
        }
    }
#pragma unroll
    for (int z = 0; z < STRIPS; ++z)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float &to = total[z][nt][i];
                if constexpr (SCALES == 2)
                    to = fmaf(s[z][SCALES - 1][i >> 1], sum[SUMS - 1][z][nt][i], fmaf(s[z][0][i >> 1], sum[0][z][nt][i], to));
                else
                    to = fmaf(s[z][0][i >> 1], SUMS == 2 ? sum[0][z][nt][i] + sum[SUMS - 1][z][nt][i] : sum[0][z][nt][i], to);
            }
}

// `ways` warps of the CTA share a strip's units; a CTA takes every gridDim.x-th set of strips.
template <typename T, int NT, int BLOCKS, int SCALES>
__global__ void __launch_bounds__(kMostWarps * 32, 1) linear4_few(const Linear4Args a, int ways, int stages) {
    constexpr int ROWS = 8 * NT, PITCH = kStrip + 4, UNIT = 512 * BLOCKS + 4 * kStrip * SCALES, STAGE_UNITS = 4 / BLOCKS;
    constexpr int STAGE = STAGE_UNITS * UNIT;
    const int warps = blockDim.x >> 5;
    extern __shared__ __align__(128) uint8_t smem[];         // rings, sums of a strip, x
    __shared__ __align__(8) uint64_t bars[kMostWarps][kFewStages];
    __shared__ int s_abort;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint8_t *ring = smem + warp * stages * STAGE;
    float *sums = reinterpret_cast<float *>(smem + warps * stages * STAGE);
    uint8_t *xs = smem + warps * stages * STAGE + warps * ROWS * PITCH * 4;
    const uint32_t bar = tc::smem_addr(bars[warp]);
    volatile int *abort_flag = &s_abort;
    if (lane < stages) tc::mbar_init(bar + 8 * lane, 1);
    tc::fence_barrier_init();
    if (threadIdx.x == 0) s_abort = 0;
    __syncthreads();
    after_prior_kernels();
    const int err = *reinterpret_cast<volatile int *>(a.err);

    const int sets = warps / ways, way = warp % ways, set = warp / ways;
    const int from = a.units * way / ways, to = a.units * (way + 1) / ways, per = (to - from + STAGE_UNITS - 1) / STAGE_UNITS;
    const int step = gridDim.x * sets;
    // ---- this warp's copies: `per` a strip
    int asked = 0, ask_stage = 0, strip = blockIdx.x * sets + set, chunk = 0;
    auto ask = [&]() {
        if (strip >= a.strips) return;
        if (lane == 0) {
            const int first = from + chunk * STAGE_UNITS, bytes = min(STAGE_UNITS, to - first) * UNIT;
            tc::mbar_expect_tx(bar + 8 * ask_stage, bytes);
            bulk_load(tc::smem_addr(ring + ask_stage * STAGE), a.w + ((long long)strip * a.units + first) * UNIT, bytes, bar + 8 * ask_stage);
        }
        ++asked;
        if (++ask_stage == stages) ask_stage = 0;
        if (++chunk == per) {
            chunk = 0;
            strip += step;
        }
    };
    for (int i = 0; i < stages; ++i) ask();

    // ---- x, behind its last input zeros
    const int k_pad = a.units * BLOCKS * kStep, row_pitch = 2 * k_pad + 64, part_pitch = a.rows * row_pitch;
    for (int row = warp; row < a.rows; row += warps) {
        const T *p = static_cast<const T *>(a.x) + (long long)row * a.ldx;
        uint8_t *to_x = xs + row * row_pitch;
        if (a.vec && kParts<T> == 1) {
#pragma unroll 4
            for (int k = 8 * lane; k < k_pad; k += 256) async_copy(tc::smem_addr(to_x + 2 * k), p + min(k, a.k - 1), min(max(2 * (a.k - k), 0), 16));
        } else {
#pragma unroll 2
            for (int k = 8 * lane; k < k_pad; k += 256) {
                uint4 v[kParts<T>];
                load8<T>(a, p, true, k, v);
#pragma unroll
                for (int part = 0; part < kParts<T>; ++part) *reinterpret_cast<uint4 *>(to_x + part * part_pitch + 2 * k) = v[part];
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    bool sound = !__syncthreads_or(err != 0);

    int done = 0, stage = 0;
    uint32_t parity = 0;
    const int rounds = (a.strips + step - 1) / step, row = min(g, a.rows - 1), next = (min(g + 8, a.rows - 1) - row) * row_pitch;
    const uint8_t *x = xs + row * row_pitch + 16 * t;
    for (int round = 0; round < rounds && sound; ++round) {
        const int strip_set = (round * (int)gridDim.x + (int)blockIdx.x) * sets;
        float total[1][NT][4] = {};
        if (strip_set + set < a.strips)
            for (int c = 0; c < per; ++c) {
                const int first = from + c * STAGE_UNITS, n = min(STAGE_UNITS, to - first);
                sound = __all_sync(0xffffffffu, tc::mbar_wait(bar + 8 * stage, parity, abort_flag, a.err));
                if (!sound) break;
                for (int i = 0; i < n; ++i)
                    unit_products<T, NT, BLOCKS, SCALES, 1>(ring + stage * STAGE + i * UNIT, 0, x + (first + i) * (BLOCKS * 2 * kStep), next, part_pitch,
                                                         lane, total);
                __syncwarp();
                ++done;
                if (++stage == stages) {
                    stage = 0;
                    parity ^= 1;
                }
                ask();
            }
        // ---- the warps' sums
        float *mine = sums + warp * ROWS * PITCH;
        if (round) __syncthreads();                          // (the last ones are read)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(8 * nt + 2 * t + (i & 1)) * PITCH + g + (i >> 1) * 8] = total[0][nt][i];
        sound = !__syncthreads_or(!sound);
        for (int i = threadIdx.x; sound && i < a.rows * kStrip * sets; i += blockDim.x) {
            const int ch = i % kStrip, r = i / kStrip % a.rows, of = i / (kStrip * a.rows), n = (strip_set + of) * kStrip + ch;
            if (n >= a.n) continue;
            const float *p = sums + of * ways * ROWS * PITCH + r * PITCH + ch;
            float v = 0.0f;
#pragma unroll 8
            for (int j = 0; j < ways; ++j) v += p[j * ROWS * PITCH];
            store_y(a, r, n, v);
        }
    }
    // copies still on their way (where a wait gave up) have to land before the CTA leaves
    const long long t0 = clock64();
    for (int i = done; i < asked; ++i)
        while (!tc::mbar_try_wait(bar + 8 * (i % stages), (uint32_t)(i / stages) & 1u) && clock64() - t0 < tc::kWaitLimitCycles) {}
}

// Rows from, from + WARPS, .. of a CTA's sums and those of the other CTAs of its cluster, added up and written. All of a row's
// (two rows') loads are on their way at once: each takes about 400 cycles.
template <int WARPS, int SPLIT>
__device__ __forceinline__ void join_rows(const Linear4Args &a, const float *sums, int pitch, int row0, int from, int to, int lane) {
    const int n = blockIdx.x * kCtaStrips * kStrip + 4 * lane;
#pragma unroll 2
    for (int row = from; row < to; row += WARPS) {
        const float *own = sums + row * pitch + 4 * lane;
        float4 u[SPLIT];
        if constexpr (SPLIT == 1) {
            u[0] = *reinterpret_cast<const float4 *>(own);
        } else {
#pragma unroll
            for (int z = 0; z < SPLIT; ++z) {
                uint32_t there;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(tc::smem_addr(own)), "r"(z));
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(u[z].x), "=f"(u[z].y), "=f"(u[z].z), "=f"(u[z].w) : "r"(there) : "memory");
            }
        }
        float v[4] = {};
#pragma unroll
        for (int z = 0; z < SPLIT; ++z) {
            v[0] += u[z].x;
            v[1] += u[z].y;
            v[2] += u[z].z;
            v[3] += u[z].w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < a.n) store_y(a, row0 + row, n + i, v[i]);
    }
}

constexpr int kManyDepth = 128;        // inputs of a piece of x
constexpr int kManyPitch = 2 * kManyDepth + 64;
constexpr int kManyRing = 1280;        // bytes of a warp's weights for a piece: a unit of 128, or two of 64
constexpr int kManyStages = 4;
template <typename T> constexpr int kXStages = std::is_same<T, float>::value ? 2 : 3;

// Strips a warp: what is read of x is read once for all of them, in return a CTA has fewer warps. Two with eight tiles of
// rows (64 rows of 8192 -> 4096: 21.4 us against 23.6), one with four (32 rows: 15.1 against 16.9) and where registers
// hold two scales a unit.
template <int NT, int SCALES> constexpr int kManyStrips = NT == 8 && SCALES == 1 ? 2 : 1;

// 8 strips a CTA, kManyStrips of them a warp, NT tiles of 8 rows; the CTAs of a cluster (along z) have a part of the
// inputs each.
template <typename T, int NT, int BLOCKS, int SCALES>
__global__ void __launch_bounds__(kCtaStrips / kManyStrips<NT, SCALES> * 32, 2) linear4_many(const Linear4Args a, int split) {
    constexpr int STRIPS = kManyStrips<NT, SCALES>, WARPS = kCtaStrips / STRIPS, RING = STRIPS * kManyRing;
    constexpr int ROWS = 8 * NT, PARTS = kParts<T>, XS = kXStages<T>, PART = ROWS * kManyPitch, XSTAGE = PARTS * PART;
    constexpr int PITCH = kCtaStrips * kStrip + 4, UNIT = 512 * BLOCKS + 4 * kStrip * SCALES, PIECE_UNITS = 2 / BLOCKS;
    extern __shared__ __align__(128) uint8_t smem[];         // rings, x; in the end the CTA's sums
    __shared__ __align__(8) uint64_t bars[WARPS][kManyStages];
    __shared__ int s_abort;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint8_t *ring = smem + warp * kManyStages * RING;
    uint8_t *xs = smem + kCtaStrips * kManyStages * kManyRing;
    const uint32_t bar = tc::smem_addr(bars[warp]);
    volatile int *abort_flag = &s_abort;
    if (lane < kManyStages) tc::mbar_init(bar + 8 * lane, 1);
    tc::fence_barrier_init();
    if (threadIdx.x == 0) s_abort = 0;
    __syncthreads();
    after_prior_kernels();
    bool sound = !__syncthreads_or(*reinterpret_cast<volatile int *>(a.err) != 0);

    const int strip = (int)blockIdx.x * kCtaStrips + warp * STRIPS, row0 = blockIdx.y * ROWS, live = min(ROWS, a.rows - row0);
    const int pieces = (a.k + kManyDepth - 1) / kManyDepth, from = pieces * (int)blockIdx.z / split, to = pieces * ((int)blockIdx.z + 1) / split;
    auto ask = [&](int i) {
        if (i >= to - from || lane) return;
        const int first = (from + i) * PIECE_UNITS, n = min(PIECE_UNITS, a.units - first), stage = i % kManyStages;
        tc::mbar_expect_tx(bar + 8 * stage, STRIPS * n * UNIT);
#pragma unroll
        for (int z = 0; z < STRIPS; ++z)
            bulk_load(tc::smem_addr(ring + stage * RING + z * kManyRing), a.w + ((long long)min(strip + z, a.strips - 1) * a.units + first) * UNIT,
                      n * UNIT, bar + 8 * stage);
    };
    // Pieces of x, zeros behind the last row and input. As they lie, by asynchronous copies; otherwise through registers.
    const bool direct = a.vec && PARTS == 1;
    // A thread has the same 8 inputs of every APARTth row.
    constexpr int APART = WARPS * 2;
    const int x_row = threadIdx.x >> 4, x_k = (threadIdx.x & 15) * 8;
    const T *x_first = static_cast<const T *>(a.x) + (long long)row0 * a.ldx, *x_mine = x_first + (long long)min(x_row, live - 1) * a.ldx + x_k;
    uint8_t *x_to = xs + x_row * kManyPitch + 2 * x_k;
    auto bring = [&](int i, int stage) {
        if (i < to - from) {
            const int k0 = (from + i) * kManyDepth;
            uint8_t *to_x = x_to + stage * XSTAGE;
            if (direct) {
                const int there = min(max(2 * (a.k - k0 - x_k), 0), 16);
                const uint32_t dst = tc::smem_addr(to_x);
                const T *p = x_mine + k0;
#pragma unroll
                for (int j = 0; j < ROWS / APART; ++j) {
                    const int bytes = x_row + APART * j < live ? there : 0;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst + APART * j * kManyPitch),
                                 "l"(bytes ? p + j * APART * a.ldx : x_first), "r"(bytes)
                                 : "memory");
                }
            } else {
                for (int j = 0; j < ROWS / APART; ++j) {
                    uint4 v[PARTS];
                    load8<T>(a, x_first + (long long)min(x_row + APART * j, live - 1) * a.ldx, x_row + APART * j < live, k0 + x_k, v);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) *reinterpret_cast<uint4 *>(to_x + APART * j * kManyPitch + part * PART) = v[part];
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (sound) {
        for (int i = 0; i < kManyStages; ++i) ask(i);
#pragma unroll
        for (int i = 0; i < XS - 1; ++i) bring(i, i);
    }
    float total[STRIPS][NT][4] = {};
    int done = 0, x_stage = 0;
    for (; sound && done < to - from; ++done) {
        const int stage = done % kManyStages, n = min(PIECE_UNITS, a.units - (from + done) * PIECE_UNITS);
        asm volatile("cp.async.wait_group %0;" ::"n"(XS - 2) : "memory");
        const bool here = tc::mbar_wait(bar + 8 * stage, (uint32_t)(done / kManyStages) & 1u, abort_flag, a.err);
        sound = !__syncthreads_or(!here);
        if (!sound) break;
        bring(done + XS - 1, x_stage == 0 ? XS - 1 : x_stage - 1);
        const uint8_t *x = xs + x_stage * XSTAGE + g * kManyPitch + 16 * t;
        for (int i = 0; i < n; ++i)
            unit_products<T, NT, BLOCKS, SCALES, STRIPS>(ring + stage * RING + i * UNIT, kManyRing, x + i * (BLOCKS * 2 * kStep), 8 * kManyPitch, PART,
                                                         lane, total);
        __syncwarp();
        ask(done + kManyStages);
        if (++x_stage == XS) x_stage = 0;
    }
    if (!sound) {                                            // (copies on their way have to land before the CTA leaves)
        const long long t0 = clock64();
        const int asked = min(done + kManyStages, to - from);
        for (int i = done; i < asked; ++i)
            while (!tc::mbar_try_wait(bar + 8 * (i % kManyStages), (uint32_t)(i / kManyStages) & 1u) && clock64() - t0 < tc::kWaitLimitCycles) {}
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    // ---- the CTA's sums, added up over the cluster, a share of the rows each
    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int z = 0; z < STRIPS; ++z)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[(8 * nt + 2 * t + (i & 1)) * PITCH + kStrip * (warp * STRIPS + z) + g + (i >> 1) * 8] = total[z][nt][i];
    if (split > 1) {
        asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    if (*abort_flag) sound = false;
    const int each = (live + split - 1) / split, row_from = (int)blockIdx.z * each, row_to = min(row_from + each, live);
    // 4 channels a thread: a warp has a row, and its store is of whole lines
    if (sound) {
        if (split == 1) join_rows<WARPS, 1>(a, sums, PITCH, row0, row_from + warp, row_to, lane);
        else if (split == 2) join_rows<WARPS, 2>(a, sums, PITCH, row0, row_from + warp, row_to, lane);
        else if (split == 4) join_rows<WARPS, 4>(a, sums, PITCH, row0, row_from + warp, row_to, lane);
        else join_rows<WARPS, 8>(a, sums, PITCH, row0, row_from + warp, row_to, lane);
    }
    if (split > 1) asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

// What a CTA of the few-row kernel has: warps, stages, bytes of shared memory.
struct FewPlan {
    int warps, ways, stages, bytes, ctas;
};
bool plan_few(const Linear4Args &a, long long x_bytes, int tiles, int sms, FewPlan &p) {
    const int stage = a.stage_units * a.unit_bytes;
    auto bytes = [&](int warps, int stages) { return warps * stages * stage + warps * 8 * tiles * (kStrip + 4) * 4 + x_bytes; };
    constexpr long long most = 226 * 1024;
    // two CTAs of 8 warps on an SM, or one of 16, or of 8
    p.stages = kFewStages;
    if (bytes(8, 3) <= most / 2) p.warps = 8;
    else if (bytes(16, 3) <= most) p.warps = 16;
    else if (bytes(16, 2) <= most) p.warps = 16, p.stages = 2;
    else if (bytes(8, 3) <= most) p.warps = 8;
    else return false;
    p.bytes = (int)bytes(p.warps, p.stages);
    // how many warps share a strip: the least time, in units: rounds over the strips, each with about one and a half for
    // the sums and the barrier (16 rows of 4096 x 16384, ways 2 instead of 16: 16.7 us against 17.6)
    const int resident = p.warps == 16 ? 1 : max(1, min(3, 227 * 1024 / (p.bytes + 1024)));
    long long best = LLONG_MAX;
    for (int ways = 1; ways <= p.warps && ways <= a.units; ways *= 2) {
        const long long sets = p.warps / ways, ctas = (a.strips + sets - 1) / sets, room = (long long)sms * resident;
        const long long cost = (ctas + room - 1) / room * (2 * ((a.units + ways - 1) / ways) + 3);
        if (cost < best) {
            best = cost;
            p.ways = ways;
            p.ctas = (int)min(ctas, room);
        }
    }
    return true;
}
template <typename T, int NT, int BLOCKS, int SCALES>
cudaError_t launch_few(const Linear4Args &a, const FewPlan &p, cudaStream_t s) {
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(linear4_few<T, NT, BLOCKS, SCALES>), p.bytes, allowed);
    if (e != cudaSuccess) return e;
    return launch_early(linear4_few<T, NT, BLOCKS, SCALES>, dim3((unsigned)p.ctas), p.warps * 32, p.bytes, s, a, p.ways, p.stages);
}
template <typename T, int NT, int BLOCKS, int SCALES>
cudaError_t launch_many(const Linear4Args &a, int sms, cudaStream_t s) {
    static std::atomic<int> allowed[64];
    constexpr int x_bytes = kXStages<T> * kParts<T> * 8 * NT * kManyPitch, sum_bytes = 8 * NT * (kCtaStrips * kStrip + 4) * 4;
    constexpr int ring = kCtaStrips * kManyStages * kManyRing, bytes = ring + x_bytes > sum_bytes ? ring + x_bytes : sum_bytes;
    static_assert(bytes <= 226 * 1024, "shared memory of a CTA");
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(linear4_many<T, NT, BLOCKS, SCALES>), bytes, allowed);
    if (e != cudaSuccess) return e;
    const int tiles = (a.strips + kCtaStrips - 1) / kCtaStrips, row_tiles = (a.rows + 8 * NT - 1) / (8 * NT);
    const int pieces = (a.k + kManyDepth - 1) / kManyDepth;
    // the split of the inputs that takes the fewest steps: waves x pieces, and about three for joining
    int split = 1;
    long long best = LLONG_MAX;
    for (int x = 1; x <= 8 && x <= pieces; x *= 2) {
        const long long ctas = (long long)tiles * row_tiles * x, room = 2LL * sms, cost = (ctas + room - 1) / room * ((pieces + x - 1) / x) + (x > 1 ? 3 : 0);
        if (cost < best) {
            best = cost;
            split = x;
        }
    }
    cudaLaunchAttribute attr[2] = {early_start(), {}};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)split;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)tiles, (unsigned)row_tiles, (unsigned)split);
    cfg.blockDim = dim3(kCtaStrips / kManyStrips<NT, SCALES> * 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, linear4_many<T, NT, BLOCKS, SCALES>, a, split);
}
template <typename T, int BLOCKS, int SCALES>
cudaError_t launch_units(const Linear4Args &a, int sms, cudaStream_t s) {
    const long long x_bytes = (long long)kParts<T> * a.rows * (2LL * a.units * BLOCKS * kStep + 64);
    FewPlan p;
    if (a.rows <= 16 && plan_few(a, x_bytes, a.rows <= 8 ? 1 : 2, sms, p))
        return a.rows <= 8 ? launch_few<T, 1, BLOCKS, SCALES>(a, p, s) : launch_few<T, 2, BLOCKS, SCALES>(a, p, s);
    // At most 64 rows a CTA, or 32 of fp32 x: their three parts of more leave an SM one CTA (64 rows of 8192 -> 4096: 54 us
    // against 109)
    if (a.rows <= 16) return launch_many<T, 2, BLOCKS, SCALES>(a, sms, s);
    if constexpr (kParts<T> == 1)
        if (a.rows > 32) return launch_many<T, 8, BLOCKS, SCALES>(a, sms, s);
    return launch_many<T, 4, BLOCKS, SCALES>(a, sms, s);
}
template <typename T>
cudaError_t launch_type(const Linear4Args &a, int sms, cudaStream_t s) {
    return a.unit_blocks == 2 ? launch_units<T, 2, 1>(a, sms, s) : a.unit_scales == 1 ? launch_units<T, 1, 1>(a, sms, s) : launch_units<T, 1, 2>(a, sms, s);
}

// A warp per strip and 64 inputs: lane (g, t) packs channels g and g + 8 (the first in the lower of two nibbles) at inputs
// 8 t .. 8 t + 7 of each half of them; a word has four inputs, their pairs 16 bits apart.
__global__ void __launch_bounds__(256) layout_kernel(const int8_t *w, long long ldw, const float *scales, long long lds, const Linear4Args a,
                                                     uint8_t *out) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, blocks = a.units * a.unit_blocks;
    const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at >= (long long)a.strips * blocks) return;
    const int strip = (int)(at / blocks), block = (int)(at % blocks), in_unit = block % a.unit_blocks;
    uint8_t *unit = out + ((long long)strip * a.units + block / a.unit_blocks) * a.unit_bytes;
    uint32_t words[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        words[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {                        // input j & 3 of the word, channel g + 8 (j >> 2)
            const int row = strip * kStrip + g + (j >> 2) * 8, col = block * kStep + (i >> 1) * 32 + 8 * t + (i & 1) * 4 + (j & 3);
            const int code = row < a.n && col < a.k ? min(max((int)w[row * ldw + col], -8), 7) : 0;
            const int nibble = (j & 1) * 4 + ((j >> 1) & 1) * 2 + (j >> 2);
            words[i] |= (uint32_t)(code + 8) << (4 * nibble);
        }
    }
    reinterpret_cast<uint4 *>(unit + 512 * in_unit)[lane] = make_uint4(words[0], words[1], words[2], words[3]);
    const int row = strip * kStrip + (lane & 15), k = block * kStep + 32 * (lane >> 4);
    if (in_unit == 0 && lane < kStrip * a.unit_scales)
        reinterpret_cast<float *>(unit + 512 * a.unit_blocks)[lane] = row < a.n && k < a.k ? scales[row * lds + k / a.group] : 0.0f;
}

// A CTA per row: transformed in shared memory, then a warp per group.
template <typename T>
__global__ void __launch_bounds__(256) quantize_groups_kernel(const T *w, long long ldw, int k, int hb, int group, float inv_norm,
                                                              int8_t *codes, long long ldc, float *scales, long long lds) {
    extern __shared__ float t[];
    const long long row = blockIdx.x;
    for (int i = threadIdx.x; i < k; i += 256) t[i] = to_f32<T>(w[row * ldw + i]);
    __syncthreads();
    for (int h = 1; h < hb; h *= 2) {
        for (int i = threadIdx.x; i < k / 2; i += 256) {
            const int at = i / h * 2 * h + i % h;
            const float x = t[at], y = t[at + h];
            t[at] = x + y;
            t[at + h] = x - y;
        }
        __syncthreads();
    }
    const int lane = threadIdx.x & 31, groups = (k - 1) / group + 1;              // (k + group may be beyond an int)
    for (int g = threadIdx.x >> 5; g < groups; g += 8) {
        const int from = g * group, to = k - from > group ? from + group : k;
        float most = 0.0f;
        for (int i = from + lane; i < to; i += 32) {
            const float v = fabsf(t[i]);
            most = v != v ? INFINITY : fmaxf(most, v);
        }
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
        const bool sound = 7.0f * most < INFINITY, some = sound && most > 0.0f;
        for (int i = from + lane; i < to; i += 32)
            codes[row * ldc + i] = some ? (int8_t)rintf(__fdiv_rn(7.0f * t[i], most)) : (int8_t)0;
        if (lane == 0)
            scales[row * lds + g] = !sound ? __int_as_float(0x7fffffff) : some ? __fdiv_rn(most, 7.0f) * inv_norm : inv_norm;
    }
}

template <typename T>
cudaError_t quantize_type(const void *w, long long ldw, int n, int k, int hb, int group, int8_t *codes, long long ldc, float *scales,
                          long long lds, cudaStream_t s) {
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(quantize_groups_kernel<T>), k * 4, allowed);
    if (e != cudaSuccess) return e;
    quantize_groups_kernel<T><<<(unsigned)n, 256, (size_t)k * 4, s>>>(static_cast<const T *>(w), ldw, k, hb, group,
                                                                    (float)(1.0 / sqrt((double)hb)), codes, ldc, scales, lds);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_linear4(const Linear4Args &a, int x_type, int sms, cudaStream_t s) {
    return x_type == HATQ_F32 ? launch_type<float>(a, sms, s) : x_type == HATQ_F16 ? launch_type<__half>(a, sms, s) : launch_type<__nv_bfloat16>(a, sms, s);
}
cudaError_t launch_linear4_layout(const int8_t *w, long long ldw, const float *scales, long long lds, const Linear4Args &a, uint8_t *out,
                                  cudaStream_t s) {
    const long long blocks = (long long)a.strips * a.units * a.unit_blocks;
    layout_kernel<<<(unsigned)((blocks + 7) / 8), 256, 0, s>>>(w, ldw, scales, lds, a, out);
    return cudaGetLastError();
}
cudaError_t launch_quantize_groups(const void *w, int type, long long ldw, int n, int k, int hb, int group, int8_t *codes,
                                   long long ldc, float *scales, long long lds, cudaStream_t s) {
    return type == HATQ_F32    ? quantize_type<float>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s)
           : type == HATQ_F16 ? quantize_type<__half>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s)
                              : quantize_type<__nv_bfloat16>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s);
}

}  // namespace hatq
