// Attention over the 4-bit cache for many queries per sequence, on the fifth-generation tensor cores.
#include "hatq_cache.h"
#include "hatq_mma4.h"
#include "hatq_sequences.h"
#include "hatq_tc.h"

namespace hatq {
namespace {

using tc::elect_one;
using tc::mbar_arrive;
using tc::mbar_expect_tx;
using tc::mbar_init;
using tc::mbar_wait;
using tc::smem_addr;

// The formulas of hatq_attend.cu for two tiles of 128 query columns of a kv head at a time: S = Q K^T (128 x 64 keys),
// O += P V (128 x D), Q and P in tensor memory (of heads of 128 the second tile's Q has no room there and is in shared
// memory), codes widened once for both tiles into shared memory. bf16 queries only:
// rounded to fp16 are q and p as there, and here also code times scale of keys and of values (an error of 2^-12 each,
// against 2^-9 of the output), so that a logit costs one instruction less than it would with a factor of its key.
//
// Scales are brought into fp16's range by powers of two. A chunk has one power for its keys, a factor of the logits, where the
// scales of those lie within 2^10 of the largest (a scale in two parts then keeps 15 bits), and one for its values, a factor of
// the weights, where those do within 2^13 (code times scale is then a normal number, and what a row's own largest term is
// rounded by at most 2^-18 of it). Otherwise every token has its own
// two, which the rows apply one by one, to this chunk and those behind it, as where logits are beyond 2^13. A row has two references: m for the sum of its weights, and
// m + vm for their products with the values' powers, which it raises by what it sees alone, to where they are below 2^8: what
// they keep is relative to the largest term of the row's own sum, whatever the scales of tokens that it does not see. A token
// whose value codes are all 0 has no power (append gives rows of zeros a scale like any other).
// A token whose scales are not finite gets values of 0 and keys of NaN, so that it makes NaN exactly of the rows that see it
// (0 times NaN in a masked place would do so of all).
//
// Roles: 4 warps per tile have a row a thread (transform of the query, softmax, transform back), twice 4 warps widen chunks
// of 64 keys in turn, one warp brings them in and one looks their scales over, one per tile issues its MMAs: S of the next
// chunk as soon as the rows have read this one's, PV when the weights are there. Two tiles share what is widened.
//
// Bound by the rows' softmax: per chunk and two tiles the tensor cores have 1200 cycles of work, a chunk takes 2500 (2048
// queries, the last of 8192 tokens, and 889 of 3445, 32 heads over 8: 326 us, 870 TFLOP/s, tensor pipe 0.41, issue 0.53).
constexpr int kRaw = 4;                // chunks on their way or being widened
constexpr int kWide = 4;               // widened chunks
constexpr int kInfo = kRaw + kWide;    // a chunk is brought in when the one this many before has been multiplied
// Five groups of four warps. Registers are handed on between them: 640 x 96 at launch.
constexpr int kPromptThreads = 20 * 32, kRegsLaunch = 96, kRegsRows = 136, kRegsWiden = 72, kRegsRest = 56;
static_assert(256 * kRegsRows + 256 * kRegsWiden + 128 * kRegsRest <= kPromptThreads * kRegsLaunch, "setmaxnreg waits for registers that there are");

template <int D>
struct Shape {
    static constexpr int kChunkBytes = kChunk * (D + 8), kK = kChunk * D * 2, kKV = 2 * kK;
    // columns of tensor memory: two tiles each of D, 64, 32; then Q, D / 2 a tile, of the second where that is left
    static constexpr int kO = 0, kS = 2 * D, kP = kS + 128, kQ = kP + 64;
    static constexpr bool kSecond = kQ + D <= 512;
    static constexpr int kQBytes = kSecond ? 0 : 128 * D * 2;
    static constexpr int kBytes = 1024 + kQBytes + kWide * kKV + kRaw * kChunkBytes;
};

struct alignas(16) Info {              // of a widened chunk, for the rows
    float k_factor;                    // 2^(exponent of the keys' scales)
    int v_exponent;                    // of the values' scales, as a float's; or kNoOne, where they or the keys' are far apart
    unsigned held[2];                  // keys that are there
};
struct alignas(16) Powers {            // the same of every token
    float k_factor[kChunk], v_power[kChunk];
};
struct alignas(16) Scaled {            // what the powers leave of the scales, for the widening warps
    float k[kChunk];
    __half v[kChunk];
};
constexpr int kKeysApart = 10, kValuesApart = 13, kNoOne = 1 << 20;
constexpr float kNoPower = -10000.0f;  // of values of 0
constexpr float kLowest = -3.402823466e38f;  // below every logit
constexpr int kLeastV = -1000;         // below any product's power

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two fp32 numbers in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t x, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ float power(int exponent) { return __int_as_float(exponent << 23); }      // 1 .. 254
__device__ __forceinline__ void butterflies(float (&v)[64], int hb) {
#pragma unroll
    for (int h = 1; h < 64; h *= 2)
        if (h < hb)
#pragma unroll
            for (int i = 0; i < 64; ++i)
                if (!(i & h)) {
                    const float x = v[i], y = v[i + h];
                    v[i] = x + y;
                    v[i + h] = x - y;
                }
}
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!tc::mbar_try_wait(bar, parity) && clock64() - t0 < tc::kWaitLimitCycles) {}
}

template <int N, bool MORE>
__device__ __forceinline__ void set_regs() {
    if constexpr (MORE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

template <int D>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_kernel(const AttendArgs a) {
    using S = Shape<D>;
    constexpr int GROUPS = D / 8;                            // of 8 neighbouring values
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t s_bars[3 * kRaw + 2 * kWide + 11];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_pages[kRaw];
    __shared__ Info s_info[kInfo];
    __shared__ Powers s_powers[kInfo];
    __shared__ Scaled s_scaled[kRaw];
    uint8_t *smem = smem_raw + (-smem_addr(smem_raw) & 1023u);
    uint8_t *wide = smem + S::kQBytes, *raw = wide + kWide * S::kKV;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const CacheArgs &c = a.c;
    volatile int *abort_flag = &s_abort;
    const uint32_t bars = smem_addr(s_bars);
    auto raw_full = [&](int i) { return bars + 8 * i; };
    auto raw_free = [&](int i) { return bars + 8 * (kRaw + i); };
    auto kv_full = [&](int i) { return bars + 8 * (2 * kRaw + i); };
    auto kv_free = [&](int i) { return bars + 8 * (2 * kRaw + kWide + i); };
    constexpr int kRest = 2 * kRaw + 2 * kWide;
    auto s_full = [&](int i) { return bars + 8 * (kRest + i); };
    auto p_full = [&](int i) { return bars + 8 * (kRest + 2 + i); };
    auto o_full = [&](int i) { return bars + 8 * (kRest + 4 + i); };
    auto s_free = [&](int i) { return bars + 8 * (kRest + 6 + i); };
    auto tail = [&](int i) { return bars + 8 * (kRest + 8 + i); };
    const uint32_t q_full = bars + 8 * (kRest + 10);
    auto scaled_full = [&](int i) { return bars + 8 * (kRest + 11 + i); };
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int i = 0; i < kRaw; ++i) {
            mbar_init(raw_full(i), 1);
            mbar_init(raw_free(i), 4);
            mbar_init(scaled_full(i), 1);
        }
        for (int i = 0; i < kWide; ++i) {
            mbar_init(kv_full(i), 4);
            mbar_init(kv_free(i), 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full(i), 1);
            mbar_init(s_free(i), 4);
            mbar_init(p_full(i), 4);
            mbar_init(o_full(i), 1);
            mbar_init(tail(i), 1);
        }
        mbar_init(q_full, 8);
        tc::fence_barrier_init();
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    after_prior_kernels();
    const int err = *reinterpret_cast<volatile int *>(a.err);
    // ---- the CTA's sequence, head and columns; of a sequence the last columns, which see most, come first
    Row<kPromptColumns> row;
    row.read(c, a.group, lane, true);
    const bool work = blockIdx.x < row.total;
    Sequence seq{};
    if (work) row.find_unit(c, a.group, lane, blockIdx.x, seq);
    const int rank = work ? (int)(blockIdx.x - seq.unit) : 0, head = rank % c.heads, x0 = (seq.tiles - 1 - rank / c.heads) * kPromptColumns;
    const int columns = min((long long)seq.m * a.group - x0, (long long)kPromptColumns), last_token = (x0 + columns - 1) / a.group;
    const int tiles = columns > 128 ? 2 : 1;
    tc::tc_fence_before();
    const bool skip = __syncthreads_or(err != 0) || !work;
    tc::tc_fence_after();
    const uint32_t tmem = s_tmem;
    // chunks that some column sees
    const int chunks = skip ? 0 : max(0, (seq.len - seq.m + last_token) / kChunk + (seq.len - seq.m + last_token >= 0 ? 1 : 0));
    const int size = 1 << c.page_bits, pages_of_chunk = kChunk >> c.page_bits;
    const uint32_t record = (uint32_t)size * (D + 8);
    bool ok = true;

    if (warp >= 16) set_regs<kRegsRest, false>();
    if (warp == 16) {
        // ---- chunks from the cache
        int issued = 0;
        for (; issued < chunks; ++issued) {
            const int stage = issued % kRaw, first = issued * pages_of_chunk;
            const int page = lane < pages_of_chunk && first + lane < c.table_width ? c.table[seq.b * c.ldt + first + lane] : -1;
            const bool take = issued * kChunk + lane * size < seq.len && page >= 0 && page < c.pages;
            const unsigned pages = __ballot_sync(0xffffffffu, take);
            if (issued >= kRaw) ok = mbar_wait(raw_free(stage), (uint32_t)(issued / kRaw - 1) & 1u, abort_flag, a.err);
            if (!__all_sync(0xffffffffu, ok)) break;
            if (lane == 0) {
                s_pages[stage] = (int)pages;
                mbar_expect_tx(raw_full(stage), (uint32_t)__popc(pages) * record);
            }
            __syncwarp();
            if (take)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                 smem_addr(raw + stage * S::kChunkBytes + lane * record)),
                             "l"(c.data + ((long long)page * c.heads + head) * record), "r"(record), "r"(raw_full(stage))
                             : "memory");
        }
        // copies land before the CTA leaves, whoever gave up
        for (int i = max(0, issued - kRaw); i < issued; ++i) drain(raw_full(i % kRaw), (uint32_t)(i / kRaw) & 1u);
    } else if (warp == 17 || warp == 18) {
        // ---- MMAs of a tile. (One warp for both took 1750 cycles a chunk: a wait, a fence and a commit cost it about 300.)
        const int tile = warp - 17;
        const uint32_t s_idesc = tc::idesc_f16(kChunk), o_idesc = tc::idesc_f16(D);
        const uint64_t q0 = tc::sdesc_sw128(smem_addr(smem)), wide0 = tc::sdesc_sw128(smem_addr(wide));
        auto issue_s = [&](int i) {
            if (elect_one()) {
                const uint64_t k0 = wide0 + (uint64_t)(i % kWide * (S::kKV >> 4));
                const uint32_t d = tmem + S::kS + 64 * tile;
                if (tile == 0 || S::kSecond) {
#pragma unroll
                    for (int j = 0; j < D / 16; ++j)
                        tc::umma_f16_ts(d, tmem + S::kQ + D / 2 * tile + 8 * j, k0 + (uint64_t)((j / 4) * 512 + 2 * (j % 4)), s_idesc, j > 0);
                } else {
#pragma unroll
                    for (int j = 0; j < D / 16; ++j)
                        tc::umma_f16_ss(d, q0 + (uint64_t)((j / 4) * 1024 + 2 * (j % 4)), k0 + (uint64_t)((j / 4) * 512 + 2 * (j % 4)), s_idesc, j > 0);
                }
                tc::umma_commit(s_full(tile));
            }
            __syncwarp();
        };
        const int mine = tile < tiles ? chunks : 0;
        if (mine) {
            ok = mbar_wait(q_full, 0, abort_flag, a.err) && mbar_wait(kv_full(0), 0, abort_flag, a.err);
            ok = __all_sync(0xffffffffu, ok);
            tc::tc_fence_after();
            if (ok) issue_s(0);
        }
        for (int i = 0; i < mine && ok; ++i) {
            if (i + 1 < chunks) {
                // S of the next chunk as soon as the rows have read this one's
                ok = mbar_wait(s_free(tile), (uint32_t)i & 1u, abort_flag, a.err) &&
                     mbar_wait(kv_full((i + 1) % kWide), (uint32_t)((i + 1) / kWide) & 1u, abort_flag, a.err);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc::tc_fence_after();
                issue_s(i + 1);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(p_full(tile), (uint32_t)i & 1u, abort_flag, a.err));
            if (!ok) break;
            tc::tc_fence_after();
            if (elect_one()) {
                const uint64_t v0 = wide0 + (uint64_t)(i % kWide * (S::kKV >> 4) + (S::kK >> 4));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    tc::umma_f16_ts(tmem + S::kO + D * tile, tmem + S::kP + 32 * tile + 8 * j, v0 + (uint64_t)(2 * j), o_idesc, i > 0 || j > 0);
                tc::umma_commit(o_full(tile));
                tc::umma_commit(kv_free(i % kWide));
                if (tiles == 1) mbar_arrive(kv_free(i % kWide));          // (no other tile's)
            }
            __syncwarp();
        }
        if (elect_one()) tc::umma_commit(tail(tile));
        __syncwarp();
        drain(tail(tile), 0);
    } else if (warp == 19) {
        // ---- scales
        for (int i = 0; i < chunks; ++i) {
            const int stage = i % kRaw;
            ok = mbar_wait(raw_full(stage), (uint32_t)(i / kRaw) & 1u, abort_flag, a.err);
            if (!__all_sync(0xffffffffu, ok)) break;
            const uint8_t *chunk = raw + stage * S::kChunkBytes;
            const int pages = s_pages[stage], left = seq.len - i * kChunk;
            // tokens lane and lane + 32: 0 where it is none; NaN of the keys' where either is not finite
            float k[2], v[2];
            unsigned held[2];
            int ke[2], ve[2];                                // exponents; of 0 and NaN 0, which set nothing
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 32 * h, in_page = j >> c.page_bits;
                const uint8_t *at = chunk + in_page * record + size * D + 4 * (j & (size - 1));
                const bool there = (pages >> in_page & 1) && j < left;
                k[h] = *reinterpret_cast<const float *>(at);
                v[h] = *reinterpret_cast<const float *>(at + 4 * size);
                const bool sound = fabsf(k[h]) < __int_as_float(0x7f800000) && fabsf(v[h]) < __int_as_float(0x7f800000);
                if (!there) k[h] = 0.0f;
                else if (!sound) k[h] = __int_as_float(0x7fffffff);
                if (!there || !sound) v[h] = 0.0f;
                held[h] = __ballot_sync(0xffffffffu, there);
                ke[h] = k[h] == k[h] ? min((int)(__float_as_uint(k[h]) >> 23 & 255u), 253) : 0;
                ve[h] = min((int)(__float_as_uint(v[h]) >> 23 & 255u), 253);
            }
            auto far = [](const float (&x)[2], const int (&e)[2], int least) {
                return __any_sync(0xffffffffu, (x[0] > 0.0f && e[0] < least) || (x[1] > 0.0f && e[1] < least)) != 0;
            };
            auto largest = [](const int (&e)[2]) { return (int)max(__reduce_max_sync(0xffffffffu, max(e[0], e[1])), 1); };
            auto codes = [&](int j) { return chunk + (j >> c.page_bits) * record + (size + (j & (size - 1))) * (D / 2); };
            const int k_exponent = largest(ke);
            const bool k_apart = far(k, ke, k_exponent - kKeysApart);
            int v_exponent = largest(ve);
            bool v_apart = far(v, ve, v_exponent - kValuesApart);
            // Values of 0 have no power: all are looked for where any counts, or where the token that has the largest is one.
            const unsigned top[2] = {__ballot_sync(0xffffffffu, ve[0] == v_exponent), __ballot_sync(0xffffffffu, ve[1] == v_exponent)};
            const int at = top[0] ? __ffs(top[0]) - 1 : top[1] ? 31 + __ffs(top[1]) : 0;
            const bool some = __any_sync(0xffffffffu, *reinterpret_cast<const uint32_t *>(codes(at) + 4 * (lane & (D / 8 - 1))) != 0x88888888u);
            if (v_apart || !some) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t z = 0;
#pragma unroll
                    for (int x = 0; x < D / 2; x += 16) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(codes(lane + 32 * h) + x);
                        z |= (u.x ^ 0x88888888u) | (u.y ^ 0x88888888u) | (u.z ^ 0x88888888u) | (u.w ^ 0x88888888u);
                    }
                    if (z == 0) v[h] = 0.0f, ve[h] = 0;
                }
                v_exponent = largest(ve);
                v_apart = far(v, ve, v_exponent - kValuesApart);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kp = k_apart ? max(ke[h], 1) : k_exponent, vp = v_apart ? max(ve[h], 1) : v_exponent;
                s_scaled[stage].k[lane + 32 * h] = k[h] * power(254 - kp);
                s_scaled[stage].v[lane + 32 * h] = __float2half_rn(v[h] * power(254 - vp));
                s_powers[i % kInfo].k_factor[lane + 32 * h] = power(kp);
                s_powers[i % kInfo].v_power[lane + 32 * h] = v[h] > 0.0f ? (float)vp : kNoPower;
            }
            if (lane == 0) {
                Info info;
                info.k_factor = power(k_exponent);
                info.v_exponent = k_apart || v_apart ? kNoOne : v_exponent;
                info.held[0] = held[0];
                info.held[1] = held[1];
                s_info[i % kInfo] = info;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(scaled_full(stage));
        }
    } else if (warp >= 8) {
        set_regs<kRegsWiden, false>();
        // ---- widening: four warps take every other chunk
        const int tid = threadIdx.x & 127, part = tid >> 6, key = tid & 63;
        const int dg = lane % GROUPS, tg = (tid >> 5) * 2 + (lane / GROUPS & 1);
        const bool has_v = GROUPS == 16 || lane < 16;
        for (int i = (warp >> 2) & 1; i < chunks; i += 2) {
            const int stage = i % kRaw, buf = i % kWide;
            ok = mbar_wait(raw_full(stage), (uint32_t)(i / kRaw) & 1u, abort_flag, a.err) &&
                 mbar_wait(scaled_full(stage), (uint32_t)(i / kRaw) & 1u, abort_flag, a.err);
            if (ok && i >= kWide) ok = mbar_wait(kv_free(buf), (uint32_t)(i / kWide - 1) & 1u, abort_flag, a.err);
            if (!__all_sync(0xffffffffu, ok)) break;
            const uint8_t *chunk = raw + stage * S::kChunkBytes;
            const Scaled &scaled = s_scaled[stage];
            uint8_t *K = wide + buf * S::kKV, *V = K + S::kK;
            {
                // keys: row = key, values in the order 0 4 1 5 2 6 3 7 of each 8, as the queries have them
                // The scale as two fp16, so that a product is rounded once: an error of the scale itself would be that of a
                // whole logit (8 rows of 1000 .. 8000 keys: 2.1e-3 off in all, against 1.8e-3).
                const float by = scaled.k[key], high = __half2float(__float2half_rn(by));
                const uint32_t scale = pack_half(by, by), rest = pack_half(by - high, by - high);
                auto product = [&](uint32_t codes) { return fma2(codes, scale, mul2(codes, rest)); };
                const uint8_t *at = chunk + (key >> c.page_bits) * record + (key & (size - 1)) * (D / 2) + part * (D / 4);
                uint32_t w[D / 16];
#pragma unroll
                for (int j = 0; j < D / 16; j += 4) *reinterpret_cast<uint4 *>(w + j) = *reinterpret_cast<const uint4 *>(at + 4 * j);
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const uint32_t u = w[j] >> 8;
                    const int word = part * (D / 16) + j;
                    const uint4 o = make_uint4(product(codes_f16<true, false>(w[j])), product(codes_f16<true, true>(w[j])),
                                               product(codes_f16<true, false>(u)), product(codes_f16<true, true>(u)));
                    *reinterpret_cast<uint4 *>(K + (word >> 3) * 8192 + key * 128 + (((word & 7) ^ (key & 7)) << 4)) = o;
                }
            }
            if (has_v) {
                // values, transposed: 8 tokens of 8 values; value 8 dg + j is row j GROUPS + dg
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int token = tg * 8 + j;
                    w[j] = *reinterpret_cast<const uint32_t *>(chunk + (token >> c.page_bits) * record + (size + (token & (size - 1))) * (D / 2) + 4 * dg);
                }
                const uint4 pairs = *reinterpret_cast<const uint4 *>(scaled.v + tg * 8);
                const uint32_t scale[4] = {pairs.x, pairs.y, pairs.z, pairs.w};
                uint32_t o[8][4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t n = __byte_perm(w[2 * j], w[2 * j + 1], half ? 0x7632 : 0x5410), u = n >> 8;
                        o[4 * half][j] = mul2(codes_f16<true, false>(n), scale[j]);
                        o[4 * half + 1][j] = mul2(codes_f16<true, true>(n), scale[j]);
                        o[4 * half + 2][j] = mul2(codes_f16<true, false>(u), scale[j]);
                        o[4 * half + 3][j] = mul2(codes_f16<true, true>(u), scale[j]);
                    }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int n = j * GROUPS + dg;
                    *reinterpret_cast<uint4 *>(V + n * 128 + ((tg ^ (n & 7)) << 4)) = make_uint4(o[j][0], o[j][1], o[j][2], o[j][3]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(kv_full(buf));
                mbar_arrive(raw_free(stage));
            }
        }
    } else {
        set_regs<kRegsRows, true>();
        // ---- a row a thread
        const int tile = warp >> 2, x = x0 + threadIdx.x, token = x / a.group, q_head = head * a.group + x - token * a.group;
        const bool live = !skip && token < seq.m;
        const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        float f = 0.0f;
        const bool here = !skip && tile < tiles;
        if (here && chunks) {
            // The query, transformed; its halves of 64 one after the other (of 128 in a block: sums, then differences).
            const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(a.q) + (long long)(seq.begin + (live ? token : 0)) * a.ldq +
                                     (long long)(live ? q_head : 0) * a.hq;
            auto load8 = [&](int i, uint32_t (&w)[4]) {
                if (a.vec) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i);
                    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                } else {
                    const unsigned short *u = reinterpret_cast<const unsigned short *>(p) + 8 * i;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = u[2 * j] | (uint32_t)u[2 * j + 1] << 16;
                }
            };
            uint32_t most = 0;
#pragma unroll 4
            for (int i = 0; i < GROUPS; ++i) {
                uint32_t w[4];
                load8(i, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) most = __vmaxu2(most, w[j] & 0x7fff7fffu);
            }
            // below 2^10 by a power of two; an infinity or a NaN makes the row NaN
            const int log_hb = 31 - __clz(c.hb), ex = max((int)(max(most & 0xffffu, most >> 16) >> 7), 10);
            const float by = !live ? 0.0f : ex == 255 ? __int_as_float(0x7fffffff) : copysignf(power(263 - log_hb - ex), a.scale);
            f = fabsf(a.scale) * c.inv_norm * power(min(ex, 254) + log_hb - 9);
#pragma unroll
            for (int half = 0; half < D / 64; ++half) {
                float v[64];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t w[4], u[4];
                    load8(D == 128 && c.hb <= 64 ? 8 * half + i : i, w);
                    if (D == 128 && c.hb == 128) load8(8 + i, u);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                        v[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                        if (D == 128 && c.hb == 128) {
                            const float y = __uint_as_float(u[j] << 16), z = __uint_as_float(u[j] & 0xffff0000u);
                            v[8 * i + 2 * j] += half ? -y : y;
                            v[8 * i + 2 * j + 1] += half ? -z : z;
                        }
                    }
                }
                butterflies(v, c.hb);
                uint32_t r[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const int d = (i >> 2) * 8 + (i & 3);
                    r[i] = pack_half(live ? v[d] * by : 0.0f, live ? v[d + 4] * by : 0.0f);
                }
                if (tile == 0 || S::kSecond) {
                    tc::tmem_st32(at + S::kQ + D / 2 * tile + 32 * half, r);
                } else {
                    // a panel of 64 values: rows of 128 bytes, 16-byte pieces exchanged by the row
                    const int of = threadIdx.x & 127;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4 *>(smem + half * 16384 + of * 128 + ((i ^ (of & 7)) << 4)) =
                            make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                }
            }
            tc::tmem_wait_st();
            tc::tc_fence_before();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
        // ---- softmax
        const int position = live ? seq.len - seq.m + token : 0x7fffffff;          // (rows that are none: nothing to mask)
        const int lowest = __reduce_min_sync(0xffffffffu, position);
        float m = kLowest, l = 0.0f;
        int vm = kLeastV;
        // A row's keys of a chunk: all of them (true), or the ones that it sees.
        auto look = [&](int i, const Info &info, unsigned (&seen)[2]) {
            seen[0] = seen[1] = 0xffffffffu;
            if (i * kChunk + kChunk - 1 <= lowest && (info.held[0] & info.held[1]) == 0xffffffffu) return true;
            const int ends = min(max(position - i * kChunk, -1), kChunk - 1) + 1;                    // keys before it
            seen[0] = info.held[0] & (ends >= 32 ? 0xffffffffu : (1u << ends) - 1u);
            seen[1] = info.held[1] & (ends >= 64 ? 0xffffffffu : ends <= 32 ? 0u : (1u << (ends - 32)) - 1u);
            return false;
        };
        // the last chunk's weights are used, and O is there
        auto wait_used = [&](int i) {
            if (i > 0) ok = __all_sync(0xffffffffu, mbar_wait(o_full(tile), (uint32_t)(i - 1) & 1u, abort_flag, a.err));
            tc::tc_fence_after();
        };
        // New references: now for m, and for the products one that they, at most 2^(now + more), exceed by 15 at most. (What l
        // loses vm takes up: a later, heavier token may be a far smaller one.)
        auto raise = [&](int i, float now, float more) {
            int next = max(vm + (int)fmaxf(floorf(m - now), (float)kLeastV), kLeastV);
            if (more > (float)(next + 15)) next = (int)ceilf(more) - 7;
            const float o_by = exp2_fast(m - now + (float)(vm - next));
            l *= exp2_fast(m - now);
            m = now;
            vm = next;
            if (i == 0) return;
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
                uint32_t o[32];
                tc::tmem_ld32(at + S::kO + D * tile + d, o);
                tc::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * o_by);
                tc::tmem_st32(at + S::kO + D * tile + d, o);
            }
            tc::tmem_wait_st();
        };
        auto written = [&]() {
            tc::tmem_wait_st();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full(tile));
        };
        // A chunk whose scales have a power together. False where they have not or logits are too large, and nothing done, or where
        // a wait gave up.
        auto together = [&](int i) {
            ok = __all_sync(0xffffffffu, mbar_wait(s_full(tile), (uint32_t)i & 1u, abort_flag, a.err));
            if (!ok) return false;
            tc::tc_fence_after();
            const Info info = s_info[i % kInfo];
            const float fs = f * info.k_factor;
            uint32_t s[64];
            tc::tmem_ld32(at + S::kS + 64 * tile, *reinterpret_cast<uint32_t (*)[32]>(s));
            tc::tmem_ld32(at + S::kS + 64 * tile + 32, *reinterpret_cast<uint32_t (*)[32]>(s + 32));
            tc::tmem_wait_ld();
            unsigned seen[2];
            const bool whole = look(i, info, seen);
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (!(seen[j >> 5] >> (j & 31) & 1)) s[j] = __float_as_uint(-3e38f);
            }
            float most = -3e38f;
#pragma unroll
            for (int j = 0; j < 64; j += 2) most = max3(most, __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
            const float top = most > -3e38f ? most * fs : kLowest;           // (none seen that is a number)
            if (__any_sync(0xffffffffu, top > m + (float)min(8, vm + 15 - info.v_exponent) || info.v_exponent == kNoOne)) {
                const float now = top > m + 8.0f ? top : m;
                // (beyond 2^13 m has no bits for what weights carry beside it)
                if (info.v_exponent == kNoOne || __any_sync(0xffffffffu, fabsf(now) > 8192.0f && now != kLowest)) return false;
                wait_used(i);
                if (!ok) return false;
                raise(i, now, top - now + (float)info.v_exponent);
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(s_free(tile));
            // weights carry what the chunk's values are brought to (2^-64 of the largest is nothing in fp16, but counts in l)
            const int less = max(info.v_exponent - vm, -64);
            const float shift = m - (float)less;
            uint64_t sum[2] = {0, 0};
            uint32_t p[32];
            const uint64_t by2 = pair(fs, fs), less2 = pair(-shift, -shift);
#pragma unroll
            for (int j = 0; j < 64; j += 2) {
                float u, v;
                unpair(fma_pair(pair(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), by2, less2), u, v);
                s[j] = __float_as_uint(exp2_fast(u));
                s[j + 1] = __float_as_uint(exp2_fast(v));
            }
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (!(seen[j >> 5] >> (j & 31) & 1)) s[j] = 0;
            }
#pragma unroll
            for (int j = 0; j < 64; j += 2) {
                const float u = __uint_as_float(s[j]), v = __uint_as_float(s[j + 1]);
                sum[j / 2 % 2] = add_pair(sum[j / 2 % 2], pair(u, v));
                p[j / 2] = pack_half(u, v);
            }
            float s0, s1;
            unpair(add_pair(sum[0], sum[1]), s0, s1);
            l = fmaf(s0 + s1, power(127 - min(less, 126)), l);
            wait_used(i);
            if (!ok) return false;
            tc::tmem_st32(at + S::kP + 32 * tile, p);
            written();
            return true;
        };
        // Any chunk, every token with its own powers: two or three times over the logits, 8 at a time, a third of the speed. (Few instructions: they
        // are in the way of the others even where no chunk comes here, 16 at a time 371 us instead of 327.)
        auto apart = [&](int i) {
            ok = __all_sync(0xffffffffu, mbar_wait(s_full(tile), (uint32_t)i & 1u, abort_flag, a.err));
            if (!ok) return;
            tc::tc_fence_after();
            const Info info = s_info[i % kInfo];
            const Powers &powers = s_powers[i % kInfo];
            unsigned seen[2];
            look(i, info, seen);
            uint32_t s[8];
            auto pass = [&](auto use) {
#pragma unroll 1
                for (int from = 0; from < 64; from += 8) {
                    tc::tmem_ld8(at + S::kS + 64 * tile + from, s);
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[j] = __float_as_uint(__fmul_rn(__uint_as_float(s[j]), f * powers.k_factor[from + j]));      // (rounded: equal ones stay equal)
                    use(from, (from < 32 ? seen[0] : seen[1]) >> (from & 31));
                }
            };
            float top = kLowest, more = kLowest, now = m, sum = 0.0f;
            auto largest = [&](int from, unsigned mask) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (mask >> j & 1) {
                        top = fmaxf(top, __uint_as_float(s[j]));
                        more = fmaxf(more, __uint_as_float(s[j]) - now + powers.v_power[from + j]);
                    }
            };
            pass(largest);
            if (top > m + 8.0f) {
                now = top;
                more = kLowest;
            }
            if (__any_sync(0xffffffffu, now != m)) pass(largest);
            wait_used(i);
            if (!ok) return;
            if (__any_sync(0xffffffffu, now != m || more > (float)(vm + 15))) raise(i, now, more);
            pass([&](int from, unsigned mask) {
                uint32_t p[4];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    float w[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float x = __uint_as_float(s[j + y]) - m;
                        const bool in = mask >> (j + y) & 1;
                        sum += in ? exp2_fast(x) : 0.0f;
                        w[y] = in ? exp2_fast(x + (powers.v_power[from + j + y] - (float)vm)) : 0.0f;
                    }
                    p[j / 2] = pack_half(w[0], w[1]);
                }
                tc::tmem_st4(at + S::kP + 32 * tile + from / 2, p);
            });
            l += sum;
            written();
            if (lane == 0) mbar_arrive(s_free(tile));
        };
        // (Two loops one after the other: the second's body within the first takes registers from it, 361 us instead of 327.)
        const int mine = here ? chunks : 0;
        int i = 0;
        while (i < mine && together(i)) ++i;
#pragma unroll 1
        for (; i < mine && ok; ++i) apart(i);
        // ---- the row's output
        ok = __all_sync(0xffffffffu, ok);
        if (here && chunks && ok) {
            ok = __all_sync(0xffffffffu, mbar_wait(o_full(tile), (uint32_t)(chunks - 1) & 1u, abort_flag, a.err));
            tc::tc_fence_after();
        }
        if (here && ok) {
            // 2^(vm - 127), in two factors: vm may be below or above what one can be
            const int v0 = (vm - 127) >> 1, v1 = vm - 127 - v0;
            const float by = (l == 0.0f ? 0.0f : c.inv_norm / l) * power(max(127 + v0, 1)), unit = power(max(127 + v1, 1));
            __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(a.out) + (long long)(seq.begin + (live ? token : 0)) * a.ldo +
                                 (long long)(live ? q_head : 0) * a.ho;
#pragma unroll 1
            for (int half = 0; half < D / 64; ++half) {
                float v[64];
                constexpr int PER = 32 / GROUPS;             // values j of each group in 32 columns
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    uint32_t o[32];
                    if (chunks) {
                        tc::tmem_ld32(at + S::kO + D * tile + 32 * j, o);
                        tc::tmem_wait_ld();
                    }
#pragma unroll
                    for (int y = 0; y < PER; ++y)
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            float u = __uint_as_float(o[y * GROUPS + g]);
                            if (D == 128) {
                                const float z = __uint_as_float(o[y * GROUPS + (GROUPS - 8) + g]);
                                u = c.hb == 128 ? (half ? u - z : u + z) : half ? z : u;
                            }
                            v[8 * g + PER * j + y] = chunks ? u : 0.0f;
                        }
                }
                butterflies(v, c.hb);
                if (live) {
                    union { uint4 u[8]; __nv_bfloat16 t[64]; } y;
#pragma unroll
                    for (int d = 0; d < 64; ++d) y.t[d] = from_f32<__nv_bfloat16>(v[d] * by * unit);
                    if (a.vec_out) {
#pragma unroll
                        for (int d = 0; d < 8; ++d) reinterpret_cast<uint4 *>(out + 64 * half)[d] = y.u[d];
                    } else {
#pragma unroll
                        for (int d = 0; d < 64; ++d) out[64 * half + d] = y.t[d];
                    }
                }
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 17)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <int D>
cudaError_t launch(const AttendArgs &a, cudaStream_t s) {
    // shares of registers that the launch does not bring would be waited for forever
    static const int regs = [] {
        cudaFuncAttributes fa{};
        return cudaFuncGetAttributes(&fa, prompt_kernel<D>) == cudaSuccess ? fa.numRegs : 0;
    }();
    if (regs != kRegsLaunch) return cudaErrorInvalidConfiguration;
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(prompt_kernel<D>), Shape<D>::kBytes, allowed);
    if (e != cudaSuccess) return e;
    const long long tasks = a.c.heads * ((long long)a.c.rows * a.group / kPromptColumns + min(a.c.seqs, a.c.rows));
    return launch_early(prompt_kernel<D>, dim3((unsigned)tasks), kPromptThreads, Shape<D>::kBytes, s, a);
}

}  // namespace

// Where a CTA's waves of 256 columns take less time than the few-column kernel's 16 columns at a time.
bool attend_prompt(int type, int width, int heads, int group, long long rows, int seqs, int sms) {
    if (type != HATQ_BF16 || width > 128 || seqs == 0) return false;
    const long long columns = (rows * group + seqs - 1) / seqs, tasks = (long long)heads * seqs * ((columns + kPromptColumns - 1) / kPromptColumns);
    return (tasks + sms - 1) / sms * 1400 < (long long)heads * seqs * ((columns + 15) / 16) * 750 / sms;
}
cudaError_t launch_prompt(const AttendArgs &a, cudaStream_t s) { return a.c.width == 64 ? launch<64>(a, s) : launch<128>(a, s); }

}  // namespace hatq
