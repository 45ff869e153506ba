// The memory-bound token operators: quantize_tokens, the weight layout of
// linear, the packing of codes for the tensor cores, combine_rows, and the
// product for a few rows on the CUDA cores.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>
#include <type_traits>

#include "hatq_tokens.h"

namespace hatq {
namespace {

// max of the magnitudes that keeps a NaN
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// two fp32 values in one register pair: one instruction for both, each rounded as alone
using pair32 = unsigned long long;
__device__ __forceinline__ pair32 pack2(float a, float b) {
    pair32 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(pair32 v, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ pair32 add2(pair32 a, pair32 b) {
    pair32 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair32 sub2(pair32 a, pair32 b) {
    pair32 r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair32 fma2(pair32 a, pair32 b, pair32 c) {
    pair32 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// ------------------------------------------------------------ quantize_tokens
//
// u = act(x) (times the row's second half where gated), t = H~_hb u,
// a = max |t|, code = round(t * min(127 / a, 2^126)), scale =
// max(a / 127, 2^-126) / sqrt(hb). fp32 throughout, one rounding to the code;
// |t| (127 / a) stays below 127.5, so nothing has to be clamped.
//
// Memory-bound: bytes of x and codes. Two kernels:
//  * many rows: CTAs stay and walk the rows. A thread owns 32 consecutive
//    values, so that blocks up to 32 are transformed without leaving the thread
//    and wider ones cost one lane exchange per doubling. A warp keeps its part
//    of the next rows on their way into shared memory (cp.async, 16-byte pieces
//    of 32 lanes next to each other) while it works on one, and the codes leave
//    through the same buffer; the pieces of a lane are XOR-swizzled, which keeps
//    both sides of the exchange free of bank conflicts.
//  * few rows: a thread owns 8 values, four times the threads per row, one row
//    per thread: latency counts there.
// Measured: 8192 x 4096 fp32 in blocks of 128 32 us (6.3 TB/s), 16384 gathered
// fp32 rows of 2000 26.2 us (instruction issue), 8192 gated rows of 2048 bf16
// 21.4 us, one gated row of 8192 3.7 us (latency).

template <int PIECES>
__device__ __forceinline__ int swizzle(int owner, int piece) {
    // the 8 lanes of one 128-byte pass sit in different 16-byte columns
    return owner * PIECES + (piece ^ (PIECES == 8 ? owner & 7 : PIECES == 4 ? (owner >> 1) & 3 : PIECES == 2 ? (owner >> 2) & 1 : 0));
}

template <typename T>
__device__ __forceinline__ pair32 widen2(uint32_t w);
template <> __device__ __forceinline__ pair32 widen2<__nv_bfloat16>(uint32_t w) {
    return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ pair32 widen2<__half>(uint32_t w) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    return pack2(f.x, f.y);
}

__device__ __forceinline__ float relu(float v) { return v < 0.0f ? 0.0f : v; }               // keeps a NaN
// The fast exp(-v) is off by about |v| + 2 ulp and counts with sigma (1 - sigma), so the product stays within a few ulp
// of |v|. Relative to the product itself that is up to |v| ulp in the lower tail, about 1e-5, a thousandth of a code's step
// at 127. Divisors above 2^126 (v below -87.3) give 0.
__device__ __forceinline__ float silu(float v) { return __fdividef(v, 1.0f + __expf(-v)); }
__device__ __forceinline__ float gelu(float v) { return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f)); }

// A row's threads: tpr, a power of two below a warp (a warp then holds 32 / tpr rows) or whole warps.
struct Lanes {
    int tpr, lane, t;                  // threads per row, lane, thread within the row
    long long row;                     // the thread's row
};

// One 16-byte piece, or its first `have` values where it is cut off or not aligned.
template <typename E, int IN>
__device__ __forceinline__ uint4 load_piece(const E *p, int have, bool vec) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (vec && have >= IN) return *reinterpret_cast<const uint4 *>(p);
    E *e = reinterpret_cast<E *>(&w);
#pragma unroll
    for (int j = 0; j < IN; ++j)
        if (j < have) e[j] = p[j];
    return w;
}
template <typename E, int IN>
__device__ __forceinline__ void store_piece(E *p, int have, bool vec, const uint4 &w) {
    if (vec && have >= IN) {
        if (sizeof(E) * IN == 16) *reinterpret_cast<uint4 *>(p) = w;
        else *reinterpret_cast<uint2 *>(p) = make_uint2(w.x, w.y);
        return;
    }
    const E *e = reinterpret_cast<const E *>(&w);
#pragma unroll
    for (int j = 0; j < IN; ++j)
        if (j < have) p[j] = e[j];
}

// Piece i of the warp's values, IN of them: the first one's place in the row, and the piece's in the buffer.
template <int PER, int IN>
__device__ __forceinline__ int piece_first(const Lanes &l, int i) {
    constexpr int kPieces = PER / IN;
    const int at = i * 32 + l.lane;
    return l.tpr >= 32 ? (l.t - l.lane) * PER + at * IN : ((at / kPieces) & (l.tpr - 1)) * PER + (at % kPieces) * IN;
}
// swizzle() of piece i * 32 + lane, from that of piece `lane`
template <int PIECES>
__device__ __forceinline__ int piece_at(int at0, int i) {
    return i * 32 + (PIECES == 8 && (i & 1) ? at0 ^ 4 : at0);
}

template <typename T, int PIECES>
__device__ __forceinline__ void widen(const uint4 (&w)[PIECES], pair32 (&v)[PIECES * 16 / sizeof(T) / 2]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const uint32_t e[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) v[4 * i + j] = widen2<T>(e[j]);
            else if (j % 2 == 0) v[2 * i + j / 2] = pack2(__uint_as_float(e[j]), __uint_as_float(e[j + 1]));
        }
    }
}

template <int PER, typename F>
__device__ __forceinline__ void map_all(pair32 (&v)[PER / 2], F f) {
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
        float x, y;
        unpack2(v[i], x, y);
        v[i] = pack2(f(x), f(y));
    }
}
template <int PER>
__device__ __forceinline__ void activate_all(pair32 (&v)[PER / 2], int act) {
    if (act == HATQ_ACT_SILU) map_all<PER>(v, silu);
    else if (act == HATQ_ACT_GELU) map_all<PER>(v, gelu);
    else map_all<PER>(v, relu);
}
template <int PER>
__device__ __forceinline__ void gate_all(pair32 (&v)[PER / 2], const pair32 (&u)[PER / 2]) {
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
        float x, y, p, q;
        unpack2(v[i], x, y);
        unpack2(u[i], p, q);
        v[i] = pack2(x * p, y * q);
    }
}

// H~_hb on blocks of hb consecutive values: up to PER in the thread, wider ones across hb / PER lanes
template <int PER>
__device__ __forceinline__ void transform(pair32 (&v)[PER / 2], int hb, int t) {
    if (hb > 1) {
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
            float x, y;
            unpack2(v[i], x, y);
            v[i] = pack2(x + y, x - y);
        }
    }
#pragma unroll
    for (int h = 1; h < PER / 2; h <<= 1) {
        if (2 * h < hb) {
#pragma unroll
            for (int i = 0; i < PER / 2; ++i) {
                if (i & h) continue;
                const pair32 x = v[i], y = v[i + h];
                v[i] = add2(x, y);
                v[i + h] = sub2(x, y);
            }
        }
    }
#pragma unroll
    for (int m = 1; m <= 128 / PER; m <<= 1) {
        if (m * PER >= hb) break;
        const float sign = (t & m) != 0 ? -1.0f : 1.0f;
        const pair32 sign2 = pack2(sign, sign);
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
            float x, y;
            unpack2(v[i], x, y);
            x = __shfl_xor_sync(0xffffffffu, x, m);
            y = __shfl_xor_sync(0xffffffffu, y, m);
            v[i] = fma2(sign2, v[i], pack2(x, y));                      // exact product: one rounding, that of the sum
        }
    }
}

// max |v| of the thread's lanes of the row (the warp, or tpr lanes of it)
template <int PER>
__device__ __forceinline__ float lane_max(const pair32 (&v)[PER / 2], int tpr) {
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
        float x, y;
        unpack2(v[i], x, y);
        amax = max_abs(amax, x, y);
    }
    for (int m = min(tpr, 32) / 2; m > 0; m >>= 1) amax = max_abs(amax, __shfl_xor_sync(0xffffffffu, amax, m), 0.0f);
    return amax;
}
// of the row's warps, whose maxima lie at m[0 .. warps)
__device__ __forceinline__ float warps_max(const float *m, int warps, int lane) {
    float amax = 0.0f;
    if (warps <= 8) {
        for (int w = 0; w < warps; ++w) amax = max_abs(amax, m[w], 0.0f);
    } else {
        amax = lane < warps ? m[lane] : 0.0f;
        for (int h = 16; h > 0; h >>= 1) amax = max_abs(amax, __shfl_xor_sync(0xffffffffu, amax, h), 0.0f);
    }
    return amax;
}

__device__ __forceinline__ bool is_fine(float amax) { return amax <= 3.402823466e38f; }   // no infinity, no NaN
// 127 / a overflows below 127 / 2^128: the step stays at the smallest normal number there
__device__ __forceinline__ float step_inverse(float amax) {
    return !is_fine(amax) || amax == 0.0f ? 0.0f : fminf(127.0f / amax, 0x1p126f);
}
__device__ __forceinline__ float step_of(float amax, float inv_norm) {
    if (!is_fine(amax)) return __int_as_float(0x7fc00000);
    return amax == 0.0f ? 1.0f : fmaxf(amax / 127.0f, 0x1p-126f) * inv_norm;
}

// fma(t, inv, 1.5 2^23 + c) rounds t inv to an integer (half to even) and leaves it, plus c, in the low bits.
// c = 0x6480 makes the low half-word the fp16 number 1152 + code.
template <bool F16, int PER>
__device__ __forceinline__ void encode(const pair32 (&v)[PER / 2], float amax, uint32_t (&w)[F16 ? PER / 2 : PER / 4]) {
    const bool fine = is_fine(amax);
    const float inv = step_inverse(amax), base = 12582912.0f + (F16 ? 25728.0f : 0.0f);
    const pair32 inv2 = pack2(inv, inv), base2 = pack2(base, base);
    if constexpr (F16) {
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
            float x, y;
            unpack2(fma2(v[i], inv2, base2), x, y);
            uint32_t h;
            asm("sub.f16x2 %0, %1, %2;"
                : "=r"(h)
                : "r"(__byte_perm(__float_as_uint(x), __float_as_uint(y), 0x5410)), "r"(0x64806480u));
            w[i] = fine ? h : 0u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER / 4; ++i) {
            float x, y, z, q;
            unpack2(fma2(v[2 * i], inv2, base2), x, y);
            unpack2(fma2(v[2 * i + 1], inv2, base2), z, q);
            const uint32_t c = __byte_perm(__byte_perm(__float_as_uint(x), __float_as_uint(y), 0x0040),
                                           __byte_perm(__float_as_uint(z), __float_as_uint(q), 0x0040), 0x5410);
            w[i] = fine ? c : 0u;
        }
    }
}

// ---- few rows: 8 values per thread, one CTA per row or more rows per CTA

template <typename T, bool F16>
__global__ void __launch_bounds__(1024) quantize_few_kernel(const __grid_constant__ TokenQuantArgs a, int tpr) {
    using E = typename std::conditional<F16, __half, int8_t>::type;
    constexpr int kPer = 8, kIn = 16 / sizeof(T), kPieces = kPer / kIn;
    __shared__ float warp_max[32];
    const int rl = threadIdx.x / tpr, lane = threadIdx.x & 31, t = threadIdx.x - rl * tpr;
    const long long row = (long long)blockIdx.x * (blockDim.x / tpr) + rl;
    after_prior_kernels();
    int src = row < a.rows ? (a.index ? a.index[row] : (int)row) : -1;
    if (src >= a.src_rows) src = -1;
    const int have = src < 0 ? 0 : a.c - t * kPer;
    const T *p = reinterpret_cast<const T *>(a.x) + (long long)max(src, 0) * a.ldx + t * kPer;
    uint4 w[kPieces], g[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        w[i] = load_piece<T, kIn>(p + i * kIn, have - i * kIn, a.vec);
        if (a.gated) g[i] = load_piece<T, kIn>(p + a.c + i * kIn, have - i * kIn, a.vec);
    }
    pair32 v[kPer / 2];
    widen<T, kPieces>(w, v);
    if (a.act != HATQ_ACT_NONE && src >= 0) activate_all<kPer>(v, a.act);
    if (a.gated) {
        pair32 u[kPer / 2];
        widen<T, kPieces>(g, u);
        gate_all<kPer>(v, u);
    }
    transform<kPer>(v, a.hb, t);
    float amax = lane_max<kPer>(v, tpr);
    if (tpr > 32) {
        if (lane == 0) warp_max[threadIdx.x >> 5] = amax;
        __syncthreads();
        amax = warps_max(warp_max + rl * (tpr / 32), tpr / 32, lane);
    }
    if (row >= a.rows) return;
    if (t == 0) a.scales[row] = step_of(amax, a.inv_norm);
    uint32_t out[4] = {0, 0, 0, 0};
    encode<F16, kPer>(v, amax, reinterpret_cast<uint32_t(&)[F16 ? 4 : 2]>(out));
    store_piece<E, kPer>(reinterpret_cast<E *>(a.codes) + row * a.ldc + t * kPer, a.c - t * kPer, a.vec,
                         make_uint4(out[0], out[1], out[2], out[3]));
}

// ---- many rows

constexpr int kPer = 32;

__device__ __forceinline__ void copy_async(uint4 *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src)
                 : "memory");
}
// the first `bytes` (at least one) of the 16, zeros behind them; the source is aligned to 16 all the same
__device__ __forceinline__ void copy_async_part(uint4 *dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(bytes)
                 : "memory");
}
template <int AHEAD> __device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
}

// STAGES buffers per warp, so STAGES - 1 rows on their way. With one buffer (wide rows, whose buffers would not
// all fit) the two halves of a gated row pass through it one after the other. PLAIN: no activation and no gate (their
// code, not run, costs 5 to 7 %).
template <typename T, bool F16, int THREADS, int STAGES, bool PLAIN>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 1)
    quantize_rows_kernel(const __grid_constant__ TokenQuantArgs a, int tpr) {
    using E = typename std::conditional<F16, __half, int8_t>::type;
    constexpr int kIn = 16 / sizeof(T), kPieces = kPer / kIn;            // pieces per thread
    constexpr int kOutIn = 16 / sizeof(E), kOutPieces = kPer / kOutIn;
    __shared__ float warp_max[2][32];
    extern __shared__ __align__(128) uint4 buffers[];
    constexpr bool kAlone = STAGES == 1;
    const int halves = !PLAIN && a.gated && !kAlone ? 2 : 1, stage_pieces = 32 * kPieces * halves;
    uint4 *stages = buffers + (threadIdx.x >> 5) * STAGES * stage_pieces;
    const int rl = threadIdx.x / tpr, per_cta = blockDim.x / tpr;
    Lanes l;
    l.tpr = tpr;
    l.lane = threadIdx.x & 31;
    l.t = threadIdx.x - rl * tpr;
    const long long step = (long long)gridDim.x * per_cta;
    const long long base = (long long)blockIdx.x * per_cta;
    auto source = [&](long long row) {
        int src = row < a.rows ? (a.index ? a.index[row] : (int)row) : -1;
        return src >= a.src_rows ? -1 : src;
    };
    // a warp whose values are all there, in 16-byte pieces, needs no look at a piece
    const int warp_first = (l.t - l.lane) * kPer;
    const bool wide = a.vec && tpr >= 32, whole = wide && warp_first + 32 * kPer <= a.c;
    const int in_at = swizzle<kPieces>(l.lane / kPieces, l.lane % kPieces);
    const int out_at = swizzle<kOutPieces>(l.lane / kOutPieces, l.lane % kOutPieces);
    auto issue = [&](int src, uint4 *buffer, int half) {
        if (wide) {
            // pieces of one row, 32 lanes next to each other; behind its end (or in an empty row) they are zeros
            const T *p = reinterpret_cast<const T *>(a.x) + (long long)max(src, 0) * a.ldx + half * a.c;
            const int first = warp_first + l.lane * kIn;
#pragma unroll 1
            for (int h = 0; h < halves; ++h) {
                if (whole && src >= 0) {
#pragma unroll
                    for (int i = 0; i < kPieces; ++i)
                        copy_async(buffer + piece_at<kPieces>(in_at, i), p + first + i * 32 * kIn);
                } else {
                    const int end = src >= 0 ? a.c : 0;
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        const int at = first + i * 32 * kIn, have = min(end - at, kIn);
                        uint4 *dst = buffer + piece_at<kPieces>(in_at, i);
                        if (have > 0) copy_async_part(dst, p + at, have * (int)sizeof(T));
                        else *dst = make_uint4(0, 0, 0, 0);              // nothing to copy from, nor an aligned address to name
                    }
                }
                buffer += 32 * kPieces;
                p += a.c;
            }
            return;
        }
#pragma unroll 1
        for (int hi = 0; hi < halves * kPieces; ++hi) {
            const int h = hi / kPieces, i = hi % kPieces;
            const int first = piece_first<kPer, kIn>(l, i);
            const int from = l.tpr >= 32 ? src : __shfl_sync(0xffffffffu, src, (i * 32 + l.lane) / kPieces);
            const T *p = reinterpret_cast<const T *>(a.x) + (long long)max(from, 0) * a.ldx + (half + h) * a.c + first;
            const int have = from < 0 ? 0 : a.c - first;
            uint4 *dst = buffer + h * 32 * kPieces + piece_at<kPieces>(in_at, i);
            if (a.vec && have >= kIn) copy_async(dst, p);
            else *dst = load_piece<T, kIn>(p, have, false);
        }
    };
    after_prior_kernels();
    int srcs[STAGES];
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        srcs[s] = source(base + s * step + rl);
        issue(srcs[s], stages + s * stage_pieces, 0);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    srcs[STAGES - 1] = source(base + (STAGES - 1) * step + rl);
    int at = 0, ahead = STAGES - 1, turn = 0;
    for (long long first = base; first < a.rows; first += step) {
        issue(srcs[STAGES - 1], stages + ahead * stage_pieces, 0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        const int src = srcs[0];
#pragma unroll
        for (int s = 0; s + 1 < STAGES; ++s) srcs[s] = srcs[s + 1];
        srcs[STAGES - 1] = source(first + STAGES * step + rl);
        l.row = first + rl;
        copies_wait<STAGES - 1>();
        __syncwarp();
        uint4 *stage = stages + at * stage_pieces;
        uint4 w[kPieces];
        pair32 v[kPer / 2];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) w[i] = stage[swizzle<kPieces>(l.lane, i)];
        widen<T, kPieces>(w, v);
        if (!PLAIN && a.act != HATQ_ACT_NONE && src >= 0) activate_all<kPer>(v, a.act);
        if (!PLAIN && a.gated) {
            pair32 u[kPer / 2];
            if (kAlone) {
                __syncwarp();
                issue(src, stage, 1);
                asm volatile("cp.async.commit_group;" ::: "memory");
                copies_wait<0>();
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < kPieces; ++i) w[i] = stage[(kAlone ? 0 : 32 * kPieces) + swizzle<kPieces>(l.lane, i)];
            widen<T, kPieces>(w, u);
            gate_all<kPer>(v, u);
        }
        transform<kPer>(v, a.hb, l.t);
        float amax = lane_max<kPer>(v, tpr);
        if (tpr > 32) {
            if (l.lane == 0) warp_max[turn][threadIdx.x >> 5] = amax;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + rl), "r"(tpr) : "memory");
            amax = warps_max(warp_max[turn] + rl * (tpr / 32), tpr / 32, l.lane);
            turn ^= 1;                                                   // the next row's maxima have a place of their own
        }
        if (l.t == 0 && l.row < a.rows) a.scales[l.row] = step_of(amax, a.inv_norm);
        union { uint4 p[kOutPieces]; uint32_t w[F16 ? kPer / 2 : kPer / 4]; } out;
        encode<F16, kPer>(v, amax, out.w);
        __syncwarp();                                                    // every lane has read the buffer
#pragma unroll
        for (int i = 0; i < kOutPieces; ++i) stage[swizzle<kOutPieces>(l.lane, i)] = out.p[i];
        __syncwarp();
        E *codes = reinterpret_cast<E *>(a.codes);
        if (wide) {
            const int first = warp_first + l.lane * kOutIn;
            E *p = codes + l.row * a.ldc + first;
            if (l.row < a.rows) {
#pragma unroll
                for (int i = 0; i < kOutPieces; ++i)
                    if (first + i * 32 * kOutIn + kOutIn <= a.c)
                        *reinterpret_cast<uint4 *>(p + i * 32 * kOutIn) = stage[piece_at<kOutPieces>(out_at, i)];
                if (!whole && a.c % kOutIn != 0) {
                    // the row's last values fill no piece: the lane that has it stores them one by one
#pragma unroll 1
                    for (int i = 0; i < kOutPieces; ++i)
                        if (first + i * 32 * kOutIn < a.c)
                            store_piece<E, kOutIn>(p + i * 32 * kOutIn, min(a.c - first - i * 32 * kOutIn, kOutIn - 1), false,
                                                   stage[piece_at<kOutPieces>(out_at, i)]);
                }
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < kOutPieces; ++i) {
                const int from = piece_first<kPer, kOutIn>(l, i);
                const long long row = l.tpr >= 32 ? l.row : l.row - l.lane / l.tpr + (i * 32 + l.lane) / kOutPieces / l.tpr;
                store_piece<E, kOutIn>(codes + row * a.ldc + from, row < a.rows ? a.c - from : 0, a.vec,
                                       stage[piece_at<kOutPieces>(out_at, i)]);
            }
        }
        __syncwarp();                                                    // the buffer is free for the next copies
        at = at + 1 == STAGES ? 0 : at + 1;
        ahead = ahead + 1 == STAGES ? 0 : ahead + 1;
    }
    copies_wait<0>();
}

// ---- many rows of 16-bit values without an activation, blocks of 16 to 256
//
// The 16-point transforms are warp-level matrix products: 16 blocks x H_16, the
// values' own bits times +-1, fp32 sums. That leaves at most four stages, three
// of them between registers of a thread: lane (g, j) = (lane / 4, lane % 4) gets
// values 2j, 2j + 1 and 2j + 8, 2j + 9 of blocks 8g .. 8g + 7, i.e. of a whole
// block of 128, so only blocks of 256 need a lane exchange. With butterflies
// alone the kernel above is bound by instruction issue: 8192 x 4096 bf16 in
// blocks of 128 took 30.7 us there and takes 22.3 us (6.0 TB/s) here.

// Place of 16-byte piece p in a buffer: 8 pieces that lie 16 apart (or, for INT8 codes, 8 apart) on different banks.
template <int APART>
__device__ __forceinline__ int spread(int p) {
    return (p & ~7) | ((p ^ (p / APART)) & 7);
}

template <typename T>
__device__ __forceinline__ void product16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <typename T, bool F16, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) quantize_blocks_kernel(const __grid_constant__ TokenQuantArgs a, int tpr) {
    using E = typename std::conditional<F16, __half, int8_t>::type;
    constexpr int kStages = 2, kPieces = 4, kIn = 8, kOutIn = 16 / sizeof(E), kOutPieces = kPer / kOutIn;
    __shared__ float warp_max[2][32];
    extern __shared__ __align__(128) uint4 buffers[];
    uint4(*stages)[32 * kPieces] = reinterpret_cast<uint4(*)[32 * kPieces]>(buffers) + (threadIdx.x >> 5) * kStages;
    const int rl = threadIdx.x / tpr, per_cta = blockDim.x / tpr, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    const int t0 = threadIdx.x - rl * tpr, warp_first = (t0 - lane) * kPer;
    const long long step = (long long)gridDim.x * per_cta, base = (long long)blockIdx.x * per_cta;
    // H_16's columns g and g + 8, rows 2j, 2j + 1 and 2j + 8, 2j + 9
    const uint32_t one = std::is_same<T, __half>::value ? 0x3c00u : 0x3f80u;
    auto sign = [&](int k, int n) { return one | (uint32_t)(__popc(k & n) & 1) << 15; };
    uint32_t h[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            h[n][k] = sign(2 * j + 8 * k, g + 8 * n) | sign(2 * j + 8 * k + 1, g + 8 * n) << 16;
    auto source = [&](long long row) {
        int src = row < a.rows ? (a.index ? a.index[row] : (int)row) : -1;
        return src >= a.src_rows ? -1 : src;
    };
    const bool whole = warp_first + 32 * kPer <= a.c;
    auto issue = [&](int src, uint4 *buffer) {
        const T *p = reinterpret_cast<const T *>(a.x) + (long long)max(src, 0) * a.ldx;
        const int first = warp_first + lane * kIn;
        if (whole && src >= 0) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) copy_async(buffer + spread<16>(i * 32 + lane), p + first + i * 32 * kIn);
        } else {
            const int end = src >= 0 ? a.c : 0;                          // c is a multiple of 16: pieces are whole
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = first + i * 32 * kIn;
                uint4 *dst = buffer + spread<16>(i * 32 + lane);
                if (at < end) copy_async(dst, p + at);
                else *dst = make_uint4(0, 0, 0, 0);                      // nothing to copy from
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    after_prior_kernels();
    issue(source(base + rl), stages[0]);
    int next = source(base + step + rl), turn = 0;
    for (long long first = base; first < a.rows; first += step) {
        issue(next, stages[turn ^ 1]);
        next = source(first + 2 * step + rl);
        const long long row = first + rl;
        copies_wait<1>();
        __syncwarp();
        uint4 *stage = stages[turn];
        // c[t][n]: values 2j + 8n, 2j + 8n + 1 of blocks 8g + t and 8g + 4 + t
        float c[4][2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int block = (lane & 7) * 8 + (lane >> 3 & 1) * 4 + t;  // of this lane's row of the four matrices
            uint32_t m[4];
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(m[0]), "=r"(m[1]), "=r"(m[2]), "=r"(m[3])
                         : "r"((uint32_t)__cvta_generic_to_shared(stage + spread<16>(block * 2 + (lane >> 4))))
                         : "memory");
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int q = 0; q < 4; ++q) c[t][n][q] = 0.0f;
                product16<T>(c[t][n], m, h[n][0], h[n][1]);
            }
        }
        // v[(rest * 4 + t) * 2 + n], rest: block 8g + 4 rest + t
        pair32 v[16];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                v[t * 2 + n] = pack2(c[t][n][0], c[t][n][1]);
                v[(4 + t) * 2 + n] = pack2(c[t][n][2], c[t][n][3]);
            }
#pragma unroll
        for (int s = 2; s < 16; s <<= 1) {
            if (16 * s <= a.hb) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i & s) continue;
                    const pair32 x = v[i], y = v[i + s];
                    v[i] = add2(x, y);
                    v[i + s] = sub2(x, y);
                }
            }
        }
        if (a.hb == 256) {
            const float up = (g & 1) ? -1.0f : 1.0f;
            const pair32 up2 = pack2(up, up);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float x, y;
                unpack2(v[i], x, y);
                x = __shfl_xor_sync(0xffffffffu, x, 4);
                y = __shfl_xor_sync(0xffffffffu, y, 4);
                v[i] = fma2(up2, v[i], pack2(x, y));
            }
        }
        float amax = lane_max<kPer>(v, 32);
        if (tpr > 32) {
            if (lane == 0) warp_max[turn][threadIdx.x >> 5] = amax;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + rl), "r"(tpr) : "memory");
            amax = warps_max(warp_max[turn] + rl * (tpr / 32), tpr / 32, lane);
        }
        if (t0 == 0 && row < a.rows) a.scales[row] = step_of(amax, a.inv_norm);
        uint32_t w[F16 ? 16 : 8];
        encode<F16, kPer>(v, amax, w);
        __syncwarp();                                                    // every lane has read the buffer
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int block = 8 * g + (i >> 1), n = i & 1;
            if constexpr (F16) reinterpret_cast<uint32_t *>(stage + spread<16>(block * 2 + n))[j] = w[i];
            else reinterpret_cast<uint16_t *>(stage + spread<8>(block))[4 * n + j] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
        __syncwarp();
        if (row < a.rows) {
            const int at = warp_first + lane * kOutIn;
            E *p = reinterpret_cast<E *>(a.codes) + row * a.ldc + at;
#pragma unroll
            for (int i = 0; i < kOutPieces; ++i)
                if (at + i * 32 * kOutIn < a.c)
                    *reinterpret_cast<uint4 *>(p + i * 32 * kOutIn) = stage[spread<F16 ? 16 : 8>(i * 32 + lane)];
        }
        __syncwarp();                                                    // the buffer is free for the next copies
        turn ^= 1;
    }
    copies_wait<0>();
}

int threads_per_row(int c, int per) {
    const int need = (c + per - 1) / per;
    if (need > 32) return (need + 31) & ~31;
    int tpr = 1;
    while (tpr < need) tpr <<= 1;
    return tpr;
}

template <typename T, bool F16, int THREADS, int STAGES, bool PLAIN>
cudaError_t quantize_rows_launch(const TokenQuantArgs &a, cudaStream_t s) {
    const int tpr = threads_per_row(a.c, kPer);
    const int per_cta = tpr >= 256 ? 1 : 256 / tpr;
    const int threads = per_cta * tpr;                                   // whole warps
    auto k = quantize_rows_kernel<T, F16, THREADS, STAGES, PLAIN>;
    const int smem = threads * kPer * (int)sizeof(T) * STAGES * (a.gated && STAGES > 1 ? 2 : 1);
    static const int regs = [] {
        cudaFuncAttributes fa{};
        return cudaFuncGetAttributes(&fa, quantize_rows_kernel<T, F16, THREADS, STAGES, PLAIN>) == cudaSuccess ? fa.numRegs : 128;
    }();
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(k), smem, allowed);
    if (e != cudaSuccess) return e;
    // as many CTAs as are resident at once: they walk the rows
    const int fit = max(1, min(min(2048 / threads, 220 * 1024 / (smem + 1024)), 65536 / (regs * threads)));
    const long long ctas = (a.rows + per_cta - 1) / per_cta, room = (long long)a.sms * fit;
    return launch_early(k, dim3((unsigned)(ctas < room ? ctas : room)), threads, smem, s, a, tpr);
}

template <typename T, bool F16, int THREADS>
cudaError_t quantize_blocks_launch(const TokenQuantArgs &a, cudaStream_t s) {
    const int tpr = threads_per_row(a.c, kPer), per_cta = tpr >= 256 ? 1 : 256 / tpr, threads = per_cta * tpr;
    const int smem = threads * 2 * kPer * 2;
    auto k = quantize_blocks_kernel<T, F16, THREADS>;
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(k), smem, allowed);
    if (e != cudaSuccess) return e;
    const long long ctas = (a.rows + per_cta - 1) / per_cta, room = (long long)a.sms * (1024 / threads);
    return launch_early(k, dim3((unsigned)(ctas < room ? ctas : room)), threads, smem, s, a, tpr);
}

template <typename T, bool F16>
cudaError_t quantize_size(const TokenQuantArgs &a, cudaStream_t s) {
    // few rows: as long as one CTA wave of 8-value threads holds them
    if (a.c <= 8192 && a.rows * a.c <= (long long)a.sms * 1024 * 8) {
        const int tpr = threads_per_row(a.c, 8), per_cta = tpr >= 256 ? 1 : 256 / tpr;
        return launch_early(quantize_few_kernel<T, F16>, dim3((unsigned)((a.rows + per_cta - 1) / per_cta)), per_cta * tpr, 0, s,
                            a, tpr);
    }
    if constexpr (sizeof(T) == 2) {
        if (threads_per_row(a.c, kPer) >= 32 && a.vec && !a.gated && a.act == HATQ_ACT_NONE && a.hb >= 16)
            return a.c <= 8192 ? quantize_blocks_launch<T, F16, 256>(a, s) : quantize_blocks_launch<T, F16, 1024>(a, s);
    }
    if (a.c > 8192) {
        if (sizeof(T) == 4 || a.gated) return quantize_rows_launch<T, F16, 1024, 1, false>(a, s);
        return quantize_rows_launch<T, F16, 1024, sizeof(T) == 4 ? 1 : 2, false>(a, s);
    }
    if (a.act == HATQ_ACT_NONE && !a.gated) return quantize_rows_launch<T, F16, 256, 2, true>(a, s);
    return quantize_rows_launch<T, F16, 256, 2, false>(a, s);
}

// ------------------------------------------------------------ weight layout
//
// codes [expert][n / 128][k / 64][4][128][16]: a block of 128 channels x 64
// codes is 8 KB in one piece, so one bulk copy moves it, and thread m of the
// converters reads its channel's 64 codes as four 16-byte words that no two
// lanes take from one bank. A code is stored as code + 128 (the converters turn
// that into fp16 with one byte permutation and one subtraction).
//
// windows[expert]: bit j set if some channel holds an aligned window of
// 1024 << j codes with sum |w| > 2^17: only below that is every fp32 partial sum
// of the window, at most 128 sum |w| <= 2^24, an exact integer.

constexpr int kLevels = 6;             // windows of 1024 .. 32768 (65536: the whole depth, level 6)

__global__ void __launch_bounds__(128) linear_layout_kernel(const int8_t *w, long long ldw, int n, int k, int n_tiles,
                                                            int kb, uint8_t *codes, int32_t *windows) {
    const int tile = blockIdx.x % n_tiles, e = blockIdx.x / n_tiles;
    const int ch = tile * kRowTile + threadIdx.x;
    const bool live = ch < n;
    const int8_t *src = w + ((long long)e * n + (live ? ch : 0)) * ldw;
    uint8_t *dst = codes + ((long long)e * n_tiles + tile) * kb * kBlockBytes + threadIdx.x * 16;
    const bool vec = ((reinterpret_cast<uintptr_t>(w) | (uintptr_t)ldw) & 15) == 0;
    int sum[kLevels + 1] = {0};
    int flags = 0;
    for (int b = 0; b < kb; ++b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k0 = b * 64 + j * 16;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (live) {
                if (vec && k0 + 16 <= k) v = *reinterpret_cast<const uint4 *>(src + k0);
                else {
                    uint8_t *p = reinterpret_cast<uint8_t *>(&v);
                    for (int i = 0; i < 16; ++i) p[i] = k0 + i < k ? (uint8_t)src[k0 + i] : 0;
                }
            }
            const uint32_t word[4] = {v.x, v.y, v.z, v.w};
            uint32_t sad = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sad = __dp4a(__vabs4(word[i]), 0x01010101u, sad);
#pragma unroll
            for (int l = 0; l <= kLevels; ++l) sum[l] += (int)sad;
            *reinterpret_cast<uint4 *>(dst + (long long)b * kBlockBytes + j * 2048) =
                make_uint4(v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u);
        }
#pragma unroll
        for (int l = 0; l <= kLevels; ++l) {
            if (sum[l] > (1 << 17)) flags |= 1 << l;
            if (((b + 1) & ((16 << l) - 1)) == 0) sum[l] = 0;
        }
    }
    if (flags) atomicOr(windows + e, flags);
}

// ------------------------------------------------------------ packing of codes
//
// For products whose codes TMA cannot take as they lie, where that pays: bound by
// its bytes, 1 or 2 read and 2 written per code (32768 x 2048 int8: about 35 us).

__global__ void __launch_bounds__(256) pack_codes_kernel(const void *x, int format, long long ldx, long long rows, int k,
                                                         int k_pad, __half *out) {
    const int per_row = k_pad / 8;
    const long long total = rows * per_row;
    after_prior_kernels();
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const long long r = i / per_row;
        const int c = (int)(i - r * per_row) * 8;
        uint4 w;
        __half *h = reinterpret_cast<__half *>(&w);
        if (format == HATQ_CODES_I8) {
            const int8_t *p = reinterpret_cast<const int8_t *>(x) + r * ldx + c;
            int8_t b[8];
            if (c + 8 <= k && (reinterpret_cast<uintptr_t>(p) & 7) == 0) {
                *reinterpret_cast<uint2 *>(b) = *reinterpret_cast<const uint2 *>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = c + j < k ? p[j] : 0;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = __int2half_rn(b[j]);
        } else {
            const __half *p = reinterpret_cast<const __half *>(x) + r * ldx + c;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = c + j < k ? p[j] : __half(0.0f);
        }
        *reinterpret_cast<uint4 *>(out + r * k_pad + c) = w;
    }
}

// ------------------------------------------------------------ a few rows
//
// Bound by the weights' bytes and by latency: every load of weights that a
// thread makes is on its way before the rows' codes are brought to shared
// memory and before the first is used. A CTA owns 8 R channels of one group and
// the whole reduction; a warp takes every 8th 64-code block, a lane 16 codes of
// R channels (8 lanes read 128 consecutive bytes). Sums are int32 dot products
// of four codes; this GPU issues them at a fraction of its other integer
// instructions, so from three rows on they, not the bytes, are the bound, and
// larger weights go to the tensor cores then (see plan_of). One row, 4096 x
// 4096: 3.5 us (4.8 TB/s with the launch); eight experts of 2048 x 1536, one row
// each: 5.6 us.

constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;

__device__ __forceinline__ void store_y(void *y, int type, long long at, float v) {
    if (type == HATQ_F32) reinterpret_cast<float *>(y)[at] = v;
    else if (type == HATQ_F16) reinterpret_cast<__half *>(y)[at] = __float2half_rn(v);
    else reinterpret_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
}

template <int MT, int R>
__global__ void __launch_bounds__(kFewThreads) linear_few_kernel(const __grid_constant__ LinearArgs a) {
    constexpr int kCh = 8 * R, kAhead = 8 / R;                          // channels of the CTA, blocks on their way
    extern __shared__ __align__(16) uint8_t xs[];                       // [MT][k_pad] codes
    __shared__ int part[kFewWarps][kCh][MT];
    const int k_pad = a.kb * 64;
    after_prior_kernels();
    int e = 0, r0 = 0, r1 = a.rows;
    if (a.offsets) {
        // row blockIdx.y, of the expert before the first offset above it (one row per CTA: MT is 1)
        __shared__ int above[kFewWarps];
        r0 = (int)blockIdx.y;
        r1 = r0 + 1;
        int mine = INT_MAX;
        for (int g = threadIdx.x; g <= a.experts; g += kFewThreads)
            if (a.offsets[g] > r0) mine = min(mine, g);
        mine = __reduce_min_sync(0xffffffffu, mine);
        if ((threadIdx.x & 31) == 0) above[threadIdx.x >> 5] = mine;
        __syncthreads();
        int to = INT_MAX;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) to = min(to, above[w]);
        if (to == 0 || to > a.experts) return;                          // no expert holds the row
        e = to - 1;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch_l = lane & 7, j = lane >> 3;
    const int ch0 = blockIdx.x * kCh;
    const uint8_t *wp = a.w + (((long long)e * a.n_tiles + ch0 / kRowTile) * a.kb + warp) * kBlockBytes + j * 2048 +
                        (ch0 % kRowTile + ch_l) * 16;
    uint4 w[kAhead][R];
    auto load = [&](int b, uint4 (&v)[R]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            v[r] = b < a.kb ? *reinterpret_cast<const uint4 *>(wp + (long long)(b - warp) * kBlockBytes + r * 128)
                            : make_uint4(0, 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(warp + i * kFewWarps, w[i]);
    // Behind an expired wait nothing is written, as in the tensor-core kernel. One thread of the CTA looks: with all of
    // them the one word is asked for by thousands of warps, and one row of 4096 x 4096 takes 4.4 us instead of 3.5.
    __shared__ int skip;
    int expired = 0;
    if (threadIdx.x == 0) expired = *a.err;
    for (int i = threadIdx.x; i < MT * (k_pad / 16); i += kFewThreads) {
        const int t = i / (k_pad / 16), c = (i - t * (k_pad / 16)) * 16;
        const long long r = r0 + t;
        uint4 v = make_uint4(0, 0, 0, 0);
        int8_t *b = reinterpret_cast<int8_t *>(&v);
        if (r < r1) {
            if (a.format == HATQ_CODES_I8) {
                const int8_t *p = reinterpret_cast<const int8_t *>(a.x) + r * a.ldx + c;
                if (c + 16 <= a.k && (reinterpret_cast<uintptr_t>(p) & 15) == 0) v = *reinterpret_cast<const uint4 *>(p);
                else
                    for (int q = 0; q < 16; ++q) b[q] = c + q < a.k ? p[q] : 0;
            } else {
                const __half *p = reinterpret_cast<const __half *>(a.x) + r * a.ldx + c;
                if (c + 16 <= a.k && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
                    const uint4 lo = reinterpret_cast<const uint4 *>(p)[0], hi = reinterpret_cast<const uint4 *>(p)[1];
                    v = make_uint4(narrow_codes(lo.x, lo.y), narrow_codes(lo.z, lo.w), narrow_codes(hi.x, hi.y), narrow_codes(hi.z, hi.w));
                } else {
                    for (int q = 0; q < 16; ++q) b[q] = c + q < a.k ? (int8_t)__half2int_rn(p[q]) : 0;
                }
            }
        }
        *reinterpret_cast<uint4 *>(xs + t * k_pad + c) = v;
    }
    if (threadIdx.x == 0) skip = expired;
    __syncthreads();
    int acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = 0;
    for (int b0 = warp; b0 < a.kb; b0 += kFewWarps * kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int b = b0 + i * kFewWarps;
            if (b < a.kb) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(xs + t * k_pad + b * 64 + j * 16);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        acc[r][t] = __dp4a((int)(w[i][r].x ^ 0x80808080u), (int)x.x, acc[r][t]);
                        acc[r][t] = __dp4a((int)(w[i][r].y ^ 0x80808080u), (int)x.y, acc[r][t]);
                        acc[r][t] = __dp4a((int)(w[i][r].z ^ 0x80808080u), (int)x.z, acc[r][t]);
                        acc[r][t] = __dp4a((int)(w[i][r].w ^ 0x80808080u), (int)x.w, acc[r][t]);
                    }
                }
                if (b + kFewWarps * kAhead < a.kb) load(b + kFewWarps * kAhead, w[i]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            acc[r][t] += __shfl_xor_sync(0xffffffffu, acc[r][t], 8);
            acc[r][t] += __shfl_xor_sync(0xffffffffu, acc[r][t], 16);
            if (j == 0) part[warp][8 * r + ch_l][t] = acc[r][t];
        }
    __syncthreads();
    if (skip) return;
    for (int i = threadIdx.x; i < kCh * MT; i += kFewThreads) {
        const int t = i / kCh, c = i % kCh;
        if (r0 + t < r1 && ch0 + c < a.n) {
            int sum = 0;
            for (int q = 0; q < kFewWarps; ++q) sum += part[q][c][t];
            const long long ch = (long long)e * a.n + ch0 + c;
            float v = (float)sum * a.s_w[ch] * a.s_x[r0 + t];
            if (a.bias) v += a.bias[ch];
            store_y(a.y, a.y_type, (r0 + t) * a.ldy + ch0 + c, v);
        }
    }
}

// ------------------------------------------------------------ combine_rows

// Bound by the rows' bytes. A thread owns 16 bytes of a token's row; the rows
// of up to kAhead slots are on their way at a time, and the next token's indices
// and weights before this one's rows are added up. Fewer slots leave room for
// more threads. 8192 tokens x 8 rows of 2048 bf16: 48 us, 6.3 TB/s.

constexpr int combine_ctas(int ahead) { return ahead == 8 ? 3 : ahead == 4 ? 4 : 6; }

// UNIT: bytes that a load or a store takes. Rows on 16-byte boundaries: one of 16 per thread and row; else four of 4 or
// of 2, `width` units apart, so that the lanes of each lie next to each other.
template <typename T, int UNIT, int kAhead>
__global__ void __launch_bounds__(256, combine_ctas(kAhead)) combine_rows_kernel(const T *y, long long ldy, long long rows,
                                                                                 const int32_t *index, const float *weights,
                                                                                 long long tokens, int topk, int c, T *out,
                                                                                 long long ldo, int width) {
    constexpr int kEach = UNIT / sizeof(T), kUnits = UNIT == 16 ? 1 : 4, kVec = kUnits * kEach;
    using U = typename std::conditional<UNIT == 16, uint4, typename std::conditional<UNIT == 4, uint32_t, uint16_t>::type>::type;
    // width threads (a power of two) for a token, or for a part of its row
    const int per_row = (c + kVec - 1) / kVec, parts = (per_row + width - 1) / width, per_cta = 256 / width;
    const int slot = threadIdx.x / width, lane = threadIdx.x - slot * width, apart = width * kEach;
    const long long groups = (tokens + per_cta - 1) / per_cta;           // of per_cta tokens; an item is a part of one
    const int step_part = gridDim.x % parts;
    const long long step_group = gridDim.x / parts;
    long long group = blockIdx.x / parts, t_next = 0;
    int part = blockIdx.x % parts, at_next = 0;
    const bool quads = topk % 4 == 0 && ((reinterpret_cast<uintptr_t>(index) | reinterpret_cast<uintptr_t>(weights)) & 15) == 0;
    int idx[kAhead];
    float w[kAhead];
    auto fetch = [&](int j0) {
        t_next = group * per_cta + slot;
        at_next = part * width * kVec + lane * kEach;
        const bool live = t_next < tokens && at_next < c;
        const int32_t *from = index + t_next * topk + j0;
        const float *by = weights + t_next * topk + j0;
        if (kAhead % 4 == 0 && quads) {
#pragma unroll
            for (int j = 0; j + 3 < kAhead; j += 4) {
                int4 i4 = make_int4(-1, -1, -1, -1);
                float4 w4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (live && j0 + j < topk) {
                    i4 = *reinterpret_cast<const int4 *>(from + j);
                    w4 = *reinterpret_cast<const float4 *>(by + j);
                }
                idx[j] = i4.x, idx[j + 1] = i4.y, idx[j + 2] = i4.z, idx[j + 3] = i4.w;
                w[j] = w4.x, w[j + 1] = w4.y, w[j + 2] = w4.z, w[j + 3] = w4.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                idx[j] = live && j0 + j < topk ? from[j] : -1;
                w[j] = live && j0 + j < topk ? by[j] : 0.0f;
            }
        }
    };
    after_prior_kernels();
    fetch(0);
    while (group < groups) {
        const long long t = t_next;
        const int at = at_next;
        float acc[kVec];
#pragma unroll
        for (int q = 0; q < kVec; ++q) acc[q] = 0.0f;
        for (int j0 = 0; j0 < topk; j0 += kAhead) {
            U v[kAhead][kUnits];
            float p[kAhead];
            bool have[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                have[j] = idx[j] >= 0 && idx[j] < rows;
                p[j] = w[j];
                const T *from = y + (long long)idx[j] * ldy + at;
#pragma unroll
                for (int u = 0; u < kUnits; ++u)
                    if (have[j] && (kUnits == 1 || at + u * apart < c)) v[j][u] = *reinterpret_cast<const U *>(from + u * apart);
            }
            if (j0 + kAhead < topk) {
                fetch(j0 + kAhead);
            } else {
                group += step_group;
                part += step_part;
                if (part >= parts) {
                    part -= parts;
                    ++group;
                }
                fetch(0);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (have[j]) {
#pragma unroll
                    for (int u = 0; u < kUnits; ++u) {
                        const T *e = reinterpret_cast<const T *>(&v[j][u]);
#pragma unroll
                        for (int q = 0; q < kEach; ++q) acc[u * kEach + q] += p[j] * to_f32(e[q]);
                    }
                }
            }
        }
        if (t < tokens) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                U v;
                T *e = reinterpret_cast<T *>(&v);
#pragma unroll
                for (int q = 0; q < kEach; ++q) e[q] = from_f32<T>(acc[u * kEach + q]);
                if (at + u * apart < c) *reinterpret_cast<U *>(out + t * ldo + at + u * apart) = v;
            }
        }
    }
}

template <typename T>
auto combine_kernel(int unit, int ahead) {
    constexpr int kSmall = sizeof(T) == 2 ? 2 : 4;
    if (unit == 16)
        return ahead == 2   ? combine_rows_kernel<T, 16, 2>
               : ahead == 4 ? combine_rows_kernel<T, 16, 4>
                            : combine_rows_kernel<T, 16, 8>;
    if (unit == 4)
        return ahead == 2   ? combine_rows_kernel<T, 4, 2>
               : ahead == 4 ? combine_rows_kernel<T, 4, 4>
                            : combine_rows_kernel<T, 4, 8>;
    return ahead == 2   ? combine_rows_kernel<T, kSmall, 2>
           : ahead == 4 ? combine_rows_kernel<T, kSmall, 4>
                        : combine_rows_kernel<T, kSmall, 8>;
}

template <typename T>
cudaError_t combine_launch(const void *y, long long ldy, long long rows, const int32_t *index, const float *weights,
                           long long tokens, int topk, int c, void *out, long long ldo, int unit, int sms, cudaStream_t s) {
    const int per_thread = (unit == 16 ? 16 : 4 * unit) / (int)sizeof(T), per_row = (c + per_thread - 1) / per_thread;
    const int ahead = topk <= 2 ? 2 : topk <= 4 ? 4 : 8;
    int width = 4;
    while (width < per_row && width < 256) width *= 2;
    const long long items = (tokens + 256 / width - 1) / (256 / width) * ((per_row + width - 1) / width);
    const long long room = (long long)combine_ctas(ahead) * sms;
    auto k = combine_kernel<T>(unit, ahead);
    return launch_early(k, dim3((unsigned)(items < room ? items : room)), 256, 0, s, (const T *)y, ldy, rows, index, weights,
                        tokens, topk, c, (T *)out, ldo, width);
}

}  // namespace

cudaError_t launch_quantize_tokens(const TokenQuantArgs &a, int x_type, int format, cudaStream_t s) {
    const bool f16 = format == HATQ_CODES_F16;
    switch (x_type) {
        case HATQ_F32: return f16 ? quantize_size<float, true>(a, s) : quantize_size<float, false>(a, s);
        case HATQ_F16: return f16 ? quantize_size<__half, true>(a, s) : quantize_size<__half, false>(a, s);
        default: return f16 ? quantize_size<__nv_bfloat16, true>(a, s) : quantize_size<__nv_bfloat16, false>(a, s);
    }
}

cudaError_t launch_linear_layout(const int8_t *w, long long ldw, int experts, int n, int k, uint8_t *codes,
                                 int32_t *windows, cudaStream_t s) {
    const int n_tiles = (n + kRowTile - 1) / kRowTile, kb = (k + 63) / 64;
    const cudaError_t e = cudaMemsetAsync(windows, 0, (size_t)experts * 4, s);
    if (e != cudaSuccess) return e;
    linear_layout_kernel<<<experts * n_tiles, 128, 0, s>>>(w, ldw, n, k, n_tiles, kb, codes, windows);
    return cudaGetLastError();
}

cudaError_t launch_pack_codes(const void *x, int format, long long ldx, long long rows, int k, int k_pad, void *out,
                              cudaStream_t s) {
    const long long blocks = (rows * (k_pad / 8) + 255) / 256;
    return launch_early(pack_codes_kernel, dim3((unsigned)(blocks < 152 * 32 ? blocks : 152 * 32)), 256, 0, s, x, format, ldx,
                        rows, k, k_pad, (__half *)out);
}

namespace {
template <int MT, int R>
cudaError_t few_launch(const LinearArgs &a, cudaStream_t s) {
    const dim3 grid((a.n + 8 * R - 1) / (8 * R), a.offsets ? a.rows : 1);
    const int smem = MT * a.kb * 64;
    static std::atomic<int> allowed[64];
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(linear_few_kernel<MT, R>), smem, allowed);
    if (e != cudaSuccess) return e;
    return launch_early(linear_few_kernel<MT, R>, grid, kFewThreads, smem, s, a);
}
}  // namespace

// rows per pass: `tokens`. A short reduction leaves a thread few loads, so it takes two channels there.
cudaError_t launch_linear_few(const LinearArgs &a, int tokens, cudaStream_t s) {
    const bool two = a.kb <= 4 * kFewWarps && (long long)a.n * (a.offsets ? a.rows : 1) >= 152 * 32;
    switch (tokens) {
        case 1: return two ? few_launch<1, 2>(a, s) : few_launch<1, 1>(a, s);
        case 2: return two ? few_launch<2, 2>(a, s) : few_launch<2, 1>(a, s);
        case 4: return few_launch<4, 1>(a, s);
        default: return few_launch<8, 1>(a, s);
    }
}

cudaError_t launch_combine_rows(const void *y, int type, long long ldy, long long rows, const int32_t *index,
                                const float *weights, long long tokens, int topk, int c, void *out, long long ldo,
                                int unit, int sms, cudaStream_t s) {
    switch (type) {
        case HATQ_F32: return combine_launch<float>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, unit, sms, s);
        case HATQ_F16: return combine_launch<__half>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, unit, sms, s);
        default: return combine_launch<__nv_bfloat16>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, unit, sms, s);
    }
}

}  // namespace hatq
