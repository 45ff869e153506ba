// The memory-bound token operators: quantize_tokens, the weight layout of
// linear, the packing of codes for the tensor cores, combine_rows, and the
// product for a few rows on the CUDA cores.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>

#include "hatq_tokens.h"

namespace hatq {
namespace {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ------------------------------------------------------------ quantize_tokens
//
// u = act(x) (times the row's second half where gated), t = H~_hb u,
// a = max |t|, code = clamp(rint(t * min(127 / a, 2^126))), scale =
// max(a / 127, 2^-126) / sqrt(hb). fp32 throughout, one rounding to the code.

constexpr int kPer = 32;               // consecutive values of one thread

template <typename T, bool VEC>
__device__ __forceinline__ void load_values(const T *p, int have, float (&v)[kPer]) {
    if (VEC && have >= kPer) {
        constexpr int kVec = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < kPer / kVec; ++i) {
            const uint4 w = reinterpret_cast<const uint4 *>(p)[i];
            const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[i * kVec + j] = to_f32(e[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i < have ? to_f32(p[i]) : 0.0f;
    }
}

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if (ACT == HATQ_ACT_RELU) return max_nan(v, 0.0f);
    if (ACT == HATQ_ACT_SILU) return v / (1.0f + expf(-v));
    if (ACT == HATQ_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    return v;
}

// tpr threads per row: a power of two below a warp, or whole warps; blockDim.x / tpr rows per CTA
template <typename T, int ACT, bool VEC, bool F16>
__global__ void __launch_bounds__(1024) quantize_tokens_kernel(const TokenQuantArgs a, int tpr) {
    __shared__ float warp_max[32];
    const int rl = threadIdx.x / tpr, t = threadIdx.x - rl * tpr;
    const long long row = (long long)blockIdx.x * (blockDim.x / tpr) + rl;
    const int have = row < a.rows ? min(kPer, max(0, a.c - t * kPer)) : 0;
    long long src = row;
    if (a.index && row < a.rows) src = a.index[row];
    float v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = 0.0f;
    if (have > 0 && src >= 0 && src < a.src_rows) {
        const T *p = reinterpret_cast<const T *>(a.x) + src * a.ldx + t * kPer;
        load_values<T, VEC>(p, have, v);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = activate<ACT>(v[i]);
        if (a.gated) {
            float u[kPer];
            load_values<T, VEC>(p + a.c, have, u);
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] *= u[i];
        }
    }
    // blocks of hb consecutive values: up to 32 in the thread, wider ones across hb / 32 lanes
#pragma unroll
    for (int h = 1; h < kPer; h <<= 1) {
        if (h < a.hb) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (i & h) continue;
                const float x = v[i], y = v[i + h];
                v[i] = x + y;
                v[i + h] = x - y;
            }
        }
    }
    for (int m = 1; m * kPer < a.hb; m <<= 1) {
        const bool upper = (t & m) != 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float o = __shfl_xor_sync(0xffffffffu, v[i], m);
            v[i] = upper ? o - v[i] : v[i] + o;
        }
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) amax = max_nan(amax, fabsf(v[i]));
    for (int m = min(tpr, 32) / 2; m > 0; m >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, m));
    if (tpr > 32) {
        const int warps = tpr / 32, w0 = rl * warps;
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = amax;
        __syncthreads();
        for (int w = 0; w < warps; ++w) amax = max_nan(amax, warp_max[w0 + w]);
    }
    if (have <= 0) return;
    const bool fine = amax <= 3.402823466e38f;                          // false for infinity and NaN
    // 127 / a overflows below 127 / 2^128: the step stays at the smallest normal number there
    const float inv = !fine || amax == 0.0f ? 0.0f : fminf(127.0f / amax, 0x1p126f);
    if (t == 0)
        a.scales[row] = !fine ? __int_as_float(0x7fc00000)
                              : (amax == 0.0f ? 1.0f : fmaxf(amax / 127.0f, 0x1p-126f) * a.inv_norm);
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = fine ? fminf(fmaxf(rintf(v[i] * inv), -127.0f), 127.0f) : 0.0f;
    if (F16) {
        __half *q = reinterpret_cast<__half *>(a.codes) + row * a.ldc + t * kPer;
        if (VEC && have >= kPer) {
#pragma unroll
            for (int i = 0; i < kPer / 8; ++i) {
                uint4 w;
                __half2 *h = reinterpret_cast<__half2 *>(&w);
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j] = __floats2half2_rn(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
                reinterpret_cast<uint4 *>(q)[i] = w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < have) q[i] = __float2half_rn(v[i]);
        }
    } else {
        int8_t *q = reinterpret_cast<int8_t *>(a.codes) + row * a.ldc + t * kPer;
        if (VEC && have >= kPer) {
#pragma unroll
            for (int i = 0; i < kPer / 16; ++i) {
                uint4 w;
                int8_t *b = reinterpret_cast<int8_t *>(&w);
#pragma unroll
                for (int j = 0; j < 16; ++j) b[j] = (int8_t)(int)v[16 * i + j];
                reinterpret_cast<uint4 *>(q)[i] = w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (i < have) q[i] = (int8_t)(int)v[i];
        }
    }
}

template <typename T, int ACT>
cudaError_t quantize_launch(const TokenQuantArgs &a, int format, bool vec, cudaStream_t s) {
    const int need = (a.c + kPer - 1) / kPer;
    int tpr = 1;
    if (need > 32) tpr = (need + 31) & ~31;
    else
        while (tpr < need) tpr <<= 1;
    const int per_cta = tpr >= 256 ? 1 : 256 / tpr;
    const long long grid = (a.rows + per_cta - 1) / per_cta;
    const int threads = ((per_cta * tpr + 31) / 32) * 32;
    if (grid > INT_MAX) return cudaErrorInvalidValue;
    void (*k)(TokenQuantArgs, int) =
        format == HATQ_CODES_F16 ? (vec ? quantize_tokens_kernel<T, ACT, true, true> : quantize_tokens_kernel<T, ACT, false, true>)
                                 : (vec ? quantize_tokens_kernel<T, ACT, true, false> : quantize_tokens_kernel<T, ACT, false, false>);
    k<<<(unsigned)grid, threads, 0, s>>>(a, tpr);
    return cudaGetLastError();
}

template <typename T>
cudaError_t quantize_act(const TokenQuantArgs &a, int format, bool vec, cudaStream_t s) {
    switch (a.act) {
        case HATQ_ACT_NONE: return quantize_launch<T, HATQ_ACT_NONE>(a, format, vec, s);
        case HATQ_ACT_RELU: return quantize_launch<T, HATQ_ACT_RELU>(a, format, vec, s);
        case HATQ_ACT_SILU: return quantize_launch<T, HATQ_ACT_SILU>(a, format, vec, s);
        default: return quantize_launch<T, HATQ_ACT_GELU>(a, format, vec, s);
    }
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

__global__ void __launch_bounds__(256) pack_codes_kernel(const void *x, int format, long long ldx, long long rows, int k,
                                                         int k_pad, __half *out) {
    const int per_row = k_pad / 8;
    const long long total = rows * per_row;
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
// A CTA owns 8 channels of one group and the whole reduction; a warp takes
// every 8th 64-code block, a lane 16 codes of one channel (8 lanes read 128
// consecutive bytes). The weights' loads are issued before the rows' codes are
// brought to shared memory, so both latencies run together. Sums are int32.

constexpr int kFewThreads = 256, kFewCh = 8;

__device__ __forceinline__ void store_y(void *y, int type, long long at, float v) {
    if (type == HATQ_F32) reinterpret_cast<float *>(y)[at] = v;
    else if (type == HATQ_F16) reinterpret_cast<__half *>(y)[at] = __float2half_rn(v);
    else reinterpret_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
}

template <int MT>
__global__ void __launch_bounds__(kFewThreads) linear_few_kernel(const LinearArgs a) {
    extern __shared__ __align__(16) uint8_t xs[];                       // [MT][k_pad] codes
    __shared__ int part[kFewThreads / 32][kFewCh][MT];
    __shared__ int s_group, s_count;
    const int k_pad = a.kb * 64;
    int e = 0, r0 = 0, r1 = a.rows;
    if (a.offsets) {
        // the blockIdx.y-th group that holds rows
        if (threadIdx.x == 0) { s_group = -1; s_count = 0; }
        __syncthreads();
        for (int g0 = 0; g0 < a.experts; g0 += kFewThreads) {
            const int g = g0 + threadIdx.x;
            const bool holds = g < a.experts && min(a.offsets[g + 1], a.rows) > max(a.offsets[g], 0);
            const unsigned ball = __ballot_sync(0xffffffffu, holds);
            __shared__ int warps[kFewThreads / 32];
            if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = __popc(ball);
            __syncthreads();
            int before = s_count;
            for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) before += warps[w];
            before += __popc(ball & ((1u << (threadIdx.x & 31)) - 1));
            if (holds && before == (int)blockIdx.y) s_group = g;
            __syncthreads();
            if (threadIdx.x == 0)
                for (int w = 0; w < kFewThreads / 32; ++w) s_count += warps[w];
            __syncthreads();
        }
        e = s_group;
        if (e < 0) return;
        r0 = max(a.offsets[e], 0);
        r1 = min(a.offsets[e + 1], a.rows);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ch_l = lane & 7, j = lane >> 3;
    const int ch0 = blockIdx.x * kFewCh;
    const uint8_t *wp = a.w + ((long long)e * a.n_tiles + ch0 / kRowTile) * a.kb * kBlockBytes + j * 2048 +
                        ((ch0 % kRowTile) + ch_l) * 16;
    constexpr int kAhead = 8;
    for (int base = r0; base < r1; base += MT) {
        int acc[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = 0;
        uint4 w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int b = warp + 8 * i;
            w[i] = b < a.kb ? *reinterpret_cast<const uint4 *>(wp + (long long)b * kBlockBytes) : make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < MT * (k_pad / 16); i += kFewThreads) {
            const int t = i / (k_pad / 16), c = (i - t * (k_pad / 16)) * 16;
            const long long r = base + t;
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
                    for (int q = 0; q < 16; ++q) b[q] = c + q < a.k ? (int8_t)__half2int_rn(p[q]) : 0;
                }
            }
            *reinterpret_cast<uint4 *>(xs + t * k_pad + c) = v;
        }
        __syncthreads();
        for (int b0 = warp;; ) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int b = b0 + 8 * i;
                if (b < a.kb) {
                    const uint32_t q[4] = {w[i].x ^ 0x80808080u, w[i].y ^ 0x80808080u, w[i].z ^ 0x80808080u,
                                           w[i].w ^ 0x80808080u};
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(xs + t * k_pad + b * 64 + j * 16);
                        acc[t] = __dp4a((int)q[0], (int)x.x, acc[t]);
                        acc[t] = __dp4a((int)q[1], (int)x.y, acc[t]);
                        acc[t] = __dp4a((int)q[2], (int)x.z, acc[t]);
                        acc[t] = __dp4a((int)q[3], (int)x.w, acc[t]);
                    }
                }
            }
            b0 += 8 * kAhead;
            if (b0 - warp >= a.kb) break;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int b = b0 + 8 * i;
                if (b < a.kb) w[i] = *reinterpret_cast<const uint4 *>(wp + (long long)b * kBlockBytes);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 8);
            acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 16);
            if (j == 0) part[warp][ch_l][t] = acc[t];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kFewCh * MT; i += kFewThreads) {
            const int t = i / kFewCh, c = i % kFewCh;
            if (base + t < r1 && ch0 + c < a.n) {
                int sum = 0;
                for (int q = 0; q < kFewThreads / 32; ++q) sum += part[q][c][t];
                const long long ch = (long long)e * a.n + ch0 + c;
                float v = (float)sum * a.s_w[ch] * a.s_x[base + t];
                if (a.bias) v += a.bias[ch];
                store_y(a.y, a.y_type, (base + t) * a.ldy + ch0 + c, v);
            }
        }
    }
}

// ------------------------------------------------------------ combine_rows

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) combine_rows_kernel(const T *y, long long ldy, long long rows, const int32_t *index,
                                                           const float *weights, long long tokens, int topk, int c, T *out,
                                                           long long ldo) {
    constexpr int kVec = VEC ? 16 / sizeof(T) : 1;
    const int per_row = (c + kVec - 1) / kVec;
    const long long total = tokens * per_row;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const long long t = i / per_row;
        const int at = (int)(i - t * per_row) * kVec;
        float acc[kVec];
#pragma unroll
        for (int q = 0; q < kVec; ++q) acc[q] = 0.0f;
        for (int j = 0; j < topk; ++j) {
            const long long r = index[t * topk + j];
            if (r < 0 || r >= rows) continue;
            const float w = weights[t * topk + j];
            if (VEC) {
                const uint4 v = *reinterpret_cast<const uint4 *>(y + r * ldy + at);
                const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
                for (int q = 0; q < kVec; ++q) acc[q] += w * to_f32(e[q]);
            } else {
                acc[0] += w * to_f32(y[r * ldy + at]);
            }
        }
        if (VEC) {
            uint4 v;
            T *e = reinterpret_cast<T *>(&v);
#pragma unroll
            for (int q = 0; q < kVec; ++q) e[q] = from_f32<T>(acc[q]);
            *reinterpret_cast<uint4 *>(out + t * ldo + at) = v;
        } else {
            out[t * ldo + at] = from_f32<T>(acc[0]);
        }
    }
}

template <typename T>
cudaError_t combine_launch(const void *y, long long ldy, long long rows, const int32_t *index, const float *weights,
                           long long tokens, int topk, int c, void *out, long long ldo, bool vec, cudaStream_t s) {
    const int kvec = vec ? 16 / (int)sizeof(T) : 1;
    const long long blocks = (tokens * ((c + kvec - 1) / kvec) + 255) / 256;
    const unsigned grid = (unsigned)(blocks < (1LL << 30) ? blocks : (1LL << 30));
    if (vec)
        combine_rows_kernel<T, true><<<grid, 256, 0, s>>>((const T *)y, ldy, rows, index, weights, tokens, topk, c, (T *)out, ldo);
    else
        combine_rows_kernel<T, false><<<grid, 256, 0, s>>>((const T *)y, ldy, rows, index, weights, tokens, topk, c, (T *)out, ldo);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize_tokens(const TokenQuantArgs &a, int x_type, int format, bool vec, cudaStream_t s) {
    switch (x_type) {
        case HATQ_F32: return quantize_act<float>(a, format, vec, s);
        case HATQ_F16: return quantize_act<__half>(a, format, vec, s);
        default: return quantize_act<__nv_bfloat16>(a, format, vec, s);
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
    pack_codes_kernel<<<(unsigned)(blocks < 152 * 32 ? blocks : 152 * 32), 256, 0, s>>>(x, format, ldx, rows, k, k_pad,
                                                                                     (__half *)out);
    return cudaGetLastError();
}

cudaError_t launch_linear_few(const LinearArgs &a, int tokens, cudaStream_t s) {
    const dim3 grid((a.n + kFewCh - 1) / kFewCh, a.offsets ? a.slots : 1);
    const int smem = tokens * a.kb * 64;
    void (*k)(LinearArgs) = tokens == 1   ? linear_few_kernel<1>
                            : tokens == 2 ? linear_few_kernel<2>
                            : tokens == 4 ? linear_few_kernel<4>
                                          : linear_few_kernel<8>;
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    k<<<grid, kFewThreads, smem, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_combine_rows(const void *y, int type, long long ldy, long long rows, const int32_t *index,
                                const float *weights, long long tokens, int topk, int c, void *out, long long ldo,
                                bool vec, cudaStream_t s) {
    switch (type) {
        case HATQ_F32: return combine_launch<float>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, vec, s);
        case HATQ_F16: return combine_launch<__half>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, vec, s);
        default: return combine_launch<__nv_bfloat16>(y, ldy, rows, index, weights, tokens, topk, c, out, ldo, vec, s);
    }
}

}  // namespace hatq
