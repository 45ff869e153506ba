// Products with 4-bit weights that have one scale per group of inputs.
#include <climits>
#include <type_traits>

#include "hatq_linear4.h"
#include "hatq_mma4.h"

namespace hatq {
namespace {

// y[r][n] = s_x[r] sum_g s[n][g] sum_{k in g} c[n][k] x[r][k] + bias[n].
//
// The inner sums run on the tensor cores as W x^T in m16n8k16 steps, 16 channels by 8 rows of x: codes are exact in
// both 16-bit types, so 16-bit x go in as they are and fp32 x as the sum of three bf16 numbers, which is exact. A
// group's sum is scaled in fp32 and added to the total.
//
// Memory-bound by the weights for few rows. Every lane reads its codes of 16 channels x 64 inputs as 16 bytes, whole
// lines in order; the CTA's warps take every so many of these blocks, and their sums are added in shared memory.
// x is read as it lies, 16 bytes a lane and 32 inputs (the order of inputs within a step is free: lane t of four has
// inputs 8 t .. 8 t + 7 of each 32, the first four in the first step).

constexpr int kCtaWarps = 8;

template <typename T> constexpr int kParts = std::is_same<T, float>::value ? 3 : 1;

// 8 inputs of a row as B operands of two steps: b[part][step][2]
template <typename T>
__device__ __forceinline__ void load_x(const Linear4Args &a, const T *row, bool live, int k, uint32_t (&b)[kParts<T>][2][2]) {
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
        // the upper 16 bits are a bf16 number, and what is left has 16, then 8 bits; nothing is left of an infinity
#pragma unroll
        for (int part = 0; part < 3; ++part)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t x = __float_as_uint(v[i]), y = __float_as_uint(v[i + 1]);
                b[part][i / 4][i / 2 % 2] = __byte_perm(x, y, 0x7632);
                v[i] = (x & 0x7f800000u) == 0x7f800000u ? 0.0f : v[i] - __uint_as_float(x & 0xffff0000u);
                v[i + 1] = (y & 0x7f800000u) == 0x7f800000u ? 0.0f : v[i + 1] - __uint_as_float(y & 0xffff0000u);
            }
    } else {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (live && a.vec && k + 8 <= a.k) {
            x = __ldg(reinterpret_cast<const uint4 *>(row + k));
        } else if (live) {
            const unsigned short *p = reinterpret_cast<const unsigned short *>(row) + k;
            unsigned short v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < a.k ? p[i] : 0;
            x = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
        b[0][0][0] = x.x;
        b[0][0][1] = x.y;
        b[0][1][0] = x.z;
        b[0][1][1] = x.w;
    }
}

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

// NT tiles of 8 rows, MS strips a warp. `ways` warps of the CTA share a strip's inputs.
template <typename T, typename Y, int NT, int MS>
__global__ void __launch_bounds__(kCtaWarps * 32, 2) linear4_kernel(const Linear4Args a, int ways) {
    constexpr int ROWS = 8 * NT, C = kStrip * MS;
    extern __shared__ float sums[];                          // [warp][row][channel + 4]
    after_prior_kernels();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int sets = kCtaWarps / ways, way = warp % ways;
    const int blocks = (a.k + kStep - 1) / kStep, strips = (a.n + kStrip - 1) / kStrip;
    const int strip0 = (blockIdx.x * sets + warp / ways) * MS, row0 = blockIdx.y * ROWS;

    float total[MS][NT][4];
#pragma unroll
    for (int m = 0; m < MS; ++m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) total[m][nt][i] = 0.0f;
    const uint4 *w[MS];
    const float *scales[MS];
#pragma unroll
    for (int m = 0; m < MS; ++m) {
        const int strip = min(strip0 + m, strips - 1);       // (what lies behind the last is computed twice and not written)
        w[m] = reinterpret_cast<const uint4 *>(a.w) + (long long)strip * blocks * 32 + lane;
        scales[m] = a.scales + (long long)strip * a.groups * kStrip + g;
    }
    const T *x[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x[nt] = static_cast<const T *>(a.x) + (long long)min(row0 + 8 * nt + g, a.rows - 1) * a.ldx;
    const bool fine = a.group % kStep != 0;                  // a block holds two groups

    uint4 next[MS];
    if (way < blocks)
#pragma unroll
        for (int m = 0; m < MS; ++m) next[m] = __ldcs(w[m] + (long long)way * 32);
    for (int block = way; block < blocks; block += ways) {
        uint4 now[MS];
#pragma unroll
        for (int m = 0; m < MS; ++m) now[m] = next[m];
        if (block + ways < blocks)
#pragma unroll
            for (int m = 0; m < MS; ++m) next[m] = __ldcs(w[m] + (long long)(block + ways) * 32);
        float sum[MS][NT][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = block * kStep + 32 * j;
            if (j == 0 || fine)
#pragma unroll
                for (int m = 0; m < MS; ++m)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[m][nt][i] = 0.0f;
            uint32_t A[MS][2][4];
#pragma unroll
            for (int m = 0; m < MS; ++m) {
                widen<T>(j ? now[m].z : now[m].x, A[m][0]);
                widen<T>(j ? now[m].w : now[m].y, A[m][1]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                uint32_t b[kParts<T>][2][2];
                load_x<T>(a, x[nt], row0 + 8 * nt + g < a.rows, k + 8 * t, b);
#pragma unroll
                for (int part = kParts<T> - 1; part >= 0; --part)
#pragma unroll
                    for (int m = 0; m < MS; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if constexpr (std::is_same<T, __half>::value)
                                mma(sum[m][nt], A[m][h], b[part][h][0], b[part][h][1]);
                            else
                                mma_bf16(sum[m][nt], A[m][h], b[part][h][0], b[part][h][1]);
                        }
            }
            if (j == 1 || fine) {
                const int group = min(k / a.group, a.groups - 1);        // (behind the last input: sums are 0)
#pragma unroll
                for (int m = 0; m < MS; ++m) {
                    const float s0 = __ldg(scales[m] + group * kStrip), s1 = __ldg(scales[m] + group * kStrip + 8);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        total[m][nt][0] = fmaf(s0, sum[m][nt][0], total[m][nt][0]);
                        total[m][nt][1] = fmaf(s0, sum[m][nt][1], total[m][nt][1]);
                        total[m][nt][2] = fmaf(s1, sum[m][nt][2], total[m][nt][2]);
                        total[m][nt][3] = fmaf(s1, sum[m][nt][3], total[m][nt][3]);
                    }
                }
            }
        }
    }
    // ---- the warps' sums, then scale, bias and the output type
    constexpr int PITCH = C + 4;
    float *mine = sums + warp * ROWS * PITCH;
#pragma unroll
    for (int m = 0; m < MS; ++m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(8 * nt + 2 * t + (i & 1)) * PITCH + 16 * m + g + (i >> 1) * 8] = total[m][nt][i];
    __syncthreads();
    const int live = min(ROWS, a.rows - row0);
    for (int i = threadIdx.x; i < live * C * sets; i += kCtaWarps * 32) {
        const int ch = i % C, set = i / C % sets, row = i / (C * sets), n = (blockIdx.x * sets + set) * C + ch;
        if (n >= a.n) continue;
        float v = 0.0f;
        for (int j = 0; j < ways; ++j) v += sums[((set * ways + j) * ROWS + row) * PITCH + ch];
        if (a.s_x) v *= __ldg(a.s_x + row0 + row);
        if (a.bias) v += __ldg(a.bias + n);
        static_cast<Y *>(a.y)[(long long)(row0 + row) * a.ldy + n] = from_f32<Y>(v);
    }
}

template <typename T, typename Y, int NT, int MS>
cudaError_t launch(const Linear4Args &a, int ways, cudaStream_t s) {
    static std::atomic<int> allowed[64];
    constexpr int bytes = kCtaWarps * 8 * NT * (kStrip * MS + 4) * 4;
    const cudaError_t e = allow_shared(reinterpret_cast<const void *>(linear4_kernel<T, Y, NT, MS>), bytes, allowed);
    if (e != cudaSuccess) return e;
    const int channels = kStrip * MS * (kCtaWarps / ways);
    return launch_early(linear4_kernel<T, Y, NT, MS>, dim3((unsigned)((a.n + channels - 1) / channels), (unsigned)((a.rows + 8 * NT - 1) / (8 * NT))),
                        kCtaWarps * 32, bytes, s, a, ways);
}
template <typename T, typename Y>
cudaError_t launch_rows(const Linear4Args &a, cudaStream_t s) {
    const int blocks = (a.k + kStep - 1) / kStep, ways = blocks >= 8 ? 8 : blocks >= 4 ? 4 : blocks >= 2 ? 2 : 1;
    if (a.rows <= 8) return launch<T, Y, 1, 1>(a, ways, s);
    if (a.rows <= 16) return launch<T, Y, 2, 2>(a, ways, s);
    return launch<T, Y, 4, 2>(a, ways, s);
}
template <typename T>
cudaError_t launch_type(const Linear4Args &a, cudaStream_t s) {
    switch (a.y_type) {
        case HATQ_F32: return launch_rows<T, float>(a, s);
        case HATQ_F16: return launch_rows<T, __half>(a, s);
        default: return launch_rows<T, __nv_bfloat16>(a, s);
    }
}

// A warp per strip and block: lane (g, t) packs channels g and g + 8 (the first in the lower of two nibbles) at inputs
// 8 t .. 8 t + 7 of each half of the block; a word has four inputs, their pairs 16 bits apart.
__global__ void __launch_bounds__(256) layout_kernel(const int8_t *w, long long ldw, int n, int k, int strips, int blocks, uint4 *out) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (unit >= (long long)strips * blocks) return;
    const int strip = (int)(unit / blocks), block = (int)(unit % blocks);
    uint32_t words[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        words[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {                        // input j & 3 of the word, channel g + 8 (j >> 2)
            const int row = strip * kStrip + g + (j >> 2) * 8, col = block * kStep + (i >> 1) * 32 + 8 * t + (i & 1) * 4 + (j & 3);
            const int code = row < n && col < k ? min(max((int)w[row * ldw + col], -8), 7) : 0;
            const int nibble = (j & 1) * 4 + ((j >> 1) & 1) * 2 + (j >> 2);
            words[i] |= (uint32_t)(code + 8) << (4 * nibble);
        }
    }
    out[unit * 32 + lane] = make_uint4(words[0], words[1], words[2], words[3]);
}
__global__ void __launch_bounds__(256) scales_kernel(const float *scales, long long lds, int n, int groups, long long total, float *out) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int ch = (int)(i % kStrip), group = (int)(i / kStrip % groups), row = (int)(i / ((long long)kStrip * groups)) * kStrip + ch;
    out[i] = row < n ? scales[row * lds + group] : 0.0f;
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
    const int lane = threadIdx.x & 31, groups = (k + group - 1) / group;
    for (int g = threadIdx.x >> 5; g < groups; g += 8) {
        const int from = g * group, to = min(k, from + group);
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
    return x_type == HATQ_F32 ? launch_type<float>(a, s) : x_type == HATQ_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}
cudaError_t launch_linear4_layout(const int8_t *w, long long ldw, const float *scales, long long lds, int n, int k, int groups,
                                  uint8_t *codes, float *out_scales, cudaStream_t s) {
    const int strips = (n + kStrip - 1) / kStrip, blocks = (k + kStep - 1) / kStep;
    const long long units = (long long)strips * blocks, total = (long long)strips * kStrip * groups;
    layout_kernel<<<(unsigned)((units + 7) / 8), 256, 0, s>>>(w, ldw, n, k, strips, blocks, reinterpret_cast<uint4 *>(codes));
    scales_kernel<<<(unsigned)((total + 255) / 256), 256, 0, s>>>(scales, lds, n, groups, total, out_scales);
    return cudaGetLastError();
}
cudaError_t launch_quantize_groups(const void *w, int type, long long ldw, int n, int k, int hb, int group, int8_t *codes,
                                   long long ldc, float *scales, long long lds, cudaStream_t s) {
    return type == HATQ_F32    ? quantize_type<float>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s)
           : type == HATQ_F16 ? quantize_type<__half>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s)
                              : quantize_type<__nv_bfloat16>(w, ldw, n, k, hb, group, codes, ldc, scales, lds, s);
}

}  // namespace hatq
