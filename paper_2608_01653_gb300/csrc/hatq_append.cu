// Keys and values of new tokens into the 4-bit cache.
#include <type_traits>

#include "hatq_cache.h"

namespace hatq {
namespace {

// t = H~_hb x, a = max|t| over the head, code = round(7 t / a), scale = a / 7 / sqrt(hb); codes are stored + 8.
//
// The code is the rounding of the correctly rounded quotient (7 t) / a, so that whoever computes t alike gets the same
// codes. A multiplication by 7 / a gives the same but near the middle of two codes: both lie within 7 * 4 * 2^-24 <
// 2^-19 of 7 t / a, so where a value of the lane comes within 2^-18 of a middle the lane divides.
//
// The values' bytes are the floor, but instructions come first (issue 0.68; keys and values of 9165 tokens of 8 heads of
// 128, 85 MB with what is handed back: 25 us, 3.4 TB/s). A warp has 8 heads, lane (g, t) of head g the values 64 c + 16 t .. + 15, so that 4 of 6 doublings (distances 16 and 32 are the
// exceptions) stay within a lane. What the cache now stands for is transformed back in pairs of fp16: sums of codes are
// whole numbers below 2^11, exact.
template <typename T>
__device__ __forceinline__ void load16(const T *p, bool vec, float *v) {
    if (vec) {
        union { uint4 u[sizeof(T)]; T t[16]; } x;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) x.u[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = to_f32<T>(x.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = to_f32<T>(p[i]);
    }
}

// Neighbours first: distances 1 .. 8 within the lane, 16 and 32 between lanes, 64 and 128 between a lane's runs of 16.
// FULL: hb is all of it, known to the compiler, which then need not bring results back to where they were for a stage that
// may be left out (a seventh of all instructions).
template <int N, bool FULL>
__device__ __forceinline__ void transform(float (&v)[N], int hb, int t) {
#pragma unroll
    for (int h = 1; h < 16; h *= 2)
        if (FULL || h < hb)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(i & h)) {
                    const float a = v[i], b = v[i + h];
                    v[i] = a + b;
                    v[i + h] = a - b;
                }
#pragma unroll
    for (int h = 1; h < 4; h *= 2)
        if (FULL || 16 * h < hb) {
            const float sign = t & h ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = fmaf(sign, v[i], __shfl_xor_sync(0xffffffffu, v[i], h));
        }
#pragma unroll
    for (int h = 16; h < (FULL ? N & -N : N); h *= 2)
        if (FULL || 4 * h < hb)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(i & h) && i + h < N) {
                    const float a = v[i], b = v[i + h];
                    v[i] = a + b;
                    v[i + h] = a - b;
                }
}

// the same of whole numbers in pairs (2 i, 2 i + 1)
template <int N, bool FULL>
__device__ __forceinline__ void transform_pairs(__half2 (&v)[N / 2], int hb, int t) {
    if (FULL || hb > 1) {
        const __half2 sign = __halves2half2(__float2half_rn(1.0f), __float2half_rn(-1.0f));
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = __hfma2(v[i], sign, __lowhigh2highlow(v[i]));
    }
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
        if (FULL || 2 * h < hb)
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (!(i & h)) {
                    const __half2 a = v[i], b = v[i + h];
                    v[i] = __hadd2(a, b);
                    v[i + h] = __hsub2(a, b);
                }
#pragma unroll
    for (int h = 1; h < 4; h *= 2)
        if (FULL || 16 * h < hb) {
            const __half2 sign = __float2half2_rn(t & h ? -1.0f : 1.0f);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[i] = __hfma2(sign, v[i], __shfl_xor_sync(0xffffffffu, v[i], h));
        }
#pragma unroll
    for (int h = 8; h < (FULL ? (N & -N) / 2 : N / 2); h *= 2)
        if (FULL || 8 * h < hb)
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (!(i & h) && i + h < N / 2) {
                    const __half2 a = v[i], b = v[i + h];
                    v[i] = __hadd2(a, b);
                    v[i + h] = __hsub2(a, b);
                }
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// C runs of 16 values a lane: heads of 64 C. Keys where blockIdx.y is 0, values where it is 1.
template <typename T, int C, bool FULL>
__global__ void __launch_bounds__(256, C <= 2 ? 3 : 1) append_kernel(const AppendArgs a) {
    constexpr int N = 16 * C;
    after_prior_kernels();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, part = blockIdx.y;
    const long long heads = (long long)c.rows * c.heads, first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 8;
    if (first >= heads) return;
    const bool live = first + g < heads;
    const uint32_t unit = (uint32_t)(live ? first + g : heads - 1);
    const int r = (int)(unit / (uint32_t)c.heads), head = (int)(unit - (uint32_t)r * c.heads);
    float v[N];
    const T *x = static_cast<const T *>(a.x[part]) + r * a.ldx[part] + head * a.hx[part] + 16 * t;
#pragma unroll
    for (int i = 0; i < C; ++i) load16(x + 64 * i, a.vec, v + 16 * i);
    // ---- the row's place: at in its sequence, and the page there
    int b = r, at = -1, page = -1;
    bool held = live;
    if (c.starts) {
        held = false;
        const int last = __shfl_sync(0xffffffffu, r, 31);
        for (int row = __shfl_sync(0xffffffffu, r, 0); row <= last; ++row) {
            int of, begin, end;
            if (sequence_of(c, row, lane, of, begin, end) && row == r && live) {
                held = true;
                b = of;
                at = row - end;
            }
        }
    }
    if (held) {
        at += length_of(c, b);
        if (at >= 0) page = c.table[b * c.ldt + (at >> c.page_bits)];            // at < length <= capacity
    }

    transform<N, FULL>(v, c.hb, t);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        most = max_nan(most, fabsf(v[i]));
    }
#pragma unroll
    for (int h = 1; h < 4; h *= 2) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, h));
    const bool sound = 7.0f * most < __int_as_float(0x7f800000), some = sound && most > 0.0f;
    // (7 / a overflows where a is subnormal: every value is then divided)
    const float inv = some ? 7.0f / most : 0.0f;
    float worst = inv < __int_as_float(0x7f800000) ? 0.0f : 1.0f;
    float n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float q = v[i] * inv;
        n[i] = rintf(q);
        worst = fmaxf(worst, fabsf(q - n[i]));
    }
    if (some && worst > 0.5f - 0x1p-18f)
#pragma unroll
        for (int i = 0; i < N; ++i) n[i] = rintf(__fdiv_rn(7.0f * v[i], most));
    if (!some)
#pragma unroll
        for (int i = 0; i < N; ++i) n[i] = 0.0f;
    const float step = !sound ? __int_as_float(0x7fffffff) : some ? __fdiv_rn(most, 7.0f) * c.inv_norm : c.inv_norm;
    if (held && page >= 0 && page < c.pages) {
        const int size = 1 << c.page_bits, slot = at & (size - 1);
        uint8_t *rec = c.data + ((long long)page * c.heads + head) * size * (64 * C + 8);
        uint2 *words = reinterpret_cast<uint2 *>(rec + (part * size + slot) * (32 * C) + 8 * t);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            // four codes + 8 at a time as a number below 2^16, exact in fp32
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *m = n + 16 * i + 4 * j;
                q[j] = (uint32_t)fmaf(m[3], 4096.0f, fmaf(m[2], 256.0f, fmaf(m[1], 16.0f, m[0] + 34952.0f)));
            }
            words[4 * i] = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
        }
        if (t == 0) *reinterpret_cast<float *>(rec + size * (64 * C) + 4 * (part * size + slot)) = step;
    }
    if (!a.kept[part]) return;
    // ---- what the cache now stands for
    __half2 pairs[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) pairs[i] = __floats2half2_rn(n[2 * i], n[2 * i + 1]);
    transform_pairs<N, FULL>(pairs, c.hb, t);
    if (!held) return;
    const float back = step * c.inv_norm;
    T *kept = static_cast<T *>(a.kept[part]) + ((long long)r * c.heads + head) * (64 * C) + 16 * t;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        union { uint4 u[sizeof(T)]; T t[16]; } y;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 f = __half22float2(pairs[8 * i + j]);
            y.t[2 * j] = from_f32<T>(f.x * back);
            y.t[2 * j + 1] = from_f32<T>(f.y * back);
        }
#pragma unroll
        for (int j = 0; j < (int)sizeof(T); ++j) reinterpret_cast<uint4 *>(kept + 64 * i)[j] = y.u[j];
    }
}

template <typename T, int C>
cudaError_t launch(const AppendArgs &a, cudaStream_t s) {
    const dim3 grid((unsigned)(((long long)a.c.rows * a.c.heads + 63) / 64), 2);
    constexpr int all = 64 * C & -(64 * C);
    return a.c.hb == all ? launch_early(append_kernel<T, C, true>, grid, 256, 0, s, a) : launch_early(append_kernel<T, C, false>, grid, 256, 0, s, a);
}
template <typename T>
cudaError_t launch_type(const AppendArgs &a, cudaStream_t s) {
    return a.c.width == 64    ? launch<T, 1>(a, s)
           : a.c.width == 128 ? launch<T, 2>(a, s)
           : a.c.width == 192 ? launch<T, 3>(a, s)
                              : launch<T, 4>(a, s);
}

}  // namespace

cudaError_t launch_append(const AppendArgs &a, int type, cudaStream_t s) {
    return type == HATQ_F32 ? launch_type<float>(a, s) : type == HATQ_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace hatq
