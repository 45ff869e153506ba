// Keys and values of new tokens into the 4-bit cache.
#include "hatq_cache.h"

namespace hatq {
namespace {

// t = H~_hb x, a = max|t| over the head, code = round(7 t / a), scale = a / 7 / sqrt(hb); codes are stored + 8.
//
// The code is the rounding of the correctly rounded quotient (7 t) / a, so that whoever computes t alike gets the same
// codes. A multiplication by 7 / a gives the same but near the middle of two codes: both lie within 7 * 4 * 2^-24 <
// 2^-19 of 7 t / a, so only what comes within 2^-18 of a middle is divided.
//
// Memory-bound: the values' bytes. A lane owns 8 neighbouring values (16 bytes of a 16-bit type in, one word of codes
// out), LANES lanes a head; blocks wider than 8 cost one lane exchange per doubling.
__device__ __forceinline__ float code_of(float t, float a, float inv) {
    const float c = t * inv;
    float r = rintf(c);
    if (fabsf(fabsf(c - r) - 0.5f) < 0x1p-18f) r = rintf(__fdiv_rn(7.0f * t, a));
    return r;
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, bool vec, float (&v)[8]) {
    if (vec) {
        union { uint4 u[sizeof(T) / 2]; T t[8]; } x;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) x.u[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(x.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(p[i]);
    }
}

// neighbours first: distances 1, 2, 4 within the lane, then 8, 16, ... between lanes
template <int LANES>
__device__ __forceinline__ void transform(float (&v)[8], int hb, int lane) {
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
        if (h < hb)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(i & h)) {
                    const float a = v[i], b = v[i + h];
                    v[i] = a + b;
                    v[i + h] = a - b;
                }
#pragma unroll
    for (int h = 1; h < LANES; h *= 2)
        if (8 * h < hb)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float o = __shfl_xor_sync(0xffffffffu, v[i], h);
                v[i] = lane & h ? o - v[i] : v[i] + o;
            }
}

template <typename T, int LANES>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
    constexpr int kUnits = 32 / LANES;                       // (head, key or value) pairs of a warp
    after_prior_kernels();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, mine = lane % LANES;
    const int per_row = (2 * c.heads + kUnits - 1) / kUnits; // warps of a row
    const long long warp = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int r = (int)(warp / per_row);
    if (r >= c.rows) return;
    const int unit = (int)(warp % per_row) * kUnits + lane / LANES;
    const bool live = unit < 2 * c.heads && 8 * mine < c.width;
    const int part = unit & 1, head = unit >> 1;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    if (live) load8(static_cast<const T *>(a.x[part]) + r * a.ldx[part] + head * a.hx[part] + 8 * mine, a.vec, v);
    int b, begin, end;
    if (!sequence_of(c, r, lane, b, begin, end)) return;
    const int at = length_of(c, b) - end + r;
    int page = -1;
    if (at >= 0) page = c.table[b * c.ldt + (at >> c.page_bits)];      // at < length <= capacity

    transform<LANES>(v, c.hb, lane);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        most = fmaxf(most, fabsf(v[i]));
        if (v[i] != v[i]) most = __int_as_float(0x7f800000);
    }
#pragma unroll
    for (int h = 1; h < LANES; h *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, h));
    const bool sound = 7.0f * most < __int_as_float(0x7f800000), some = sound && most > 0.0f;
    // (7 / a overflows where a is subnormal: every value is then divided)
    const float inv = 7.0f / most;
    const bool fast = inv < __int_as_float(0x7f800000);
    uint32_t word = 0x88888888u;
    float n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = 0.0f;
    if (some) {
        word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = fast ? code_of(v[i], most, inv) : rintf(__fdiv_rn(7.0f * v[i], most));
            word |= (uint32_t)((int)n[i] + 8) << (4 * i);
        }
    }
    const float step = !sound ? __int_as_float(0x7fffffff) : some ? __fdiv_rn(most, 7.0f) * c.inv_norm : c.inv_norm;
    if (live && page >= 0 && page < c.pages) {
        const int size = 1 << c.page_bits, slot = at & (size - 1), half = c.width / 2;
        uint8_t *rec = c.data + ((long long)page * c.heads + head) * size * (c.width + 8);
        *reinterpret_cast<uint32_t *>(rec + (part * size + slot) * half + 4 * mine) = word;
        if (mine == 0) *reinterpret_cast<float *>(rec + size * c.width + 4 * (part * size + slot)) = step;
    }
    if (!a.kept[part]) return;
    // what the cache now stands for: the codes' transform is an integer, exact
    transform<LANES>(n, c.hb, lane);
    if (!live) return;
    const float back = step * c.inv_norm;
    T *kept = static_cast<T *>(a.kept[part]) + ((long long)r * c.heads + head) * c.width + 8 * mine;
    union { uint4 u[sizeof(T) / 2]; T t[8]; } y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y.t[i] = from_f32<T>(n[i] * back);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(kept)[i] = y.u[i];
}

template <typename T, int LANES>
cudaError_t launch(const AppendArgs &a, cudaStream_t s) {
    const long long warps = (long long)a.c.rows * ((2 * a.c.heads + 32 / LANES - 1) / (32 / LANES));
    return launch_early(append_kernel<T, LANES>, dim3((unsigned)((warps + 7) / 8)), 256, 0, s, a);
}
template <typename T>
cudaError_t launch_type(const AppendArgs &a, cudaStream_t s) {
    return a.c.width <= 64 ? launch<T, 8>(a, s) : a.c.width <= 128 ? launch<T, 16>(a, s) : launch<T, 32>(a, s);
}

}  // namespace

cudaError_t launch_append(const AppendArgs &a, int type, cudaStream_t s) {
    return type == HATQ_F32 ? launch_type<float>(a, s) : type == HATQ_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace hatq
