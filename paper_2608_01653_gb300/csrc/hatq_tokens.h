// Internal interface of the token operators (quantize_tokens, linear,
// grouped_linear, combine_rows) between the host side (hatq_tokens_api.cu) and
// the kernels. Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <thread>

#include "hatq.h"

namespace hatq {

constexpr int kRowTile = 128;          // output channels per block of the weight layout
constexpr int kBlockBytes = 8192;      // one block: 128 channels x 64 codes
constexpr int kMaxExperts = 1024;
constexpr int kMaxTokenWidth = 32768;  // values per row of quantize_tokens
constexpr int kMaxDepth = 65536;       // reduction length of a product: 128 * 128 * 65536 < 2^31

struct TokenQuantArgs {
    const void *x;
    long long ldx, src_rows;
    const int32_t *index;
    long long rows;
    int c, hb, act, gated;
    int sms;                           // of the device
    bool vec;                          // rows of x and codes lie on 16-byte boundaries
    float inv_norm;                    // 1 / sqrt(hb)
    void *codes;
    long long ldc;
    float *scales;
};
cudaError_t launch_quantize_tokens(const TokenQuantArgs &a, int x_type, int format, cudaStream_t s);

cudaError_t launch_linear_layout(const int8_t *w, long long ldw, int experts, int n, int k, uint8_t *codes,
                                 int32_t *windows, cudaStream_t s);
// codes of either format and any pitch -> fp16 codes [rows][k_pad], zero behind k
cudaError_t launch_pack_codes(const void *x, int format, long long ldx, long long rows, int k, int k_pad, void *out,
                              cudaStream_t s);

struct LinearArgs {
    const void *x;                     // codes
    int format;
    long long ldx;
    const float *s_x;
    int rows;
    const int32_t *offsets;            // [experts + 1], or null: one group of all rows
    int experts, n, k, kb;             // kb: 64-wide blocks of the reduction
    int n_tiles;                       // 128-channel tiles
    const uint8_t *w;
    const float *s_w, *bias;
    const int32_t *windows;
    void *y;
    long long ldy;
    int y_type;
    bool y_even;                       // 16-bit outputs: pairs of an even channel and the next lie on 4-byte boundaries
    int split;                         // CTAs of a cluster that share one tile's reduction
    int *err;
};
// few rows per group: integer dot products on the CUDA cores
cudaError_t launch_linear_few(const LinearArgs &a, int tokens, cudaStream_t s);
// the tensor-core kernel; tile: tokens per tile, pair: two CTAs per tile, loose: token codes as they lie (no tensor map);
// clusters (of a.split CTAs, or pairs) in the grid
cudaError_t launch_linear_tc(const CUtensorMap &tm, const LinearArgs &a, int tile, bool pair, bool loose, int clusters,
                             cudaStream_t s);

cudaError_t launch_combine_rows(const void *y, int type, long long ldy, long long rows, const int32_t *index,
                                const float *weights, long long tokens, int topk, int c, void *out, long long ldo,
                                int unit, int sms, cudaStream_t s);   // unit: bytes that all rows are aligned to, 16, 4 or 2

// A kernel of this file's operators may be started while the one before it in
// the stream is ending: it sets itself up and then waits here, before its first
// access to global memory, until everything before it in the stream is done and
// visible. From then on its own successor may be started the same way.
#ifdef __CUDACC__
// four fp16 codes as bytes: 1152 + code has code + 128 in its low byte
__device__ __forceinline__ uint32_t narrow_codes(uint32_t x, uint32_t y) {
    uint32_t a, b;
    asm("add.f16x2 %0, %1, %2;" : "=r"(a) : "r"(x), "r"(0x64806480u));
    asm("add.f16x2 %0, %1, %2;" : "=r"(b) : "r"(y), "r"(0x64806480u));
    return __byte_perm(a, b, 0x6420) ^ 0x80808080u;
}
__device__ __forceinline__ void after_prior_kernels() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
#endif
inline cudaLaunchAttribute early_start() {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    return attr;
}
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t s, Args... args) {
    cudaLaunchAttribute attr = early_start();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

// Lets `kernel` have `bytes` of dynamic shared memory: asked of CUDA where no call on this device has had as many, not
// per launch. `allowed` is the caller's static array. A call sets the limit, to less than it was if so asked, so host
// threads ask one at a time and look again when it is their turn. (A flag, held for one driver call: a mutex may throw.)
inline cudaError_t allow_shared(const void *kernel, int bytes, std::atomic<int> (&allowed)[64]) {
    if (bytes <= 40 * 1024) return cudaSuccess;                          // what every launch may have (48 KB), less static arrays
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (allowed[dev].load(std::memory_order_acquire) >= bytes) return cudaSuccess;
    static std::atomic_flag busy = ATOMIC_FLAG_INIT;
    while (busy.test_and_set(std::memory_order_acquire)) std::this_thread::yield();
    if (allowed[dev].load(std::memory_order_relaxed) < bytes) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) allowed[dev].store(bytes, std::memory_order_release);
    }
    busy.clear(std::memory_order_release);
    return e;
}

// host services of hatq_api.cu
int *device_error_word();
CUresult encode_tiled_2d(CUtensorMap *tm, CUtensorMapDataType type, const void *base, unsigned long long inner,
                         unsigned long long outer, unsigned long long pitch_bytes, unsigned box_inner,
                         unsigned box_outer);

}  // namespace hatq
