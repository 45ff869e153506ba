// Internal interface of the products with 4-bit weights between the host side
// (hatq_linear4_api.cu) and the kernels. Not part of the public ABI.
#pragma once

#include "hatq_tokens.h"

namespace hatq {

constexpr int kStrip = 16;             // channels of a strip of the layout
constexpr int kStep = 64;              // inputs of a block of it: 16 x 64 codes are 512 bytes, 16 a lane

struct Linear4Args {
    const void *x;
    long long ldx;
    bool vec;                          // rows of x lie on 16-byte boundaries
    const float *s_x;                  // or null
    int rows, n, k, group;
    const uint8_t *w;                  // [strip][unit]
    int strips, units;                 // units of a strip
    int unit_blocks, unit_scales;      // 2 blocks, 1 scale a channel; or 1 block, 1 or 2
    int unit_bytes, stage_units;       // stage_units: of a piece of a few-row ring
    const float *bias;
    void *y;
    long long ldy;
    int y_type;
    int *err;
};
// what follows from n, k and group
inline void linear4_units(int n, int k, int group, Linear4Args &a) {
    a.n = n;
    a.k = k;
    a.group = group;
    a.unit_blocks = group % (2 * kStep) == 0 ? 2 : 1;
    a.unit_scales = group % kStep == 0 ? 1 : 2;
    a.unit_bytes = 512 * a.unit_blocks + 4 * kStrip * a.unit_scales;
    a.stage_units = 4 / a.unit_blocks;
    a.strips = (int)(((long long)n + kStrip - 1) / kStrip);
    a.units = (k + kStep * a.unit_blocks - 1) / (kStep * a.unit_blocks);
}
cudaError_t launch_linear4(const Linear4Args &a, int x_type, int sms, cudaStream_t s);
cudaError_t launch_linear4_layout(const int8_t *w, long long ldw, const float *scales, long long lds, const Linear4Args &a, uint8_t *out,
                                  cudaStream_t s);
cudaError_t launch_quantize_groups(const void *w, int type, long long ldw, int n, int k, int hb, int group, int8_t *codes,
                                   long long ldc, float *scales, long long lds, cudaStream_t s);

}  // namespace hatq
