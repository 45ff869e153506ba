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
    int rows, n, k, group, groups;
    const uint8_t *w;
    const float *scales, *bias;
    void *y;
    long long ldy;
    int y_type;
};
cudaError_t launch_linear4(const Linear4Args &a, int x_type, int sms, cudaStream_t s);
cudaError_t launch_linear4_layout(const int8_t *w, long long ldw, const float *scales, long long lds, int n, int k, int groups,
                                  uint8_t *codes, float *out_scales, cudaStream_t s);
cudaError_t launch_quantize_groups(const void *w, int type, long long ldw, int n, int k, int hb, int group, int8_t *codes,
                                   long long ldc, float *scales, long long lds, cudaStream_t s);

}  // namespace hatq
