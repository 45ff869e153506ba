// Host side of the products with 4-bit weights: argument checks.
#include <climits>

#include "hatq_host.h"
#include "hatq_linear4.h"

namespace {

constexpr int kMaxDepth4 = 1 << 20, kMaxChannels4 = 1 << 27;

hatq_status check_weights(const hatq_linear4_weights *L) {
    if (!L) return fail(HATQ_ERR_INVALID_ARG, "null weights");
    if (L->n < 1 || L->k < 1) return fail(HATQ_ERR_INVALID_ARG, "n and k must be positive");
    if (L->k > kMaxDepth4) return fail(HATQ_ERR_UNSUPPORTED, "k must be at most %d", kMaxDepth4);
    if (L->n > kMaxChannels4) return fail(HATQ_ERR_UNSUPPORTED, "n must be at most %d", kMaxChannels4);
    if (L->group < 32 || L->group % 32) return fail(HATQ_ERR_INVALID_ARG, "a group is a multiple of 32 inputs, not %d", L->group);
    return HATQ_OK;
}
hatq_status check_buffers(const hatq_linear4_weights *L) {
    if (!L->data) return fail(HATQ_ERR_INVALID_ARG, "null weights");
    if (!aligned(L->data, 16) || !aligned(L->bias, 4))
        return fail(HATQ_ERR_INVALID_ARG, "weights must be 16-byte aligned, the bias to its elements");
    return HATQ_OK;
}
long long groups_of(const hatq_linear4_weights *L) { return ((long long)L->k + L->group - 1) / L->group; }

}  // namespace

extern "C" {

hatq_status hatq_linear4_sizes(int n, int k, int group, size_t *bytes) {
    hatq_linear4_weights L{};
    L.n = n;
    L.k = k;
    L.group = group;
    const hatq_status st = check_weights(&L);
    if (st != HATQ_OK) return st;
    if (!bytes) return fail(HATQ_ERR_INVALID_ARG, "null output");
    hatq::Linear4Args a{};
    hatq::linear4_units(n, k, group, a);
    *bytes = (size_t)a.strips * (size_t)a.units * (size_t)a.unit_bytes;
    return HATQ_OK;
}

hatq_status hatq_quantize_groups(const void *w, int type, long long ldw, int n, int k, int hb, int group, int8_t *codes,
                                 long long ldc, float *scales, long long lds, hatq_stream stream) {
    if (!is_type(type)) return fail(HATQ_ERR_INVALID_ARG, "unknown type %d", type);
    if (n < 0 || k < 1) return fail(HATQ_ERR_INVALID_ARG, "negative or empty shape");
    if (n > kMaxChannels4) return fail(HATQ_ERR_UNSUPPORTED, "at most %d rows", kMaxChannels4);
    if (k > hatq::kMaxTokenWidth) return fail(HATQ_ERR_UNSUPPORTED, "at most %d values per row", hatq::kMaxTokenWidth);
    if (hb < 1 || hb > 256 || (hb & (hb - 1)) || k % hb)
        return fail(HATQ_ERR_INVALID_ARG, "hb must be a power of two <= 256 that divides k");
    if (group < 32 || group % 32) return fail(HATQ_ERR_INVALID_ARG, "a group is a multiple of 32 inputs, not %d", group);
    const long long groups = ((long long)k + group - 1) / group;
    if (ldw < k || ldc < k || lds < groups) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldw > kMaxPitch || ldc > kMaxPitch || lds > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (n == 0) return HATQ_OK;
    if (!w || !codes || !scales) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    if (!aligned(w, type_size(type)) || !aligned(scales, 4)) return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (overlap(w, n, ldw, k, type_size(type), codes, n, ldc, k, 1) || overlap(w, n, ldw, k, type_size(type), scales, n, lds, groups, 4) ||
        overlap(codes, n, ldc, k, 1, scales, n, lds, groups, 4))
        return fail(HATQ_ERR_INVALID_ARG, "w, codes and scales overlap");
    const cudaError_t e = hatq::launch_quantize_groups(w, type, ldw, n, k, hb, group, codes, ldc, scales, lds,
                                                       reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "weight quantization launch");
}

hatq_status hatq_linear4_layout(const int8_t *w, long long ldw, const float *scales, long long lds, const hatq_linear4_weights *L,
                                hatq_stream stream) {
    hatq_status st = check_weights(L);
    if (st != HATQ_OK || (st = check_buffers(L)) != HATQ_OK) return st;
    if (ldw < L->k || lds < groups_of(L)) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldw > kMaxPitch || lds > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (!w || !scales) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    if (!aligned(scales, 4)) return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    hatq::Linear4Args a{};
    hatq::linear4_units(L->n, L->k, L->group, a);
    const cudaError_t e = hatq::launch_linear4_layout(w, ldw, scales, lds, a, L->data, reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "weight layout launch");
}

hatq_status hatq_linear4(const void *x, int x_type, long long ldx, const float *s_x, long long rows, const hatq_linear4_weights *L,
                         int y_type, void *y, long long ldy, hatq_stream stream) {
    hatq_status st = check_weights(L);
    if (st != HATQ_OK) return st;
    if (!is_type(x_type) || !is_type(y_type)) return fail(HATQ_ERR_INVALID_ARG, "unknown type %d", is_type(x_type) ? y_type : x_type);
    if (rows < 0) return fail(HATQ_ERR_INVALID_ARG, "negative row count");
    if (rows > (1 << 20)) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^20 rows per call");
    if (ldx < L->k || ldy < L->n) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldx > kMaxPitch || ldy > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (rows == 0) return HATQ_OK;
    if (!x || !y) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    if ((st = check_buffers(L)) != HATQ_OK) return st;
    if (!aligned(x, type_size(x_type)) || !aligned(y, type_size(y_type)) || !aligned(s_x, 4))
        return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (overlap(x, rows, ldx, L->k, type_size(x_type), y, rows, ldy, L->n, type_size(y_type)))
        return fail(HATQ_ERR_INVALID_ARG, "x and y overlap");
    const int sms = sm_count();
    hatq::Linear4Args a{};
    a.err = hatq::device_error_word();
    if (!sms || !a.err) return fail(HATQ_ERR_CUDA, "no CUDA device");
    a.x = x;
    a.ldx = ldx;
    a.vec = aligned(x, 16) && ldx * type_size(x_type) % 16 == 0;
    a.s_x = s_x;
    a.rows = (int)rows;
    hatq::linear4_units(L->n, L->k, L->group, a);
    a.w = L->data;
    a.bias = L->bias;
    a.y = y;
    a.ldy = ldy;
    a.y_type = y_type;
    const cudaError_t e = hatq::launch_linear4(a, x_type, sms, reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "product launch");
}

}  // extern "C"
