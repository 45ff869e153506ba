// Host side of the token operators: argument checks and the choice of kernel.
#include <climits>
#include <cmath>

#include "hatq_host.h"
#include "hatq_tokens.h"

namespace {

using hatq::LinearArgs;

constexpr int kMaxChannels = INT_MAX - 1023;    // the last tiles of 128 (of 256 on a pair) still count in int
constexpr int kMaxCombined = INT_MAX - 4095;    // and so does a row's end in whole steps of a CTA

struct Plan {
    bool few;        // the dot-product kernel
    int tokens;      // rows per pass of it, or per tile of the tensor-core kernel
    bool pair;       // two CTAs per tile
    int split;       // CTAs that share a tile's reduction
    bool pack;       // codes are packed as TMA takes them first
    long long tiles;
};

// How the tensor cores may take x: as it lies (fp16 at a pitch and a base that TMA takes), by the widening warps
// (anything else), or that or packed into a workspace first.
enum Operand { kDirect, kLoose, kEither };

// Rows per pass of the dot-product kernel (hatq_tokens.cu), or 0 for the tensor-core kernel (hatq_linear.cu). The
// former has no pipeline to fill, but its instructions are slow and every CTA brings in all rows. Measured, against the
// latter: 4096 x 4096 with 1 / 4 / 8 rows 3.5 / 5.4 / 10.9 us against 8.1 .. 9.1; 4096 x 16384 with 2 / 4 rows 15 / 21
// against 18.5; 16384 x 4096 with 1 / 2 rows 14 / 23 against 16.6; experts of 2048 x 1536 with a row each, 8 / 16 / 24
// of them, 5.6 / 12 / 15 against 12 / 19 / 19. Of grouped products only such small experts were measured: the kernel
// reads the weights once per row, so that with few and large experts the tensor-core kernel may be the faster one.
int few_rows(long long rows, const hatq_linear_weights *L, bool grouped) {
    const int few = grouped ? 1 : rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8;
    const long long weights = (long long)L->n * L->k;
    const bool take = grouped ? rows <= 24 : rows <= 2 || (rows <= 4 && weights <= 28'000'000) || (rows <= 8 && weights <= 13'000'000);
    return take && few * round_up(L->k, 64) <= 24 * 1024 ? few : 0;
}

// Which kernel and which tile. Of the tensor-core kernel's tiles the one with the least estimated time: waves
// of tiles x blocks of the reduction x time per block, the last measured with every SM at work (a wider tile costs
// more per block and less per product), and about 0.8 us to join a split reduction. Codes that TMA cannot take are
// brought in by the widening warps, with single-CTA tiles only (48 rows, 4096 -> 8192: 16.8 us against 11.8; 512 rows,
// 4096 -> 4096: 36 against 16.9), or packed first: a launch of about 3 us and 3 bytes a code.
Plan plan_of(long long rows, const hatq_linear_weights *L, bool grouped, int sms, Operand operand) {
    Plan p{};
    const int k_pad = round_up(L->k, 64), kb = k_pad / 64, n_tiles = (L->n + hatq::kRowTile - 1) / hatq::kRowTile;
    p.split = 1;
    p.tokens = few_rows(rows, L, grouped);
    p.few = p.tokens > 0;
    if (p.few) return p;
    static const struct { int tokens; bool pair; int ns; } options[] = {
        {32, false, 115}, {64, false, 140}, {128, false, 202}, {128, true, 165}, {192, true, 224}};
    const long long held = rows < L->experts ? rows : L->experts;
    long long best = LLONG_MAX;
    for (const auto &o : options) {
        const int ctas = o.pair ? 2 : 1, room = sms / ctas;
        if (o.pair && operand == kLoose) continue;
        // experts leave half a tile over each, and one tile at least
        const long long full = (rows + o.tokens - 1) / o.tokens, ragged = rows / o.tokens + held / 2;
        const long long tiles = (!grouped ? full : ragged > held ? ragged : held) * ((n_tiles + ctas - 1) / ctas);
        // clusters of four leave a few SMs of each group of SMs idle, clusters of eight too many
        for (int split = 1; split <= (o.pair ? 1 : 4); split *= 2) {
            if (split > 1 && (tiles * split > (split == 4 ? room * 15 / 16 : room) || kb / split < 4)) break;
            const long long ns = (tiles * split + room - 1) / room * ((kb + split - 1) / split) * o.ns + (split > 1 ? 800 : 0);
            const long long loose = o.pair ? LLONG_MAX : ns * 185 / 100;
            const long long packed = operand == kLoose ? LLONG_MAX : ns + 3000 + rows * k_pad * 3 / 5000;
            const long long cost = operand == kDirect ? ns : loose < packed ? loose : packed;
            if (cost < best) {
                best = cost;
                p.pack = operand == kEither && packed <= loose;
                p.tokens = o.tokens;
                p.pair = o.pair;
                p.split = split;
                // what the grid has to hold: every tile there may be, where a cluster takes only one
                p.tiles = (full + (grouped ? held : 0)) * ((n_tiles + ctas - 1) / ctas);
            }
        }
    }
    return p;
}

hatq_status check_weights(const hatq_linear_weights *L) {
    if (!L) return fail(HATQ_ERR_INVALID_ARG, "null weights");
    if (L->experts < 1 || L->experts > hatq::kMaxExperts)
        return fail(HATQ_ERR_INVALID_ARG, "experts must be in 1..%d", hatq::kMaxExperts);
    if (L->n < 1 || L->k < 1) return fail(HATQ_ERR_INVALID_ARG, "n and k must be positive");
    if (L->k > hatq::kMaxDepth) return fail(HATQ_ERR_UNSUPPORTED, "k must be at most %d", hatq::kMaxDepth);
    if (L->n > kMaxChannels || (long long)L->experts * ((L->n + 127LL) / 128) > (1LL << 30))
        return fail(HATQ_ERR_UNSUPPORTED, "too many output channels");
    return HATQ_OK;
}

// where x can go to the tensor cores as it lies: fp16 at a pitch and a base that TMA takes
bool direct(const void *x, int format, long long ldx) {
    return format == HATQ_CODES_F16 && ldx % 8 == 0 && aligned(x, 16);
}

Plan plan_for(const void *x, int format, long long ldx, long long rows, const hatq_linear_weights *L, bool grouped,
              size_t workspace_bytes, int sms) {
    const bool room_to_pack = workspace_bytes >= (size_t)rows * (size_t)round_up(L->k, 64) * 2;
    return plan_of(rows, L, grouped, sms, direct(x, format, ldx) ? kDirect : room_to_pack ? kEither : kLoose);
}

// what packing takes; it is used where it pays
size_t workspace_of(const void *x, int format, long long ldx, long long rows, const hatq_linear_weights *L, bool grouped) {
    if (rows == 0 || direct(x, format, ldx) || few_rows(rows, L, grouped) > 0) return 0;
    return (size_t)rows * (size_t)round_up(L->k, 64) * 2;
}

hatq_status product(const void *x, int format, long long ldx, const float *s_x, long long rows, const int32_t *offsets,
                    bool grouped, const hatq_linear_weights *L, int y_type, void *y, long long ldy, void *workspace,
                    size_t workspace_bytes, hatq_stream stream) {
    const hatq_status st = check_weights(L);
    if (st != HATQ_OK) return st;
    if (!is_codes(format)) return fail(HATQ_ERR_INVALID_ARG, "unknown code format %d", format);
    if (!is_type(y_type)) return fail(HATQ_ERR_INVALID_ARG, "unknown output type %d", y_type);
    if (rows < 0) return fail(HATQ_ERR_INVALID_ARG, "negative row count");
    if (rows > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows per call");
    if (ldx < L->k || ldy < L->n) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldx > kMaxPitch || ldy > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (!grouped && L->experts != 1) return fail(HATQ_ERR_INVALID_ARG, "a layer with experts needs hatq_grouped_linear");
    if (rows == 0) return HATQ_OK;
    if (!x || !s_x || !y || !L->codes || !L->windows || !L->s_w || (grouped && !offsets))
        return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    if (!aligned(L->codes, 16)) return fail(HATQ_ERR_INVALID_ARG, "the weight codes must be 16-byte aligned");
    if (!aligned(x, codes_size(format)) || !aligned(y, type_size(y_type)) || !aligned(s_x, 4) || !aligned(L->s_w, 4) ||
        !aligned(L->bias, 4) || !aligned(L->windows, 4) || !aligned(offsets, 4))
        return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (overlap(x, rows, ldx, L->k, codes_size(format), y, rows, ldy, L->n, type_size(y_type)))
        return fail(HATQ_ERR_INVALID_ARG, "x and y overlap");
    const int sms = sm_count();
    LinearArgs a{};
    a.err = hatq::device_error_word();
    if (!sms || !a.err) return fail(HATQ_ERR_CUDA, "no CUDA device");
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    a.x = x;
    a.format = format;
    a.ldx = ldx;
    a.s_x = s_x;
    a.rows = (int)rows;
    a.offsets = offsets;
    a.experts = L->experts;
    a.n = L->n;
    a.k = L->k;
    a.kb = (L->k + 63) / 64;
    a.n_tiles = (L->n + hatq::kRowTile - 1) / hatq::kRowTile;
    a.w = L->codes;
    a.s_w = L->s_w;
    a.bias = L->bias;
    a.windows = L->windows;
    a.y = y;
    a.ldy = ldy;
    a.y_type = y_type;
    a.y_even = ldy % 2 == 0 && aligned(y, 4);
    a.split = 1;
    if (workspace && !aligned(workspace, 16)) return fail(HATQ_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const Plan p = plan_for(x, format, ldx, rows, L, grouped, workspace ? workspace_bytes : 0, sms);
    cudaError_t e;
    if (p.few) {
        if ((e = hatq::launch_linear_few(a, p.tokens, s)) != cudaSuccess) return cuda_fail(e, "product launch");
        return HATQ_OK;
    }
    if (p.pack) {
        if ((e = hatq::launch_pack_codes(x, format, ldx, rows, L->k, a.kb * 64, workspace, s)) != cudaSuccess)
            return cuda_fail(e, "code packing launch");
        a.x = workspace;
        a.ldx = a.kb * 64;
        a.format = HATQ_CODES_F16;
    }
    const bool loose = !direct(x, format, ldx) && !p.pack;
    const int ctas = p.pair ? 2 : 1;
    if (p.tiles > INT_MAX / 16) return fail(HATQ_ERR_UNSUPPORTED, "too many output tiles");
    a.split = p.split;
    CUtensorMap tm{};
    if (!loose) {
        const CUresult r = hatq::encode_tiled_2d(&tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a.x, (unsigned long long)a.k,
                                                 (unsigned long long)rows, (unsigned long long)a.ldx * 2, 64,
                                                 (unsigned)(p.tokens / ctas));
        if (r != CUDA_SUCCESS) return fail(HATQ_ERR_CUDA, "code tensor map encoding failed (%d)", (int)r);
    }
    const int room = sms / ctas;
    const int clusters = a.split > 1 ? (int)p.tiles : (int)(p.tiles < room ? p.tiles : room);
    if ((e = hatq::launch_linear_tc(tm, a, p.tokens, p.pair, loose, clusters, s)) != cudaSuccess)
        return cuda_fail(e, "product launch");
    return HATQ_OK;
}

}  // namespace

extern "C" {

hatq_status hatq_quantize_tokens(const void *x, int x_type, long long ldx, long long src_rows, const int32_t *index,
                                 long long rows, int c, int hb, int act, int gated, int format, void *codes,
                                 long long ldc, float *scales, hatq_stream stream) {
    if (!is_type(x_type)) return fail(HATQ_ERR_INVALID_ARG, "unknown input type %d", x_type);
    if (!is_codes(format)) return fail(HATQ_ERR_INVALID_ARG, "unknown code format %d", format);
    if (act < HATQ_ACT_NONE || act > HATQ_ACT_GELU) return fail(HATQ_ERR_INVALID_ARG, "unknown activation %d", act);
    if (gated != 0 && gated != 1) return fail(HATQ_ERR_INVALID_ARG, "gated is 0 or 1");
    if (rows < 0 || src_rows < 0 || c < 1) return fail(HATQ_ERR_INVALID_ARG, "negative or empty shape");
    if (c > hatq::kMaxTokenWidth) return fail(HATQ_ERR_UNSUPPORTED, "at most %d values per row", hatq::kMaxTokenWidth);
    if (rows > kMaxRows || src_rows > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows per call");
    if (hb < 1 || hb > 256 || (hb & (hb - 1)) || c % hb)
        return fail(HATQ_ERR_INVALID_ARG, "hb must be a power of two <= 256 that divides c");
    const long long width = (long long)c * (gated ? 2 : 1);
    if (ldx < width || ldc < c) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldx > kMaxPitch || ldc > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (!index && src_rows < rows) return fail(HATQ_ERR_INVALID_ARG, "fewer source rows than rows and no index");
    if (rows == 0) return HATQ_OK;
    if ((!x && src_rows > 0) || !codes || !scales) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    const size_t xs = type_size(x_type), cs = codes_size(format);
    if (!aligned(x, xs) || !aligned(codes, cs) || !aligned(scales, 4) || !aligned(index, 4))
        return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (overlap(x, src_rows, ldx, width, xs, codes, rows, ldc, c, cs))
        return fail(HATQ_ERR_INVALID_ARG, "x and codes overlap");
    hatq::TokenQuantArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.src_rows = src_rows;
    a.index = index;
    a.rows = rows;
    a.c = c;
    a.hb = hb;
    a.act = act;
    a.gated = gated;
    a.inv_norm = (float)(1.0 / std::sqrt((double)hb));
    a.codes = codes;
    a.ldc = ldc;
    a.scales = scales;
    a.sms = sm_count();
    if (!a.sms) return fail(HATQ_ERR_CUDA, "no CUDA device");
    a.vec = aligned(x, 16) && ldx * xs % 16 == 0 && (!gated || (size_t)c * xs % 16 == 0) && aligned(codes, 16) &&
                     ldc * cs % 16 == 0;
    const cudaError_t e = hatq::launch_quantize_tokens(a, x_type, format, reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "token quantization launch");
}

hatq_status hatq_linear_sizes(int experts, int n, int k, size_t *code_bytes) {
    hatq_linear_weights L{};
    L.experts = experts;
    L.n = n;
    L.k = k;
    const hatq_status st = check_weights(&L);
    if (st != HATQ_OK) return st;
    if (!code_bytes) return fail(HATQ_ERR_INVALID_ARG, "null output");
    *code_bytes = (size_t)experts * ((size_t)(n + 127) / 128 * 128) * (size_t)round_up(k, 64);
    return HATQ_OK;
}

hatq_status hatq_linear_layout(const int8_t *w, long long ldw, const hatq_linear_weights *L, hatq_stream stream) {
    const hatq_status st = check_weights(L);
    if (st != HATQ_OK) return st;
    if (ldw < L->k) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldw > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (!w || !L->codes || !L->windows) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    if (!aligned(L->codes, 16) || !aligned(L->windows, 4))
        return fail(HATQ_ERR_INVALID_ARG, "the weight codes must be 16-byte aligned");
    const cudaError_t e = hatq::launch_linear_layout(w, ldw, L->experts, L->n, L->k, L->codes, L->windows,
                                                     reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "weight layout launch");
}

hatq_status hatq_linear_workspace(const void *x, int format, long long ldx, long long rows,
                                  const hatq_linear_weights *L, size_t *bytes) {
    const hatq_status st = check_weights(L);
    if (st != HATQ_OK) return st;
    if (!bytes) return fail(HATQ_ERR_INVALID_ARG, "null output");
    if (!is_codes(format)) return fail(HATQ_ERR_INVALID_ARG, "unknown code format %d", format);
    if (rows < 0) return fail(HATQ_ERR_INVALID_ARG, "negative row count");
    // the larger of what the dense and the grouped product want
    const size_t dense = workspace_of(x, format, ldx, rows, L, false), grouped = workspace_of(x, format, ldx, rows, L, true);
    *bytes = dense > grouped ? dense : grouped;
    return HATQ_OK;
}

hatq_status hatq_linear_plan(const void *x, int format, long long ldx, long long rows, const hatq_linear_weights *L,
                             int grouped, size_t workspace_bytes, int plan[5]) {
    const hatq_status st = check_weights(L);
    if (st != HATQ_OK) return st;
    if (!plan) return fail(HATQ_ERR_INVALID_ARG, "null output");
    if (!is_codes(format)) return fail(HATQ_ERR_INVALID_ARG, "unknown code format %d", format);
    if (rows < 1) return fail(HATQ_ERR_INVALID_ARG, "no rows");
    if (rows > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows per call");
    const int sms = sm_count();
    if (!sms) return fail(HATQ_ERR_CUDA, "no CUDA device");
    const Plan p = plan_for(x, format, ldx, rows, L, grouped != 0, workspace_bytes, sms);
    plan[0] = p.few;
    plan[1] = p.tokens;
    plan[2] = p.pair ? 2 : 1;
    plan[3] = p.split;
    plan[4] = p.few || direct(x, format, ldx) ? 0 : p.pack ? 2 : 1;
    return HATQ_OK;
}

hatq_status hatq_linear(const void *x, int format, long long ldx, const float *s_x, long long rows,
                        const hatq_linear_weights *L, int y_type, void *y, long long ldy, void *workspace,
                        size_t workspace_bytes, hatq_stream stream) {
    return product(x, format, ldx, s_x, rows, nullptr, false, L, y_type, y, ldy, workspace, workspace_bytes, stream);
}

hatq_status hatq_grouped_linear(const void *x, int format, long long ldx, const float *s_x, long long rows,
                                const int32_t *offsets, const hatq_linear_weights *L, int y_type, void *y,
                                long long ldy, void *workspace, size_t workspace_bytes, hatq_stream stream) {
    return product(x, format, ldx, s_x, rows, offsets, true, L, y_type, y, ldy, workspace, workspace_bytes, stream);
}

hatq_status hatq_combine_rows(const void *y, int type, long long ldy, long long rows, const int32_t *index,
                              const float *weights, long long tokens, int topk, int c, void *out, long long ldo,
                              hatq_stream stream) {
    if (!is_type(type)) return fail(HATQ_ERR_INVALID_ARG, "unknown type %d", type);
    if (rows < 0 || tokens < 0 || c < 1) return fail(HATQ_ERR_INVALID_ARG, "negative or empty shape");
    if (topk < 1 || topk > 64) return fail(HATQ_ERR_INVALID_ARG, "topk must be in 1..64");
    if (rows > kMaxRows || tokens > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows per call");
    if (c > kMaxCombined) return fail(HATQ_ERR_UNSUPPORTED, "at most %d values per row", kMaxCombined);
    if (ldy < c || ldo < c) return fail(HATQ_ERR_INVALID_ARG, "a pitch is smaller than its row");
    if (ldy > kMaxPitch || ldo > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "a pitch is larger than 2^32 elements");
    if (tokens == 0) return HATQ_OK;
    if ((!y && rows > 0) || !index || !weights || !out) return fail(HATQ_ERR_INVALID_ARG, "null tensor");
    const size_t ts = type_size(type);
    if (!aligned(y, ts) || !aligned(out, ts) || !aligned(index, 4) || !aligned(weights, 4))
        return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    if (overlap(y, rows, ldy, c, ts, out, tokens, ldo, c, ts)) return fail(HATQ_ERR_INVALID_ARG, "y and out overlap");
    auto all = [&](size_t u) {
        return aligned(y, u) && aligned(out, u) && ldy * ts % u == 0 && ldo * ts % u == 0 && c * ts % u == 0;
    };
    const int unit = all(16) ? 16 : all(4) ? 4 : 2;
    const int sms = sm_count();
    if (!sms) return fail(HATQ_ERR_CUDA, "no CUDA device");
    const cudaError_t e = hatq::launch_combine_rows(y, type, ldy, rows, index, weights, tokens, topk, c, out, ldo, unit, sms,
                                                    reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "combine launch");
}

}  // extern "C"
