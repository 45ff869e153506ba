// Host side of the 4-bit cache: argument checks of append_tokens and attend_tokens.
#include <climits>
#include <cmath>

#include "hatq_host.h"
#include "hatq_cache.h"

namespace {

constexpr int kMaxHeads = 1024;
constexpr long long kMaxTokens = 1LL << 30;      // of a sequence, as its row of the table counts them

hatq_status check_cache(const hatq_token_cache *c) {
    if (!c) return fail(HATQ_ERR_INVALID_ARG, "null cache");
    if (c->width != 64 && c->width != 128 && c->width != 192 && c->width != 256)
        return fail(HATQ_ERR_UNSUPPORTED, "the heads of a cache are 64, 128, 192 or 256 wide, not %d", c->width);
    if (c->page != 16 && c->page != 32 && c->page != 64)
        return fail(HATQ_ERR_UNSUPPORTED, "a page holds 16, 32 or 64 tokens, not %d", c->page);
    if (c->heads < 1 || c->heads > kMaxHeads) return fail(HATQ_ERR_INVALID_ARG, "heads must be in 1..%d", kMaxHeads);
    if (c->pages < 0) return fail(HATQ_ERR_INVALID_ARG, "negative page count");
    if (c->hb < 1 || c->hb > 256 || (c->hb & (c->hb - 1)) || c->width % c->hb)
        return fail(HATQ_ERR_INVALID_ARG, "hb must be a power of two <= 256 that divides the width");
    if (c->pages > 0 && !c->data) return fail(HATQ_ERR_INVALID_ARG, "null cache data");
    if (!aligned(c->data, 16)) return fail(HATQ_ERR_INVALID_ARG, "the cache must be 16-byte aligned");
    return HATQ_OK;
}

// the sizes of a call's sequences, into what the kernels take
hatq_status check_sizes(const hatq_token_cache *c, long long rows, int table_width, int seqs, bool starts, hatq::CacheArgs &a) {
    if (seqs < 0 || rows < 0 || table_width < 0) return fail(HATQ_ERR_INVALID_ARG, "negative count");
    if (seqs > hatq::kMaxSequences) return fail(HATQ_ERR_UNSUPPORTED, "at most %d sequences per call", hatq::kMaxSequences);
    if (rows > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows per call");
    if (!starts && rows != seqs) return fail(HATQ_ERR_INVALID_ARG, "without starts, every sequence has one row");
    if ((long long)table_width * c->page > kMaxTokens) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^30 tokens per sequence");
    a.data = c->data;
    a.pages = c->pages;
    a.page_bits = c->page == 16 ? 4 : c->page == 32 ? 5 : 6;
    a.heads = c->heads;
    a.width = c->width;
    a.hb = c->hb;
    a.inv_norm = (float)(1.0 / std::sqrt((double)c->hb));
    a.table_width = table_width;
    a.capacity = table_width * c->page;
    a.seqs = seqs;
    a.rows = (int)rows;
    return HATQ_OK;
}
hatq_status check_sequences(const int32_t *table, long long ldt, const int32_t *lengths, const int32_t *starts, hatq::CacheArgs &a) {
    if (ldt < 0 || ldt > kMaxPitch) return fail(HATQ_ERR_INVALID_ARG, "the table's pitch is out of range");
    if (!lengths || (!table && a.table_width > 0)) return fail(HATQ_ERR_INVALID_ARG, "null lengths or table");
    if (!aligned(table, 4) || !aligned(lengths, 4) || !aligned(starts, 4))
        return fail(HATQ_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    a.table = table;
    a.ldt = ldt;
    a.lengths = lengths;
    a.starts = starts;
    return HATQ_OK;
}

// [rows][heads][width] at a pitch of rows and one of heads
struct Heads {
    const void *p;
    long long rows, pitch, heads, head_pitch, width;
    size_t size;
};
hatq_status check_heads(const Heads &t, const char *name, bool written) {
    if (!t.p) return fail(HATQ_ERR_INVALID_ARG, "%s: null tensor", name);
    if (!aligned(t.p, t.size)) return fail(HATQ_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (t.pitch < 0 || t.head_pitch < 0) return fail(HATQ_ERR_INVALID_ARG, "%s: negative pitch", name);
    if (t.pitch > kMaxPitch || t.head_pitch > kMaxPitch) return fail(HATQ_ERR_UNSUPPORTED, "%s: a pitch is larger than 2^32 elements", name);
    if (!written) return HATQ_OK;
    // rows outside heads, or heads outside rows
    const long long head = (t.heads - 1) * t.head_pitch + t.width, row = (t.rows - 1) * t.pitch + t.width;
    const bool rows_out = (t.heads == 1 || t.head_pitch >= t.width) && (t.rows == 1 || t.pitch >= head);
    const bool heads_out = (t.rows == 1 || t.pitch >= t.width) && (t.heads == 1 || t.head_pitch >= row);
    return rows_out || heads_out ? HATQ_OK : fail(HATQ_ERR_INVALID_ARG, "%s: rows or heads overlap", name);
}
// Whether two tensors may share an element: columns of one buffer at the same pitch do not, otherwise what lies between
// the first and the last element counts.
bool overlap(const Heads &a, const Heads &b) {
    auto packed = [](const Heads &t) { return t.heads == 1 || t.head_pitch == t.width; };
    if (packed(a) && packed(b))
        return overlap(a.p, a.rows, a.pitch, a.heads * a.width, a.size, b.p, b.rows, b.pitch, b.heads * b.width, b.size);
    auto span = [](const Heads &t) { return (t.rows - 1) * t.pitch + (t.heads - 1) * t.head_pitch + t.width; };
    if (a.rows == 0 || b.rows == 0) return false;
    return overlap(a.p, 1, 0, span(a), a.size, b.p, 1, 0, span(b), b.size);
}
Heads whole(const hatq_token_cache *c) {
    return {c->data, c->pages, (long long)c->heads * c->page * (c->width + 8), 1, 0, (long long)c->heads * c->page * (c->width + 8), 1};
}

hatq_status attend_args(const hatq_token_cache *c, int type, int q_heads, long long rows, int table_width, int seqs, bool starts,
                        hatq::AttendArgs &a) {
    hatq_status st = check_cache(c);
    if (st != HATQ_OK || (st = check_sizes(c, rows, table_width, seqs, starts, a.c)) != HATQ_OK) return st;
    if (type != HATQ_F16 && type != HATQ_BF16) return fail(HATQ_ERR_INVALID_ARG, "queries are fp16 or bf16, not type %d", type);
    if (q_heads < 1 || q_heads % c->heads) return fail(HATQ_ERR_INVALID_ARG, "the query heads are no multiple of the cache's");
    if (q_heads > 16 * kMaxHeads) return fail(HATQ_ERR_UNSUPPORTED, "at most %d query heads", 16 * kMaxHeads);
    if (rows * q_heads > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows x heads per call");
    a.q_heads = q_heads;
    a.group = q_heads / c->heads;
    a.columns = hatq::attend_columns(c->width, a.group, rows, seqs);
    // tiles of columns: no more than whole tiles of all rows, and one cut tile a sequence
    a.segments = c->heads * (rows * a.group / a.columns + (seqs < rows ? seqs : rows));
    a.c.small = a.segments * ((a.c.capacity + hatq::kChunk - 1) / hatq::kChunk) < INT_MAX;
    return HATQ_OK;
}
size_t before_bytes(const hatq::AttendArgs &a) { return ((size_t)a.c.seqs + 1) * 16; }
// once a.sms is set
size_t attend_bytes(hatq::AttendArgs &a, int type) {
    a.prompt = hatq::attend_prompt(type, a.c.width, a.c.heads, a.group, a.c.rows, a.c.seqs, a.sms);
    // as many segments as there are if all sequences have as many rows
    const long long seqs = a.c.seqs < a.c.rows ? a.c.seqs : a.c.rows, columns = ((long long)a.c.rows * a.group + seqs - 1) / seqs;
    const long long segments = a.c.heads * seqs * ((columns + a.columns - 1) / a.columns);
    a.direct = hatq::attend_direct(a.c.width, a.columns, segments, a.c.capacity, a.sms);
    return a.prompt || a.direct ? 0 : before_bytes(a) + ((size_t)a.segments + (size_t)hatq::attend_workers(a.c.width, a.sms)) * a.columns * (a.c.width + 2) * 4;
}

}  // namespace

extern "C" {

hatq_status hatq_append_tokens(const hatq_token_cache *cache, const void *k, long long ldk, long long hk, const void *v,
                               long long ldv, long long hv, int type, long long rows, const int32_t *table,
                               long long ldt, int table_width, const int32_t *lengths, const int32_t *starts, int seqs,
                               void *kept_k, void *kept_v, hatq_stream stream) {
    hatq::AppendArgs a{};
    hatq_status st = check_cache(cache);
    if (st != HATQ_OK || (st = check_sizes(cache, rows, table_width, seqs, starts != nullptr, a.c)) != HATQ_OK) return st;
    if (!is_type(type)) return fail(HATQ_ERR_INVALID_ARG, "unknown type %d", type);
    if (rows * cache->heads > kMaxRows) return fail(HATQ_ERR_UNSUPPORTED, "at most 2^31 - 1024 rows x heads per call");
    if (!kept_k != !kept_v) return fail(HATQ_ERR_INVALID_ARG, "kept keys without kept values, or values without keys");
    if (rows == 0 || seqs == 0) return HATQ_OK;
    if ((st = check_sequences(table, ldt, lengths, starts, a.c)) != HATQ_OK) return st;
    const size_t size = type_size(type);
    const long long heads = cache->heads, width = cache->width;
    const Heads in[2] = {{k, rows, ldk, heads, hk, width, size}, {v, rows, ldv, heads, hv, width, size}};
    const Heads kept[2] = {{kept_k, rows, heads * width, 1, 0, heads * width, size}, {kept_v, rows, heads * width, 1, 0, heads * width, size}};
    if ((st = check_heads(in[0], "k", false)) != HATQ_OK || (st = check_heads(in[1], "v", false)) != HATQ_OK) return st;
    for (int i = 0; i < 2; ++i) {
        if (overlap(in[i], whole(cache))) return fail(HATQ_ERR_INVALID_ARG, "the new tokens and the cache overlap");
        if (!kept_k) continue;
        if (!aligned(kept[i].p, 16)) return fail(HATQ_ERR_INVALID_ARG, "kept values must be 16-byte aligned");
        if (overlap(kept[i], in[0]) || overlap(kept[i], in[1]) || overlap(kept[i], whole(cache)))
            return fail(HATQ_ERR_INVALID_ARG, "kept values overlap the new tokens or the cache");
    }
    if (kept_k && overlap(kept[0], kept[1])) return fail(HATQ_ERR_INVALID_ARG, "kept keys and kept values overlap");
    for (int i = 0; i < 2; ++i) {
        a.x[i] = in[i].p;
        a.ldx[i] = in[i].pitch;
        a.hx[i] = in[i].head_pitch;
    }
    a.kept[0] = kept_k;
    a.kept[1] = kept_v;
    a.vec = aligned(k, 16) && aligned(v, 16) && ldk * size % 16 == 0 && ldv * size % 16 == 0 && hk * size % 16 == 0 && hv * size % 16 == 0;
    const cudaError_t e = hatq::launch_append(a, type, reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "append launch");
}

hatq_status hatq_attend_workspace(const hatq_token_cache *cache, int type, int q_heads, long long rows, int seqs, int starts,
                                  int table_width, size_t *bytes) {
    hatq::AttendArgs a{};
    if (!bytes) return fail(HATQ_ERR_INVALID_ARG, "null output");
    const hatq_status st = attend_args(cache, type, q_heads, rows, table_width, seqs, starts != 0, a);
    if (st != HATQ_OK) return st;
    *bytes = 0;
    if (rows == 0 || seqs == 0) return HATQ_OK;
    if (!(a.sms = sm_count())) return fail(HATQ_ERR_CUDA, "no CUDA device");
    *bytes = attend_bytes(a, type);
    return HATQ_OK;
}

hatq_status hatq_attend_tokens(const void *q, int type, long long ldq, long long hq, int q_heads, long long rows,
                               const hatq_token_cache *cache, const int32_t *table, long long ldt, int table_width,
                               const int32_t *lengths, const int32_t *starts, int seqs, float scale, void *out,
                               long long ldo, long long ho, void *workspace, size_t workspace_bytes, hatq_stream stream) {
    hatq::AttendArgs a{};
    hatq_status st = attend_args(cache, type, q_heads, rows, table_width, seqs, starts != nullptr, a);
    if (st != HATQ_OK) return st;
    a.scale = scale * 1.44269504088896340736f;
    if (!std::isfinite(a.scale)) return fail(HATQ_ERR_INVALID_ARG, "the scale, or scale * log2(e), is not finite");
    if (rows == 0 || seqs == 0) return HATQ_OK;
    if ((st = check_sequences(table, ldt, lengths, starts, a.c)) != HATQ_OK) return st;
    const Heads in{q, rows, ldq, q_heads, hq, cache->width, 2}, to{out, rows, ldo, q_heads, ho, cache->width, 2};
    if ((st = check_heads(in, "q", false)) != HATQ_OK || (st = check_heads(to, "out", true)) != HATQ_OK) return st;
    if (overlap(in, to)) return fail(HATQ_ERR_INVALID_ARG, "q and out overlap");
    if (overlap(to, whole(cache))) return fail(HATQ_ERR_INVALID_ARG, "out and the cache overlap");
    if (!(a.sms = sm_count())) return fail(HATQ_ERR_CUDA, "no CUDA device");
    const size_t bytes = attend_bytes(a, type);
    if (bytes && (!workspace || !aligned(workspace, 16))) return fail(HATQ_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    if (workspace_bytes < bytes) return fail(HATQ_ERR_INVALID_ARG, "the workspace is too small");
    a.err = hatq::device_error_word();
    if (!a.err) return fail(HATQ_ERR_CUDA, "no CUDA device");
    a.q = q;
    a.ldq = ldq;
    a.hq = hq;
    a.vec = aligned(q, 16) && ldq % 8 == 0 && hq % 8 == 0;
    a.out = out;
    a.ldo = ldo;
    a.ho = ho;
    a.vec_out = aligned(out, 16) && ldo % 8 == 0 && ho % 8 == 0;
    if (bytes) {
        a.before = static_cast<long long *>(workspace);
        a.pieces = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + before_bytes(a));
    }
    const cudaStream_t on = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = a.prompt ? hatq::launch_prompt(a, on) : hatq::launch_attend(a, type, on);
    return e == cudaSuccess ? HATQ_OK : cuda_fail(e, "attention launch");
}

}  // extern "C"
