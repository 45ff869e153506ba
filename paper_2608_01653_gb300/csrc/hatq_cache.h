// Internal interface of the 4-bit cache (append_tokens, attend_tokens) between
// the host side (hatq_cache_api.cu) and the kernels. Not part of the public ABI.
#pragma once

#include <climits>

#include "hatq_tokens.h"

namespace hatq {

constexpr int kChunk = 64;             // keys that a warp of the attention works on at a time
constexpr int kMaxSequences = 65536;

// A cache and the sequences that lie in it. A page holds, per head, page * width / 2 bytes of key codes, as many of
// value codes, page float32 key scales and page value scales: page * (width + 8) bytes in one piece.
struct CacheArgs {
    uint8_t *data;
    int pages, page_bits, heads, width, hb;
    float inv_norm;                    // 1 / sqrt(hb)
    const int32_t *table;
    long long ldt;
    int table_width, capacity;         // of a sequence, in pages and in tokens
    int seqs;
    const int32_t *lengths, *starts;
    int rows;
    bool small;                        // all (sequence, head, tile, chunk) are fewer than 2^31
};

struct AppendArgs {
    CacheArgs c;
    const void *x[2];                  // keys, values
    long long ldx[2], hx[2];           // pitch of rows and of heads
    void *kept[2];
    bool vec;                          // rows lie on 16-byte boundaries
};
cudaError_t launch_append(const AppendArgs &a, int type, cudaStream_t s);

struct AttendArgs {
    CacheArgs c;
    const void *q;
    long long ldq, hq;
    void *out;
    long long ldo, ho;
    int q_heads, group;                // group = q_heads / heads
    int columns;                       // of a tile
    bool vec;                          // rows of q lie on 16-byte boundaries
    float scale;                       // times log2(e): weights are powers of two
    long long *before;                 // [2 seqs + 2]: units and segments before every sequence; all units (parts only)
    float *pieces;
    long long segments;                // (sequence, head, tile): upper bound
    int direct;                        // see attend_direct
    bool prompt;
    bool vec_out;                      // rows of out lie on 16-byte boundaries
    int sms;
    int *err;
};
int attend_columns(int width, int group, long long rows, int seqs);
int attend_workers(int width, int sms);
// CTAs an SM where one takes a whole segment and writes its outputs, or 0: equal parts of all segments, which a second
// kernel joins
int attend_direct(int width, int columns, long long segments, int capacity, int sms);
cudaError_t launch_attend(const AttendArgs &a, int type, cudaStream_t s);

constexpr int kPromptColumns = 256;    // of a CTA of the kernel for many queries per sequence
bool attend_prompt(int type, int width, int heads, int group, long long rows, int seqs, int sms);
cudaError_t launch_prompt(const AttendArgs &a, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ int length_of(const CacheArgs &c, int b) {
    return min(max(c.lengths[b], 0), c.capacity);
}

// The sequence that row r belongs to, its first row and the row behind its last; false where no sequence holds r.
// Offsets that step back count as the largest before them. A whole warp calls this.
__device__ __forceinline__ bool sequence_of(const CacheArgs &c, int r, int lane, int &b, int &begin, int &end) {
    if (!c.starts) {
        b = begin = r;
        end = r + 1;
        return r < c.seqs;
    }
    // eight offsets a lane at a time, so that a call of thousands of sequences waits for memory less often
    unsigned first = 0xffffffffu;
    int most = 0;
    for (int j0 = 0; j0 <= c.seqs && first == 0xffffffffu; j0 += 256) {
        int v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = j0 + 32 * i + lane <= c.seqs ? c.starts[j0 + 32 * i + lane] : INT_MIN;
#pragma unroll
        for (int i = 7; i >= 0; --i)
            if (v[i] > r) first = (unsigned)(j0 + 32 * i + lane);
        first = __reduce_min_sync(0xffffffffu, first);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((unsigned)(j0 + 32 * i + lane) < first) most = max(most, v[i]);
    }
    if (first == 0xffffffffu || first == 0) return false;
    b = (int)first - 1;
    end = min(c.starts[first], c.rows);
    begin = __reduce_max_sync(0xffffffffu, most);
    return true;
}
#endif

}  // namespace hatq
