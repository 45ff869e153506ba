// Attention over the 4-bit cache.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "hatq_cache.h"
#include "hatq_mma4.h"
#include "hatq_sequences.h"
#include "hatq_tc.h"

namespace hatq {
namespace {

using tc::mbar_init;
using tc::mbar_expect_tx;
using tc::smem_addr;

// For query column c of a kv head (token i and head h of the group: c = i * group + h) and keys j:
//   s_j = f_c k_j sum_d n_jd q_cd, p_j = 2^(s_j - m_c), o_cd = sum_j p_j v_j n'_jd / sum_j p_j
// with the codes n, n' and the scales k, v of the keys and values, q transformed as the keys were and f the constant
// factors (softmax scale, log2 e, the transform's norm). o is transformed back when the pieces are joined.
//
// Both products run as S^T = K Q^T and O^T = V^T P^T in m16n8k16 steps: codes are the A operand, so that 8 columns
// cost no more than one. For bf16 queries widening a code is a mask: a nibble x at bits 0-3 of a 16-bit half is the
// subnormal fp16 number x 2^-24, at bits 4-7 x 2^-20. The latter's factor of 16 goes into q (keys: the value is in the
// reduction) and into the result (values: it is a row). Codes are stored + 8; that is subtracted once per sum, 8 * 2^-24
// sum_d q_d as the accumulators' first value, 8 * 2^-24 sum_j p_j by one step with constant A. The scales of keys
// multiply s, those of values p: no code is ever multiplied by a scale.
//
// Rounded to fewer than 32 bits: q and p v, to fp16. q is brought into its range by a power of two per column, p v by the
// choice of m_c, so that what it keeps is relative to the largest term of the column's own sum: a token that the column does
// not see has no part in that, whatever its scale, nor has one whose codes are all 0 (append gives rows of zeros a scale like
// any other). For fp16 queries, whose outputs would show it, both go through in two parts, high and low,
// and codes are widened whole: the tensor cores align a subnormal's product as if it were a normal one's, and what they
// then drop left sums off by up to 2^-14 of their terms.
// m_c is raised only where some p v would exceed 2^15 (bf16: 2^12), to where it is just below 2^8. (What is dropped of
// subnormal products goes by the power of two of the largest p v: it is least there, and codes of 0, which are looked for
// where m_c may be raised alone, cost the others 2^-14 of at most 2^4 times the largest of them. 64 ragged sequences 73.3 us, with 2^15
// 72.7.) Sums are in fp32, and so is that of p, which
// may be large or small as the scales are: p stays below 2^103, so that scales of 2^-109 and more have all their bits, and
// those up to 2^110 leave room for weights of 2^-23 of the heaviest. Logits count from a base per column, 0 unless they are
// beyond 2^13, so that m_c has bits for all that whatever their size.
//
// Memory-bound for few queries. A warp works by itself: its own ring of chunks (64 keys of one head, brought in by one
// bulk copy per page), its own maxima and sums; no barrier between warps. The chunks of all sequences and heads are
// laid in a row and every warp takes an equal part of it, whatever the lengths; what a warp finds of a (sequence, head,
// column tile) goes to a piece in memory, and a second kernel joins the pieces. Where a CTA's whole part lies in one
// (sequence, head, tile) its warps are joined first; where such segments are short a CTA takes one each and no second
// kernel is needed. 12 warps (heads of 128) are what 227 KB of rings and 168 registers allow. Measured: one query behind
// 131072 keys, 32 heads over 8: 42 us (3.4 TB/s; 0.9 of the memory's rate once all warps are under way, 12 us to set out
// and to join); 64 ragged sequences up to 8192 keys 73 us (4.2 TB/s).

__host__ __device__ constexpr int kWarps(int d, int nt) { return d == 256 ? 6 : d == 192 || nt == 2 ? 8 : 12; }
__host__ __device__ constexpr int kStages(int d, int nt) { return (d == 64 ? 3 : 2) + (d <= 128 && nt == 2); }
__host__ __device__ constexpr int stage_bytes(int d) { return kChunk * (d + 8); }
__host__ __device__ constexpr int piece_floats(int d, int cols) { return cols * (d + 2); }
__host__ __device__ constexpr int warp_smem(int d, int nt) {   // ring, chunk descriptions, barriers; in whole 128 bytes, as bulk copies take 16
    return (kStages(d, nt) * (stage_bytes(d) + 32 + 8) + 127) / 128 * 128;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int N>
__device__ __forceinline__ void load_words(const uint8_t *at, uint32_t (&w)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at + 4 * i);
            w[i] = v.x;
            w[i + 1] = v.y;
            w[i + 2] = v.z;
            w[i + 3] = v.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(at + 4 * i);
            w[i] = v.x;
            w[i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const uint32_t *>(at + 4 * i);
    }
}
__device__ __forceinline__ float load_float(const uint8_t *at) { return *reinterpret_cast<const float *>(at); }
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float low_half(uint32_t x) { return __half2float(__ushort_as_half((unsigned short)(x & 0xffff))); }
__device__ __forceinline__ float high_half(uint32_t x) { return __half2float(__ushort_as_half((unsigned short)(x >> 16))); }

constexpr float kLowest = -3.402823466e38f;  // below every logit

// A logit from its column's base on: not fused with the product that it is, so that equal ones stay equal.
__device__ __forceinline__ float below(float s, float base) { return __fsub_rn(s, base); }

// A scale's logarithm. Those below 2^-88 count as that, so that weights stay below 2^103; an infinity has one of no NaN.
__device__ __forceinline__ float log2_of(float v) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fminf(fmaxf(v, 0x1p-88f), 0x1p127f)));
    return y;
}

// Sums of weights below a maximum that is raised: by 2^less, which may be below what fp32 holds when the sum itself is not.
// Returns 2^less (or 0), for sums of products.
__device__ __forceinline__ float lowered(float &l, float less) {
    const float half = exp2_fast(0.5f * less);
    l = l * half * half;
    return half * half;
}

// Equal parts for the warps: of `active` ones in every CTA, as few as give every CTA a unit.
struct Parts {
    int active;
    long long units;                   // of a worker
    __device__ Parts(long long total, int ctas, int warps) {
        const long long each = divide(total + ctas - 1, ctas);
        active = each < warps ? (int)max(each, 1LL) : warps;
        const long long workers = (long long)ctas * active;
        units = max(divide(total + workers - 1, workers), 1LL);
    }
};

// What a warp knows of a chunk between asking for it and working on it.
struct alignas(16) Chunk {
    int begin, m, len;                 // of its sequence
    int head, tile, chunk;
    int pages;                         // bit i: its page i holds keys
    int first_last;                    // of the warp's part of the segment: bit 0 first, bit 1 last
};
static_assert(sizeof(Chunk) == 32, "two 16-byte loads");

// A head's E values a lane (32 e + lane), transformed in place, unnormalized.
template <int E>
__device__ __forceinline__ void transform(float (&v)[E], int hb, int lane) {
#pragma unroll
    for (int h = 1; h < 32; h *= 2)
        if (h < hb)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float other = __shfl_xor_sync(0xffffffffu, v[e], h);
                v[e] = lane & h ? other - v[e] : v[e] + other;
            }
#pragma unroll
    for (int h = 1; h < E; h *= 2)
        if (32 * h < hb)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!(e & h) && e + h < E) {
                    const float x = v[e], y = v[e + h];
                    v[e] = x + y;
                    v[e + h] = x - y;
                }
}

// 8 columns of queries from column x0 on as B operands of the steps over keys: transformed, brought below 2^10 by a power
// of two per column, rounded to fp16 (part 0; part 1 is what that left). f: the factors of logits of columns 2 t and 2 t + 1.
//
// The transform is a product with a matrix of signs: exact operands, fp32 sums, all columns at once. Lane (g, t) reads the
// values 32 J + 8 t .. + 7 of column g as they lie; step s of J has + 4 s .. 4 s + 3. Result rows may come in any order,
// so that of tile (x, p) row r < 8 is value ((r / 2) WORDS + x) 8 + 2 p + 4 (r % 2) and row r + 8 the next one: transposed,
// rows 2 t and 2 t + 1 are the pair that lane t multiplies with the codes at bits 0-3 (r + 8: 4-7) of its word x. A sign is
// the parity of row & column & (hb - 1), zero where they are in different blocks; the two lowest bits of both make a
// pattern of 4 words, the others flip it or clear it.
template <int D, typename T, bool TWO>
struct Queries {
    static constexpr int WORDS = D / 32, PARTS = TWO ? 2 : 1;
    static constexpr uint32_t kOne = std::is_same<T, __half>::value ? 0x3c00u : 0x3f80u;
    static constexpr float kOdd = TWO ? 1.0f : 0.0625f, kUnit = TWO ? 1.0f : 0x1p24f;
    uint32_t b[WORDS][4], pattern[2][4];
    float by[2], f[2];

    __device__ __forceinline__ void load(const AttendArgs &a, int begin, int m, int kv_head, int x0, int lane) {
        const int g = lane >> 2, t = lane & 3, x = x0 + g, token = x / a.group, h = x - token * a.group;
        if (token < m) {
            const T *p = static_cast<const T *>(a.q) + (long long)(begin + token) * a.ldq + (long long)(kv_head * a.group + h) * a.hq + 8 * t;
            if (a.vec) {
#pragma unroll
                for (int j = 0; j < WORDS; ++j) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p + 32 * j));
                    b[j][0] = v.x;
                    b[j][1] = v.y;
                    b[j][2] = v.z;
                    b[j][3] = v.w;
                }
            } else {
                const unsigned short *u = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
                for (int j = 0; j < WORDS; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) b[j][i] = u[32 * j + 2 * i] | (uint32_t)u[32 * j + 2 * i + 1] << 16;
            }
        } else {                                             // zeros, which give logits of 0
#pragma unroll
            for (int j = 0; j < WORDS; ++j) b[j][0] = b[j][1] = b[j][2] = b[j][3] = 0;
        }
    }
    __device__ __forceinline__ void measure(const AttendArgs &a, int lane) {
        const int t = lane & 3;
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < WORDS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = __vmaxu2(most, b[j][i] & 0x7fff7fffu);
        most = max(most & 0xffffu, most >> 16);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        union { unsigned short u; T v; } m;
        m.u = (unsigned short)most;
        const uint32_t log_hb = 31 - __clz(a.c.hb), own = max(__float_as_uint(to_f32<T>(m.v)) >> 23, 10u);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            // a sum is below hb 2^(ex - 126); an infinity or a NaN makes the whole column NaN
            const uint32_t ex = __shfl_sync(0xffffffffu, own, 8 * t + 4 * y);
            by[y] = ex == 255u ? __int_as_float(0x7fffffff) : __uint_as_float((263u - log_hb - ex) << 23);
            f[y] = a.scale * a.c.inv_norm * kUnit * __uint_as_float((min(ex, 254u) + log_hb - 9u) << 23);
        }
        // patterns of the lowest bits: rows 2 p and 2 p + 1, columns 0, 1 and 2, 3
        const int low = (a.c.hb - 1) & 3;
        auto sign = [&](int row, int col) { return ((row ^ col) & 3 & ~low) ? 0u : kOne ^ (uint32_t)(__popc(row & col & low) & 1) << 15; };
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) pattern[p][i] = sign(2 * p + (i & 1), i & 2) | sign(2 * p + (i & 1), (i & 2) + 1) << 16;
    }
    // the operands of steps 2 w and 2 w + 1: q[part][p][2]
    __device__ __forceinline__ void tile(const AttendArgs &a, int w, int lane, uint32_t (&q)[PARTS][2][2]) const {
        const int g = lane >> 2, t = lane & 3, high = (a.c.hb - 1) >> 2, row = (g >> 1) * (2 * WORDS) + 2 * w + (g & 1);
        float c[2][4] = {};
#pragma unroll
        for (int j = 0; j < WORDS; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int col = 8 * j + 2 * t + s;
                const uint32_t keep = ((row ^ col) & ~high) ? 0u : 0xffffffffu, flip = (__popc(row & col & high) & 1) ? 0x80008000u : 0u;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    uint32_t A[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) A[i] = (pattern[p][i] ^ flip) & keep;
                    if constexpr (std::is_same<T, __half>::value)
                        mma(c[p], A, b[j][2 * s], b[j][2 * s + 1]);
                    else
                        mma_bf16(c[p], A, b[j][2 * s], b[j][2 * s + 1]);
                }
            }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int o = 0; o < 2; ++o) {                    // values at odd places meet codes of 16-fold value
                const float u = c[p][2 * o] * by[0] * (o ? kOdd : 1.0f), v = c[p][2 * o + 1] * by[1] * (o ? kOdd : 1.0f);
                const uint32_t r = pack_half(u, v);
                q[0][p][o] = transposed(r);
                if constexpr (TWO) q[1][p][o] = transposed(pack_half(u - low_half(r), v - high_half(r)));
            }
    }
};
// the accumulators' first values: 8 * 2^-24 of every value, as the codes' offset meets them
template <int STEPS>
__device__ __forceinline__ void offsets_of(const uint32_t (&qf)[STEPS][2], float (&off)[2]) {
    const uint32_t A[4] = {0x00080008u, 0x00080008u, 0x00800080u, 0x00800080u};
    float c[4] = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) mma(c, A, qf[s][0], qf[s][1]);
    off[0] = -c[0];
    off[1] = -c[1];
}

// Writes a head of a row: o / l (zeros where no key was seen) transformed back.
template <int D, typename T>
__device__ __forceinline__ void finish(const AttendArgs &a, int r, int head, int lane, float (&o)[D / 32], float l) {
    transform<D / 32>(o, a.c.hb, lane);
    const float by = l == 0.0f ? 0.0f : a.c.inv_norm / l;
    T *out = static_cast<T *>(a.out) + (long long)r * a.ldo + (long long)head * a.ho + lane;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) out[32 * e] = from_f32<T>(o[e] * by);
}

template <int D, typename T, int NT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, kWarps(D, NT) / WARPS) attend_kernel(const AttendArgs a) {
    constexpr int COLS = 8 * NT, STAGES = kStages(D, NT), STAGE = stage_bytes(D);
    constexpr int WORDS = D / 32, VW = D / 64, STEPS = D / 16, E = D / 32;
    constexpr bool kTwo = std::is_same<T, __half>::value;      // q and p in two parts
    constexpr int PARTS = kTwo ? 2 : 1;
    constexpr float kOdd = kTwo ? 1.0f : 0.0625f, kUnit = kTwo ? 1.0f : 0x1p24f;     // of a code at an odd place; of a sum
    constexpr float kMost = kTwo ? 15.0f : 12.0f;              // logarithm of what p v may be before m is raised
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int s_abort;
    const CacheArgs &c = a.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint8_t *mine = smem + warp * warp_smem(D, NT);
    Chunk *chunks = reinterpret_cast<Chunk *>(mine + STAGES * STAGE);
    const uint32_t ring = smem_addr(mine), bars = smem_addr(mine + STAGES * (STAGE + 32));
    volatile int *abort_flag = &s_abort;

    if (lane < STAGES) mbar_init(bars + 8 * lane, 1);
    tc::fence_barrier_init();
    if (threadIdx.x == 0) s_abort = 0;
    __syncthreads();
    after_prior_kernels();
    const int err = *reinterpret_cast<volatile int *>(a.err);

    // ---- this warp's part
    Row<COLS> row;
    row.read(c, a.group, lane, a.direct);
    const long long total = row.total;
    long long cta_from, cta_to, from, to, joined_place = 0;
    bool joined = true;                                      // the CTA's part lies in one segment:
    long long first_segment;                                 // this one of its sequence
    Sequence seq{};
    if (a.direct) {
        // a segment per CTA, all of it
        if (blockIdx.x >= total) return;
        row.find_unit(c, a.group, lane, blockIdx.x, seq);
        first_segment = blockIdx.x - seq.unit;
        const int each = (seq.chunks + WARPS - 1) / WARPS;
        seq.unit = -first_segment * seq.chunks;                    // units count from the segment's first
        cta_from = 0;
        cta_to = seq.chunks;
        from = min(warp * each, seq.chunks);
        to = min(from + each, cta_to);
    } else {
        // for the second kernel (by a warp of the last part, which may be a short one)
        if (blockIdx.x + 1 == gridDim.x && warp + 1 == WARPS) row.write(c, a.group, lane, a.before);
        const Parts parts(total, gridDim.x, WARPS);
        cta_from = min(blockIdx.x * (parts.active * parts.units), total);
        cta_to = min((blockIdx.x + 1LL) * (parts.active * parts.units), total);
        from = warp < parts.active ? min(cta_from + warp * parts.units, total) : cta_to;
        to = min(from + parts.units, cta_to);
        if (cta_from == cta_to) return;
        row.find_unit(c, a.group, lane, cta_from, seq);
        first_segment = divide(cta_from - seq.unit, seq.chunks);
        joined = cta_to <= seq.unit + (first_segment + 1) * seq.chunks;
        joined_place = cta_from == seq.unit + first_segment * seq.chunks ? seq.segment + first_segment : a.segments + blockIdx.x * (long long)WARPS;
    }
    const Sequence first = seq;
    if (__syncthreads_or(err != 0)) return;
    if (from < to && from >= seq.unit + seq.units(c.heads)) row.find_unit(c, a.group, lane, from, seq);
    const int size = 1 << c.page_bits, pages_of_chunk = kChunk >> c.page_bits;
    const uint32_t record = (uint32_t)size * (D + 8);

    // ---- asking for chunks
    long long unit = from;                                   // the next one to ask for
    int segment = 0, chunk = 0, asked = 0;                   // segment within the sequence
    if (from < to) {
        segment = (int)divide(from - seq.unit, seq.chunks);
        chunk = (int)(from - seq.unit - (long long)segment * seq.chunks);
    }
    int entry = -1, entries_from = -1;                       // 32 entries of the sequence's row of the table, one a lane
    auto ask = [&]() {
        if (unit >= to) return;
        const int stage = asked % STAGES;
        const int first_page = chunk * pages_of_chunk;
        if (entries_from < 0 || first_page < entries_from || first_page >= entries_from + 32) {
            entries_from = first_page;
            entry = first_page + lane < c.table_width ? c.table[seq.b * c.ldt + first_page + lane] : -1;
        }
        const int page = __shfl_sync(0xffffffffu, entry, (first_page - entries_from + lane) & 31);
        const int head = segment / seq.tiles;
        const bool take = lane < pages_of_chunk && chunk * kChunk + lane * size < seq.len && page >= 0 && page < c.pages;
        const unsigned pages = __ballot_sync(0xffffffffu, take);
        if (lane == 0) {
            Chunk k;
            k.begin = seq.begin;
            k.m = seq.m;
            k.len = seq.len;
            k.head = head;
            k.tile = segment - head * seq.tiles;
            k.chunk = chunk;
            k.pages = (int)pages;
            const bool first = unit == from || chunk == 0, last = unit + 1 == to || chunk + 1 == seq.chunks;
            k.first_last = (first ? 1 : 0) | (last ? 2 : 0);
            chunks[stage] = k;
            mbar_expect_tx(bars + 8 * stage, (uint32_t)__popc(pages) * record);
        }
        __syncwarp();
        if (take)
            bulk_load(ring + stage * STAGE + lane * record, c.data + ((long long)page * c.heads + head) * record, record, bars + 8 * stage);
        if (!joined && chunk == 0) {                         // a new segment: its queries on their way to L2
            const int x = (segment - head * seq.tiles) * COLS + lane, at = x / a.group;
            if (lane < COLS && at < seq.m) {
                const T *p = static_cast<const T *>(a.q) + (long long)(seq.begin + at) * a.ldq + (long long)(head * a.group + x - at * a.group) * a.hq;
#pragma unroll
                for (int e = 0; e < D; e += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + e));
            }
        }
        ++asked;
        ++unit;
        if (++chunk == seq.chunks) {
            chunk = 0;
            if (entries_from != 0) entries_from = -1;
            if (++segment == c.heads * seq.tiles && unit < to) {
                // the next sequence that has units
                Sequence next = seq;
                do {
                    const long long u = next.unit + next.units(c.heads), sg = next.segment + next.segments(c.heads);
                    const int end = next.begin + next.m, b = next.b + 1;
                    measure<COLS>(c, a.group, next, b, c.starts ? end : b, c.starts ? max(end, c.starts[b + 1]) : b + 1);
                    next.unit = u;
                    next.segment = sg;
                } while (next.units(c.heads) == 0 && next.b + 1 < c.seqs);
                seq = next;
                segment = 0;
                entries_from = -1;
            }
        }
    };
    // Where the pieces go: one that begins its segment has the segment's place, any other (a worker has at most one, its
    // first) the warp's.
    long long piece = 0;
    if (from < to)
        piece = from == seq.unit + (long long)segment * seq.chunks ? seq.segment + segment
                    : a.segments + blockIdx.x * (long long)WARPS + warp;
    long long next_piece = from < to ? seq.segment + segment + 1 : 0;
    // Where the CTA has one segment, its warps transform the queries together, a word of the codes each; the loads go out
    // before those of keys, which would hold them up.
    uint8_t *shared_q = smem + WARPS * warp_smem(D, NT);     // [tile of 8 columns][word][lane][part][2][2], then factors
    constexpr int kQ = PARTS * 16, SHARERS = NT * WORDS;
    Queries<D, T, kTwo> own;
    const int first_head = (int)divide(first_segment, first.tiles), first_x = ((int)first_segment - first_head * first.tiles) * COLS;
    if (joined && warp < SHARERS) own.load(a, first.begin, first.m, first_head, first_x + warp / WORDS * 8, lane);
    for (int i = 0; i < STAGES; ++i) ask();
    if (joined) {
        for (int x = warp; x < SHARERS; x += WARPS) {
            if (x != warp) own.load(a, first.begin, first.m, first_head, first_x + x / WORDS * 8, lane);
            own.measure(a, lane);
            uint32_t q[PARTS][2][2];
            own.tile(a, x % WORDS, lane, q);
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
                *reinterpret_cast<uint4 *>(shared_q + (x * 32 + lane) * kQ + 16 * part) = make_uint4(q[part][0][0], q[part][0][1], q[part][1][0], q[part][1][1]);
            if (x % WORDS == 0 && lane < 4)
                *reinterpret_cast<float2 *>(shared_q + SHARERS * 32 * kQ + 32 * (x / WORDS) + 8 * lane) = make_float2(own.f[0], own.f[1]);
        }
        __syncthreads();
    }

    float o[NT][STEPS][4], off[NT][4], base[NT][2], m[NT][2], l[NT][2];      // m from base on
    uint32_t qf[NT][PARTS][STEPS][2];
    float q_off[NT][2], q_f[NT][2];
    int lim[NT][2];
    bool sound = true;
    const int units = (int)(to - from);
    const int near = (g & 1) ? 7 - (g >> 1) : g >> 1;        // the key of the tile that row g of A is; row g + 8: + 8
    const uint32_t ones[4] = {0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u};       // 8 * 2^-24

    for (int i = 0; i < units; ++i) {
        const int stage = i % STAGES;
        sound = tc::mbar_wait(bars + 8 * stage, (uint32_t)(i / STAGES) & 1u, abort_flag, a.err);
        sound = __all_sync(0xffffffffu, sound);
        if (!sound) break;
        const Chunk k = chunks[stage];

        if (k.first_last & 1) {
            // ---- a new segment: its queries, 8 columns at a time
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (joined) {
#pragma unroll
                    for (int w = 0; w < WORDS; ++w)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) {
                            const uint4 q = *reinterpret_cast<const uint4 *>(shared_q + ((nt * WORDS + w) * 32 + lane) * kQ + 16 * part);
                            qf[nt][part][2 * w][0] = q.x;
                            qf[nt][part][2 * w][1] = q.y;
                            qf[nt][part][2 * w + 1][0] = q.z;
                            qf[nt][part][2 * w + 1][1] = q.w;
                        }
                    const float2 f = *reinterpret_cast<const float2 *>(shared_q + SHARERS * 32 * kQ + 32 * nt + 8 * t);
                    q_f[nt][0] = f.x;
                    q_f[nt][1] = f.y;
                } else {
                    Queries<D, T, kTwo> own;
                    own.load(a, k.begin, k.m, k.head, k.tile * COLS + nt * 8, lane);
                    own.measure(a, lane);
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) {
                        uint32_t q[PARTS][2][2];
                        own.tile(a, w, lane, q);
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                qf[nt][part][2 * w + p][0] = q[part][p][0];
                                qf[nt][part][2 * w + p][1] = q[part][p][1];
                            }
                    }
                    q_f[nt][0] = own.f[0];
                    q_f[nt][1] = own.f[1];
                }
                q_off[nt][0] = q_off[nt][1] = 0.0f;
                if constexpr (!kTwo) offsets_of<STEPS>(qf[nt][0], q_off[nt]);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int x = k.tile * COLS + nt * 8 + 2 * t + y, token = x / a.group;
                    lim[nt][y] = token < k.m ? k.len - k.m + token : -1;
                    base[nt][y] = 0.0f;
                    m[nt][y] = kLowest;
                    l[nt][y] = 0.0f;
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[nt][s][y] = 0.0f;
#pragma unroll
                for (int y = 0; y < 4; ++y) off[nt][y] = 0.0f;
            }
        }

        // ---- S^T of the chunk's 64 keys (what lies behind the last one is computed from whatever is there, and masked)
        const uint8_t *keys = mine + stage * STAGE;
        const int key0 = k.chunk * kChunk;
        const bool whole = key0 + kChunk <= k.len - k.m + k.tile * COLS / a.group + 1 && k.pages == (1 << pages_of_chunk) - 1;
        float s[NT][4][4], vs[4][2], ks[4][2], most[NT][2];
        const uint8_t *rec[4];
        int token[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            rec[j] = keys + ((16 * j) >> c.page_bits) * record;
            token[j] = (16 * j) & (size - 1);
            const uint8_t *sc = rec[j] + size * D + 4 * (token[j] + near);
            ks[j][0] = load_float(sc);
            ks[j][1] = load_float(sc + 32);
            vs[j][0] = load_float(sc + 4 * size);
            vs[j][1] = load_float(sc + 4 * size + 32);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint8_t *krow = rec[j] + (token[j] + near) * (D / 2);
            uint32_t w0[WORDS], w1[WORDS];
            load_words<WORDS>(krow + t * (WORDS * 4), w0);
            load_words<WORDS>(krow + 8 * (D / 2) + t * (WORDS * 4), w1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][j][0] = s[nt][j][2] = q_off[nt][0];
                s[nt][j][1] = s[nt][j][3] = q_off[nt][1];
            }
#pragma unroll
            for (int x = 0; x < WORDS; ++x) {
                const uint32_t u0 = w0[x] >> 8, u1 = w1[x] >> 8;
                const uint32_t A[4] = {codes_f16<kTwo, false>(w0[x]), codes_f16<kTwo, false>(w1[x]), codes_f16<kTwo, true>(w0[x]),
                                       codes_f16<kTwo, true>(w1[x])};
                const uint32_t B[4] = {codes_f16<kTwo, false>(u0), codes_f16<kTwo, false>(u1), codes_f16<kTwo, true>(u0),
                                       codes_f16<kTwo, true>(u1)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        mma(s[nt][j], A, qf[nt][part][2 * x][0], qf[nt][part][2 * x][1]);
                        mma(s[nt][j], B, qf[nt][part][2 * x + 1][0], qf[nt][part][2 * x + 1][1]);
                    }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][j][0] *= ks[j][0] * q_f[nt][0];
                s[nt][j][1] *= ks[j][0] * q_f[nt][1];
                s[nt][j][2] *= ks[j][1] * q_f[nt][0];
                s[nt][j][3] *= ks[j][1] * q_f[nt][1];
            }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = key0 + 16 * j + near;
                const bool held = (k.pages >> ((16 * j) >> c.page_bits)) & 1;
                const bool in0 = held && key < k.len, in1 = held && key + 8 < k.len;
                if (!in0) vs[j][0] = 0.0f;
                if (!in1) vs[j][1] = 0.0f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if (!in0 || key > lim[nt][y]) s[nt][j][y] = -INFINITY;
                        if (!in1 || key + 8 > lim[nt][y]) s[nt][j][2 + y] = -INFINITY;
                    }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                most[nt][y] = kLowest;
#pragma unroll
                for (int j = 0; j < 4; ++j) most[nt][y] = fmaxf(most[nt][y], fmaxf(s[nt][j][y], s[nt][j][2 + y]));
            }

        // how far a logit of these keys may exceed m
        float largest = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) largest = fmaxf(largest, fmaxf(vs[j][0], vs[j][1]));
        const float room = kMost - log2_of(largest);
        // ---- raise the maxima where a weight, or its product with a scale, may leave the range
        bool high = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) high |= most[nt][0] - base[nt][0] > m[nt][0] + room || most[nt][1] - base[nt][1] > m[nt][1] + room;
        if (__any_sync(0xffffffffu, high)) {
            // Tokens whose codes are all 0: nothing of them, whatever their scale. A lane has two, one after the other: every warp
            // comes here once, and code that runs once is waited for (131072 keys 42.6 us, both at once 43.7).
            unsigned none[2] = {0, 0};
#pragma unroll 1
            for (int i = 0; i < kChunk; i += 32) {
                const int at = i + lane;
                const uint4 *row = reinterpret_cast<const uint4 *>(keys + (at >> c.page_bits) * record + (size + (at & (size - 1))) * (D / 2));
                uint32_t z = 0;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {           // (from a piece on that leaves no two lanes the same banks)
                    const int piece = x + (lane >> (D == 128 ? 1 : D == 256 ? 0 : 2)) % (D / 32);
                    const uint4 w = row[piece < D / 32 ? piece : piece - D / 32];
                    z |= (w.x ^ 0x88888888u) | (w.y ^ 0x88888888u) | (w.z ^ 0x88888888u) | (w.w ^ 0x88888888u);
                }
                none[0] = none[1];
                none[1] = __ballot_sync(0xffffffffu, z == 0);
            }
            if (none[0] | none[1])
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if ((none[j >> 1] >> (16 * (j & 1) + 8 * h + near) & 1) && vs[j][h] < INFINITY) vs[j][h] = 0.0f;
            // the largest product of every column, by what it sees alone
            auto largest = [&](int nt, int y) {
                float u = kLowest;
#pragma unroll
                for (int j = 0; j < 4; ++j) u = fmaxf(u, fmaxf(below(s[nt][j][y], base[nt][y]) + log2_of(vs[j][0]), below(s[nt][j][2 + y], base[nt][y]) + log2_of(vs[j][1])));
#pragma unroll
                for (int h = 4; h < 32; h *= 2) u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, h));
                return u;
            };
            float x[NT][2];
            bool move = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    x[nt][y] = largest(nt, y);
                    move |= x[nt][y] > m[nt][y] + kMost && fabsf(x[nt][y]) > 8192.0f;
                }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const bool own = x[nt][y] > m[nt][y] + kMost && fabsf(x[nt][y]) > 8192.0f;
                        const float to = base[nt][y] + (own ? x[nt][y] : 0.0f), up = to - base[nt][y];
                        base[nt][y] = to;
                        m[nt][y] = fmaxf(m[nt][y] - up, kLowest);
                        x[nt][y] = largest(nt, y);
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float by[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float to = x[nt][y] > m[nt][y] + kMost ? x[nt][y] - 7.9f : m[nt][y];
                    by[y] = lowered(l[nt][y], m[nt][y] - to);
                    m[nt][y] = to;
                    off[nt][y] *= by[y];
                }
#pragma unroll
                for (int x = 0; x < STEPS; ++x) {
                    o[nt][x][0] *= by[0];
                    o[nt][x][1] *= by[1];
                    o[nt][x][2] *= by[0];
                    o[nt][x][3] *= by[1];
                }
            }
        }

        // ---- weights, and O^T
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t pf[PARTS][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) p[y] = exp2_fast(below(s[nt][j][y], base[nt][y & 1]) - m[nt][y & 1]);
                l[nt][0] += p[0] + p[2];
                l[nt][1] += p[1] + p[3];
                // (nothing of a value that this query does not see, whatever its scale)
#pragma unroll
                for (int y = 0; y < 4; ++y) p[y] = whole || p[y] != 0.0f ? p[y] * vs[j][y >> 1] : 0.0f;
                const uint32_t x = pack_half(p[0], p[1]), y = pack_half(p[2], p[3]);
                pf[0][nt][0] = transposed(x);
                pf[0][nt][1] = transposed(y);
                if constexpr (kTwo) {
                    pf[1][nt][0] = transposed(pack_half(p[0] - low_half(x), p[1] - high_half(x)));
                    pf[1][nt][1] = transposed(pack_half(p[2] - low_half(y), p[3] - high_half(y)));
                }
                if constexpr (!kTwo) mma(off[nt], ones, pf[0][nt][0], pf[0][nt][1]);
            }
            const uint8_t *row = rec[j] + (size + token[j]) * (D / 2) + g * (VW * 4);
            uint32_t w[4][VW];
            load_words<VW>(row + t * (D / 2), w[0]);
            load_words<VW>(row + (7 - t) * (D / 2), w[1]);
            load_words<VW>(row + (8 + t) * (D / 2), w[2]);
            load_words<VW>(row + (15 - t) * (D / 2), w[3]);
#pragma unroll
            for (int x = 0; x < VW; ++x)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t n0 = __byte_perm(w[0][x], w[1][x], half ? 0x7632 : 0x5410);
                    const uint32_t n1 = __byte_perm(w[2][x], w[3][x], half ? 0x7632 : 0x5410);
                    const uint32_t u0 = n0 >> 8, u1 = n1 >> 8;
                    const uint32_t A[4] = {codes_f16<kTwo, false>(n0), codes_f16<kTwo, true>(n0), codes_f16<kTwo, false>(n1),
                                           codes_f16<kTwo, true>(n1)};
                    const uint32_t B[4] = {codes_f16<kTwo, false>(u0), codes_f16<kTwo, true>(u0), codes_f16<kTwo, false>(u1),
                                           codes_f16<kTwo, true>(u1)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) {
                            mma(o[nt][4 * x + 2 * half], A, pf[part][nt][0], pf[part][nt][1]);
                            mma(o[nt][4 * x + 2 * half + 1], B, pf[part][nt][0], pf[part][nt][1]);
                        }
                }
        }
        __syncwarp();

        if (k.first_last & 2) {
            // ---- the warp's part of the segment is done: m, l and o of every column to its piece
            bool based = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) based |= base[nt][0] != 0.0f || base[nt][1] != 0.0f;
            if (__any_sync(0xffffffffu, based)) {            // what base + m loses of m goes into l and o
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float rest = exp2_fast(base[nt][y] - (base[nt][y] + m[nt][y]) + m[nt][y]);
                        l[nt][y] *= rest;
                        off[nt][y] *= rest;
#pragma unroll
                        for (int x = 0; x < STEPS; ++x) {
                            o[nt][x][y] *= rest;
                            o[nt][x][2 + y] *= rest;
                        }
                    }
            }
            float *to_piece = joined ? reinterpret_cast<float *>(mine) : a.pieces + piece * piece_floats(D, COLS);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float x = l[nt][y];
#pragma unroll
                    for (int h = 4; h < 32; h *= 2) x += __shfl_xor_sync(0xffffffffu, x, h);
                    const int col = nt * 8 + 2 * t + y;
                    if (g == 0) {
                        to_piece[col] = base[nt][y] + m[nt][y];
                        to_piece[COLS + col] = x;
                    }
                    float *p = to_piece + 2 * COLS + col * D + g * (D / 8);
#pragma unroll
                    for (int x = 0; x < STEPS; ++x)
                        *reinterpret_cast<float2 *>(p + 2 * x) =
                            make_float2((o[nt][x][y] - off[nt][y]) * kUnit, (o[nt][x][2 + y] * kOdd - off[nt][y]) * kUnit);
                }
            piece = next_piece++;
        }
        if (!joined || i + STAGES < units) ask();
    }
    if (!sound) {
        // copies still on their way have to land before the CTA leaves
        const long long t0 = clock64();
        for (int i = 0; i < STAGES; ++i)
            if (i < asked) {
                const int last = (asked - 1 - i) / STAGES, stage = (asked - 1 - i) % STAGES;
                while (!tc::mbar_try_wait(bars + 8 * stage, (uint32_t)last & 1u) && clock64() - t0 < tc::kWaitLimitCycles) {}
            }
    }
    if (!joined) return;

    // ---- one segment: the warps' parts become one piece
    if (from == to && lane < COLS) {
        float *p = reinterpret_cast<float *>(mine);
        p[lane] = kLowest;
        p[COLS + lane] = 0.0f;
    }
    __syncthreads();
    if (s_abort) return;
    // a warp per column: a lane each for the warps' maxima, then all lanes along the head
    for (int col = warp; col < COLS; col += WARPS) {
        const int token = a.direct ? (first_x + col) / a.group : 0;
        if (a.direct && token >= first.m) break;
        const uint8_t *part = smem + min(lane, WARPS - 1) * warp_smem(D, NT) + 4 * col;
        const float pm = load_float(part), pl = lane < WARPS ? load_float(part + 4 * COLS) : 0.0f;
        float most = pl == 0.0f ? kLowest : pm;
#pragma unroll
        for (int d = 16; d; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        float sum = pl, v[E];
        const float by = pl == 0.0f ? 0.0f : lowered(sum, pm - most);
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = __shfl_sync(0xffffffffu, by, w);
            const uint8_t *p = smem + w * warp_smem(D, NT) + 4 * (2 * COLS + col * D + lane);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = load_float(p + 128 * e);     // (anything, where the warp had no keys)
                v[e] = f == 0.0f ? v[e] : fmaf(f, x, v[e]);
            }
        }
        if (a.direct) {
            finish<D, T>(a, first.begin + token, first_head * a.group + first_x + col - token * a.group, lane, v, sum);
        } else {
            float *out = a.pieces + joined_place * piece_floats(D, COLS);
#pragma unroll
            for (int e = 0; e < E; ++e) out[2 * COLS + col * D + 32 * e + lane] = v[e];
            if (lane == 0) {
                out[col] = most;
                out[COLS + col] = sum;
            }
        }
    }
}

// Joins the pieces of every row and head: o = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p, transformed back. A warp has
// a row and a head, or `ways` warps next to each other share one's pieces.
template <int D, typename T, int NT>
__global__ void __launch_bounds__(256) join_kernel(const AttendArgs a, int ctas, int ways) {
    constexpr int COLS = 8 * NT, WARPS = kWarps(D, NT), E = D / 32;
    __shared__ float s_m[8], s_l[8], s_o[8][D];
    after_prior_kernels();
    if (__syncthreads_or(*reinterpret_cast<volatile int *>(a.err) != 0)) return;
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_row = (a.q_heads * ways + 7) / 8;          // CTAs
    const int r = (int)(blockIdx.x / per_row), way = warp % ways, q_head = (int)(blockIdx.x % per_row) * (8 / ways) + warp / ways;
    const int head = q_head / a.group, h = q_head - head * a.group;
    int b, begin, end;
    if (!sequence_of(c, r, lane, b, begin, end)) return;
    Sequence s{};
    measure<COLS>(c, a.group, s, b, begin, end);
    const long long before = a.before[2 * b], segs = a.before[2 * b + 1], total = a.before[2 * c.seqs];
    const Parts parts(total, ctas, WARPS);
    const long long cta_units = parts.active * parts.units;
    const int x = (r - begin) * a.group + h, tile = x / COLS, col = x % COLS;
    float mx = kLowest, l = 0.0f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    if (q_head < a.q_heads && s.chunks > 0) {
        // The segment's pieces: those of its first CTA (one if that lies in the segment, else its warps'), one of each
        // CTA between, those of its last.
        const long long seg = (long long)head * s.tiles + tile, u0 = before + seg * s.chunks, u1 = u0 + s.chunks;
        const long long c0 = divide(u0, cta_units), c1 = divide(u1 - 1, cta_units);
        const long long from0 = c0 * cta_units, to0 = min(total, from0 + cta_units), from1 = c1 * cta_units;
        const bool one0 = from0 == u0 && to0 <= u1, one1 = min(total, from1 + cta_units) <= u1;
        const int w0 = (int)divide(u0 - from0, parts.units);
        const int n0 = one0 ? 1 : (int)divide(min(u1, to0) - 1 - from0, parts.units) - w0 + 1;
        const int n1 = c1 == c0 ? 0 : one1 ? 1 : (int)divide(u1 - 1 - from1, parts.units) + 1;
        const int between = (int)max(c1 - c0 - 1, 0LL), n = n0 + between + n1;
        // 32 pieces at a time: a lane each for their maxima, then all lanes along the head
        for (int i0 = 0; i0 < n; i0 += 32 * ways) {
            const int i = i0 + lane * ways + way;
            long long place = 0;
            if (i == 0) place = segs + seg;
            else if (i < n0) place = a.segments + c0 * WARPS + w0 + i;
            else if (i < n0 + between) place = a.segments + (c0 + 1 + i - n0) * WARPS;
            else place = a.segments + c1 * WARPS + i - n0 - between;
            float pm = kLowest, pl = 0.0f;
            if (i < n) {
                pm = a.pieces[place * piece_floats(D, COLS) + col];
                pl = a.pieces[place * piece_floats(D, COLS) + COLS + col];
            }
            if (pl == 0.0f) pm = kLowest;
            float now = fmaxf(mx, pm);
#pragma unroll
            for (int d = 16; d; d /= 2) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, d));
            const float by = lowered(l, mx - now), add = pl == 0.0f ? 0.0f : lowered(pl, pm - now);
            mx = now;
            float sum = pl;
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            l += sum;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= by;
            const int here = min(32, (n - i0 - way + ways - 1) / ways);
#pragma unroll 4
            for (int y = 0; y < here; ++y) {
                const float f = __shfl_sync(0xffffffffu, add, y);
                const float *p = a.pieces + __shfl_sync(0xffffffffu, place, y) * piece_floats(D, COLS) + 2 * COLS + col * D + lane;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(f, p[32 * e], o[e]);
            }
        }
    }
    if (ways > 1) {
        if (lane == 0) {
            s_m[warp] = mx;
            s_l[warp] = l;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[warp][32 * e + lane] = o[e];
        __syncthreads();
        if (way) return;
        const float pm = lane < ways ? s_m[warp + lane] : kLowest;
        float pl = lane < ways ? s_l[warp + lane] : 0.0f;
        mx = pl == 0.0f ? kLowest : pm;
#pragma unroll
        for (int d = 4; d; d /= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float by = pl == 0.0f ? 0.0f : lowered(pl, pm - mx);
        l = pl;
#pragma unroll
        for (int d = 4; d; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
        l = __shfl_sync(0xffffffffu, l, 0);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.0f;
        for (int y = 0; y < ways; ++y) {
            const float f = __shfl_sync(0xffffffffu, by, y);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(f, s_o[warp + y][32 * e + lane], o[e]);
        }
    }
    if (q_head < a.q_heads) finish<D, T>(a, r, q_head, lane, o, l);
}

template <int D, typename T, int NT, int WARPS>
cudaError_t launch_warps(const AttendArgs &a, cudaStream_t s) {
    static std::atomic<int> allowed[64];
    constexpr int bytes = WARPS * warp_smem(D, NT) + NT * (D / 32) * 512 * (std::is_same<T, __half>::value ? 2 : 1) + 32 * NT;
    static_assert(bytes <= 227 * 1024 - 256, "shared memory of a CTA");
    cudaError_t e = allow_shared(reinterpret_cast<const void *>(attend_kernel<D, T, NT, WARPS>), bytes, allowed);
    if (e != cudaSuccess) return e;
    if ((e = launch_early(attend_kernel<D, T, NT, WARPS>, dim3((unsigned)(a.direct ? a.segments : a.sms)), WARPS * 32, bytes, s, a)) != cudaSuccess ||
        a.direct)
        return e;
    // warps: no fewer than two for every SM's four schedulers
    int ways = 1;
    while (ways < 8 && (long long)a.c.rows * a.q_heads * ways < 8 * a.sms) ways *= 2;
    const long long joiners = (long long)a.c.rows * ((a.q_heads * ways + 7) / 8);
    return launch_early(join_kernel<D, T, NT>, dim3((unsigned)joiners), 256, 0, s, a, a.sms, ways);
}
template <int D, typename T, int NT>
cudaError_t launch(const AttendArgs &a, cudaStream_t s) {
    return a.direct == 2 ? launch_warps<D, T, NT, kWarps(D, NT) / 2>(a, s) : launch_warps<D, T, NT, kWarps(D, NT)>(a, s);
}
template <int D, typename T>
cudaError_t launch_columns(const AttendArgs &a, cudaStream_t s) {
    if constexpr (D <= 128)
        if (a.columns == 16) return launch<D, T, 2>(a, s);
    return launch<D, T, 1>(a, s);
}
template <typename T>
cudaError_t launch_type(const AttendArgs &a, cudaStream_t s) {
    switch (a.c.width) {
        case 64: return launch_columns<64, T>(a, s);
        case 128: return launch_columns<128, T>(a, s);
        case 192: return launch_columns<192, T>(a, s);
        default: return launch_columns<256, T>(a, s);
    }
}

}  // namespace

// 16 columns where most sequences have more than 8 (queries times heads of a group)
int attend_columns(int width, int group, long long rows, int seqs) { return width <= 128 && rows * group > 8LL * seqs ? 16 : 8; }
int attend_workers(int width, int sms) { return sms * kWarps(width, 1); }
int attend_direct(int width, int columns, long long segments, int capacity, int sms) {
    if (segments >= 1LL << 31) return 0;
    // All the host knows of lengths is the table's width. Measured: a CTA takes about 4 us to set out and end, a warp 1.2 us
    // for a chunk, or what the memory takes where all SMs are at work (2.4 us for 12 warps' chunks of heads of 128); equal
    // parts and the second kernel 18 us for both, and about 4.5 us (heads of 128) for the queries of every segment a warp
    // comes to. Two CTAs of half the warps an SM where there are more segments than SMs: one sets out while the other reads.
    // Direct against parts: 256 segments of 2050 keys, 64 wide, 18.9 us against 24; 328 of 320, 192 wide, 25 against 38;
    // 512 of 8192 and fewer, 128 wide, 94 against 78; 2048 of one key, 192 wide, 62 against 45.
    const int per_sm = segments > sms ? 2 : 1, full = kWarps(width, columns / 8), warps = full / per_sm;
    const double slots = (double)sms * per_sm, chunks = (double)((capacity + kChunk - 1) / kChunk), workers = (double)sms * full;
    const double memory = 2.4 * width / 128, waves = std::ceil((double)segments / slots), steps = std::ceil(chunks / warps);
    const double direct = waves * (4 + std::max(1.2, memory * std::min(1.0, (double)segments / slots)) * steps);
    const double parts = 18 + (double)segments * chunks / workers * memory + (double)segments / workers * 4.5 * (width / 128.0) * (width / 128.0);
    return direct <= parts ? per_sm : 0;
}
cudaError_t launch_attend(const AttendArgs &a, int type, cudaStream_t s) {
    return type == HATQ_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace hatq
