// How the attention kernels lay out their work over the sequences of a call.
// Not part of the public ABI.
#pragma once

#include "hatq_cache.h"

namespace hatq {

// The row of chunks: sequence after sequence, in it head after head, in it tile after tile of the columns.
struct Sequence {
    int b, begin, m, len;              // its index, first row, new tokens, length
    int tiles, chunks;                 // column tiles of a head, chunks of 64 keys
    long long unit, segment;           // units and segments (head, tile) of the sequences before it
    __device__ long long units(int heads) const { return (long long)heads * tiles * chunks; }
    __device__ long long segments(int heads) const { return chunks ? (long long)heads * tiles : 0; }
};

template <int COLS>
__device__ __forceinline__ void measure(const CacheArgs &c, int group, Sequence &s, int b, int most_before, int next) {
    s.b = b;
    s.begin = min(max(most_before, 0), c.rows);
    s.m = min(max(next, 0), c.rows) - s.begin;
    if (s.m < 0) s.m = 0;
    s.len = length_of(c, b);
    s.tiles = (int)(((long long)s.m * group + COLS - 1) / COLS);
    s.chunks = (s.len + kChunk - 1) / kChunk;
}

// (small: the sum of all is below 2^31)
__device__ __forceinline__ long long scan_add(long long v, int lane, bool small) {
    if (small) {
        int u = (int)v;
#pragma unroll
        for (int h = 1; h < 32; h *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, u, h);
            if (lane >= h) u += o;
        }
        return u;
    }
#pragma unroll
    for (int h = 1; h < 32; h *= 2) {
        const long long o = __shfl_up_sync(0xffffffffu, v, h);
        if (lane >= h) v += o;
    }
    return v;
}
__device__ __forceinline__ int scan_max(int v) {
#pragma unroll
    for (int h = 1; h < 32; h *= 2) v = max(v, __shfl_up_sync(0xffffffffu, v, h));     // (lane < h: its own)
    return v;
}
// quotients are of numbers below 2^32 nearly always
__device__ __forceinline__ long long divide(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// All sequences as one warp holds them: every lane a run of `per` of them, and what lies before it.
template <int COLS>
struct Row {
    bool flat;                         // units are segments, those of sequences without tokens among them
    int per, most;                     // most: of the offsets before the lane's run
    long long units, segments;         // before the lane's run
    long long total;
    Sequence own;                      // per == 1: the lane's sequence

    __device__ __forceinline__ long long units_of(const Sequence &s, int heads) const {
        return flat ? (long long)heads * s.tiles : s.units(heads);
    }
    // the next sequence of the lane's run
    __device__ __forceinline__ void take(const CacheArgs &c, int group, Sequence &s, int b, int &most) const {
        if (c.starts) {
            const int here = max(c.starts[b], most), next = max(c.starts[b + 1], here);
            measure<COLS>(c, group, s, b, here, next);
            most = next;
        } else {
            measure<COLS>(c, group, s, b, b, b + 1);
        }
    }
    __device__ __forceinline__ void read(const CacheArgs &c, int group, int lane, bool flat_) {
        flat = flat_;
        per = (c.seqs + 31) / 32;
        const int from = min(lane * per, c.seqs), to = min(from + per, c.seqs);
        most = 0;
        if (c.starts) {
            int mine = 0;
            for (int b = from; b < to; ++b) mine = max(mine, c.starts[b]);
            const int before = __shfl_up_sync(0xffffffffu, scan_max(mine), 1);
            most = lane ? max(before, 0) : 0;
        }
        long long u = 0, sg = 0;
        int m = most;
        for (int b = from; b < to; ++b) {
            Sequence s{};
            take(c, group, s, b, m);
            u += units_of(s, c.heads);
            sg += s.segments(c.heads);
            own = s;
        }
        const long long up_to = scan_add(u, lane, c.small);
        units = up_to - u;
        segments = scan_add(sg, lane, c.small) - sg;
        total = __shfl_sync(0xffffffffu, up_to, 31);
    }
    __device__ __forceinline__ static void copy(Sequence &to, const Sequence &s, long long unit, long long segment, int from) {
        to.b = __shfl_sync(0xffffffffu, s.b, from);
        to.begin = __shfl_sync(0xffffffffu, s.begin, from);
        to.m = __shfl_sync(0xffffffffu, s.m, from);
        to.len = __shfl_sync(0xffffffffu, s.len, from);
        to.tiles = __shfl_sync(0xffffffffu, s.tiles, from);
        to.chunks = __shfl_sync(0xffffffffu, s.chunks, from);
        to.unit = __shfl_sync(0xffffffffu, unit, from);
        to.segment = __shfl_sync(0xffffffffu, segment, from);
    }
    // the sequence that holds a unit (0 <= unit < total)
    __device__ __forceinline__ void find_unit(const CacheArgs &c, int group, int lane, long long unit, Sequence &found) const {
        // the last lane whose run begins at or before it: those behind the last sequence begin at total
        const int who = 31 - __clz(__ballot_sync(0xffffffffu, units <= unit));
        if (per == 1) {
            copy(found, own, units, segments, who);
            return;
        }
        const int from = who * per, to = min(from + per, c.seqs);
        int m = __shfl_sync(0xffffffffu, most, who);
        long long u = __shfl_sync(0xffffffffu, units, who), sg = __shfl_sync(0xffffffffu, segments, who);
        for (int b0 = from;; b0 += 32) {
            const int b = b0 + lane;
            Sequence s{};
            if (c.starts) {
                const int here = scan_max(max(b < to ? c.starts[b] : 0, m)), next = max(b < to ? c.starts[b + 1] : 0, here);
                if (b < to) measure<COLS>(c, group, s, b, here, next);
                m = __shfl_sync(0xffffffffu, next, 31);
            } else if (b < to) {
                measure<COLS>(c, group, s, b, b, b + 1);
            }
            const long long n = units_of(s, c.heads), up_to = u + scan_add(n, lane, c.small);
            const long long segs = sg + scan_add(s.segments(c.heads), lane, c.small);
            const unsigned here = __ballot_sync(0xffffffffu, unit < up_to);
            if (here || b0 + 32 >= to) {
                copy(found, s, up_to - n, segs - s.segments(c.heads), here ? __ffs(here) - 1 : 31);
                return;
            }
            u = __shfl_sync(0xffffffffu, up_to, 31);
            sg = __shfl_sync(0xffffffffu, segs, 31);
        }
    }
    // units and segments before every sequence, and all units, to memory
    __device__ __forceinline__ void write(const CacheArgs &c, int group, int lane, long long *to) const {
        const int from = min(lane * per, c.seqs), end = min(from + per, c.seqs);
        long long u = units, sg = segments;
        int m = most;
        for (int b = from; b < end; ++b) {
            to[2 * b] = u;
            to[2 * b + 1] = sg;
            Sequence s{};
            take(c, group, s, b, m);
            u += units_of(s, c.heads);
            sg += s.segments(c.heads);
        }
        if (lane == 0) to[2 * c.seqs] = total;
    }
};

}  // namespace hatq
