// Host-side helpers shared by the token operators' entry points: messages of
// refusals, checks of alignment and overlap, limits of a call. Not part of the
// public ABI.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "hatq_internal.h"

namespace {

hatq_status fail(hatq_status st, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return hatq::report(st, buf);
}
hatq_status cuda_fail(cudaError_t e, const char *what) {
    return fail(HATQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t type_size(int t) { return t == HATQ_F32 ? 4 : 2; }
bool is_type(int t) { return t == HATQ_F32 || t == HATQ_F16 || t == HATQ_BF16; }
size_t codes_size(int f) { return f == HATQ_CODES_F16 ? 2 : 1; }
bool is_codes(int f) { return f == HATQ_CODES_I8 || f == HATQ_CODES_F16; }
int round_up(int v, int m) { return (v + m - 1) / m * m; }

// Whether rows of width elements at a pitch share memory with others. Rows between one another, as the columns of one
// buffer, do not: where both have the same pitch, their places within it are compared. (A single row has any pitch.)
bool overlap(const void *p, long long p_rows, long long p_pitch, long long p_width, size_t p_size, const void *q,
             long long q_rows, long long q_pitch, long long q_width, size_t q_size) {
    if (p_rows == 0 || q_rows == 0) return false;
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(p), q0 = reinterpret_cast<uintptr_t>(q);
    const uintptr_t p_bytes = (uintptr_t)p_width * p_size, q_bytes = (uintptr_t)q_width * q_size;
    const uintptr_t p_step = (uintptr_t)p_pitch * p_size, q_step = (uintptr_t)q_pitch * q_size;
    const uintptr_t p1 = p0 + (uintptr_t)(p_rows - 1) * p_step + p_bytes, q1 = q0 + (uintptr_t)(q_rows - 1) * q_step + q_bytes;
    if (!(p0 < q1 && q0 < p1)) return false;
    if (p_rows > 1 && q_rows > 1 ? p_step != q_step : p_rows == 1 && q_rows == 1) return true;
    const uintptr_t step = p_rows > 1 ? p_step : q_step;
    if (step == 0) return true;                              // (all of its rows are one)
    const uintptr_t at = q0 >= p0 ? (q0 - p0) % step : (step - (p0 - q0) % step) % step;   // q's place, p's is 0
    return at < p_bytes || at + q_bytes > step;
}

constexpr long long kMaxRows = (1LL << 31) - 1024;
constexpr long long kMaxPitch = 1LL << 32;

int sm_count() {
    static int counts[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (!counts[dev]) {
        int v = 0;
        if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        counts[dev] = v;
    }
    return counts[dev];
}

}  // namespace
