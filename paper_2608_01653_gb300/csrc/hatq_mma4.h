// Tensor-core steps on 4-bit codes, shared by the attention over the cache and
// the products with 4-bit weights. Not part of the public ABI.
#pragma once

#include <stdint.h>

namespace hatq {

// D += A B, 16 x 8 x 16: both operands fp16, or both bf16
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// D += A B, and D = A B
template <bool HALF>
__device__ __forceinline__ void mma_more(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF) mma(d, a, b0, b1);
    else mma_bf16(d, a, b0, b1);
}
template <bool HALF>
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}

// (w & mask) | bits in one instruction, which has room for one constant: the other is in a register
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t mask, uint32_t bits) {
    uint32_t x;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w), "r"(mask), "r"(bits));
    return x;
}
// The codes of a word at bits 0-3 (ODD: 4-7) of its halves, as A operands: bare, subnormal numbers (code + 8) 2^-24 and
// 2^-20, or (WHOLE) the codes themselves: 1024 + x and 1024 + 16 x are fp16 numbers whose last bits are x.
template <bool WHOLE, bool ODD>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {
    if constexpr (!WHOLE) return w & (ODD ? 0x00f000f0u : 0x000f000fu);
    uint32_t x = masked(w, ODD ? 0x00f000f0u : 0x000f000fu, 0x64006400u);
    if constexpr (ODD)
        asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(x) : "r"(0x2c002c00u), "r"(0xd480d480u));      // x / 16 - 72
    else
        asm("add.rn.f16x2 %0, %0, %1;" : "+r"(x) : "r"(0xe408e408u));                            // x - 1032
    return x;
}

// The codes at bits 0-3 of a word's halves as bf16: 128 + x has x in its last bits.
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
    uint32_t x = masked(w, 0x000f000fu, 0x43004300u);
    asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(x) : "r"(0xc308c308u));                               // x - 136
    return x;
}

}  // namespace hatq
