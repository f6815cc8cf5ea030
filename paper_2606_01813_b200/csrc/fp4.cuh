// The 4-bit form in registers: codes to bf16 pairs without a table.
#pragma once
#include "cache.cuh"

namespace cadd {

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Elements 0..7 of a chunk in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ uint4 order_pairs(uint4 w) {
    return make_uint4(__byte_perm(w.x, w.z, 0x5410), __byte_perm(w.x, w.z, 0x7632), __byte_perm(w.y, w.w, 0x5410), __byte_perm(w.y, w.w, 0x7632));
}
// Eight e2m1 codes times a scale: `f` holds scale * 2^118 twice; the result is code * scale * 2^-8 in the order above.
__device__ __forceinline__ uint4 fp4_unit_values(uint32_t w, uint32_t f) {
    uint4 r;
    r.x = mul_bf16x2(((w << 6) & 0x01c001c0u) | ((w << 12) & 0x80008000u), f);
    r.y = mul_bf16x2(((w << 2) & 0x01c001c0u) | ((w << 8) & 0x80008000u), f);
    r.z = mul_bf16x2(((w >> 2) & 0x01c001c0u) | ((w << 4) & 0x80008000u), f);
    r.w = mul_bf16x2(((w >> 6) & 0x01c001c0u) | (w & 0x80008000u), f);
    return r;
}
// Scale bytes 2i, 2i+1 of a word as bf16 pairs (each twice), times 2^118: seven bits moved to bf16's exponent and fraction are the
// scale times 2^-120; two multiplications by 2^119 stay inside bf16's range.
__device__ __forceinline__ void fp4_unit_scales(uint32_t two_bytes, uint32_t& f0, uint32_t& f1) {
    uint32_t t = ((two_bytes & 0x7fu) << 4) | ((two_bytes & 0x7f00u) << 12);
    t = mul_bf16x2(mul_bf16x2(t, 0x7b007b00u), 0x7b007b00u);                       // 0x7b00 = 2^119
    f0 = __byte_perm(t, 0, 0x1010);
    f1 = __byte_perm(t, 0, 0x3232);
}

}  // namespace cadd
