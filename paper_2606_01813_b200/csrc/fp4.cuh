// The 4-bit form in registers.
//
// Codes become fp16 pairs by the conversion instruction, four for a 32-bit word of eight codes, and one packed product with the
// scale for each pair: 10 cycles a word and warp on an SM's quarter, against some 22 for shifting and masking the codes into
// bf16's fields (logic instructions issue every second cycle; measured on a B200).  code * scale has at most six significant
// bits and lies in [2^-10, 2688]: exact in fp16.
//
// The other factor, queries, comes as bf16, whose range fp16 does not have.  A row of queries is therefore divided by the power
// of two that brings its largest element into [1, 2) (half_row_exponent), which its scores are multiplied by again: elements down
// to 2^-14 of the largest stay exact, smaller ones are off by at most 2^-25 of the largest.
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

// Eight codes times a scale (twice in `f`, fp16), elements in order.
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint4 fp4_half_values(uint32_t w, uint32_t f) {
    uint4 r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(w));
    return make_uint4(mul_f16x2(r.x, f), mul_f16x2(r.y, f), mul_f16x2(r.z, f), mul_f16x2(r.w, f));
}
// Two neighbouring scale bytes as fp16, each twice.
__device__ __forceinline__ void fp4_half_scales(uint32_t two_bytes, uint32_t& f0, uint32_t& f1) {
    uint32_t t;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(t) : "h"((unsigned short)two_bytes));
    f0 = __byte_perm(t, 0, 0x1010);
    f1 = __byte_perm(t, 0, 0x3232);
}
// Exponent of the largest magnitude of a row; 0 for a row of zeros or one with non-finite elements (which stay what they are).
__device__ __forceinline__ int half_row_exponent(float amax) {
    const int e = (int)((__float_as_uint(amax) >> 23) & 255u) - 127;
    return e < -126 || e > 127 ? 0 : e;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Eight bf16 elements times 2^-e as fp16.
__device__ __forceinline__ uint4 half_chunk(const uint4& x, float down) {
    float f[8];
    Elem<CADD_DTYPE_BF16>::unpack(x, f);
    return make_uint4(pack_half(f[0] * down, f[1] * down), pack_half(f[2] * down, f[3] * down), pack_half(f[4] * down, f[5] * down), pack_half(f[6] * down, f[7] * down));
}
__device__ __forceinline__ float chunk_amax(const uint4& x) {
    float f[8], m = 0.0f;
    Elem<CADD_DTYPE_BF16>::unpack(x, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = !(fabsf(f[i]) <= m) ? fabsf(f[i]) : m;            // NaN stays
    return m;
}

}  // namespace cadd
