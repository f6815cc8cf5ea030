// The 4-bit form in registers.
//
// Codes become fp16 pairs by the conversion instruction, four for a 32-bit word of eight codes, and one packed product with the
// scale for each pair: 10 cycles a word and warp on an SM's quarter, against some 22 for shifting and masking the codes into
// bf16's fields (logic instructions issue every second cycle; measured on a B200).  code * scale has at most six significant
// bits and lies in [2^-10, 2688]: exact in fp16.
//
// The other factor, queries, comes as bf16, whose range fp16 does not have.  A row of queries is therefore multiplied by the power
// of two that brings its largest element into [2^14, 2^15) (half_row_exponent), and its scores by the inverse: bf16's eight bits
// then fit fp16 exactly down to 2^-31 of the largest element.  Smaller ones are rounded, by at most 2^-25; where that could move a
// score by more than 2^-20 of a power of two, or the largest element is beyond 2^54, the row is lost to fp16 (half_row_lost) and
// goes another way: slower, and not rounded.
#pragma once
#include <cuda_fp16.h>
#include "common.cuh"

namespace cadd {

__device__ __forceinline__ float exp2i(int e) { return __int_as_float((e + 127) << 23); }          // 2^e, -126 <= e <= 127
// An e2m1 code (four bits: sign, two of exponent, one behind the point) in fp32: the three low bits moved to where fp32 keeps
// the low exponent bits and the first fraction bit give the number times 2^-126 (0.5 as an fp32 subnormal).
__device__ __forceinline__ float e2m1_value(uint32_t c) {
    return __uint_as_float(((c & 7u) << 22) | ((c & 8u) << 28)) * 0x1p126f;
}
// The same for an e4m3 number that is not negative: seven bits, times 2^-120.
__device__ __forceinline__ float e4m3_value(uint32_t c) { return __uint_as_float((c & 0x7fu) << 20) * 0x1p120f; }
__device__ __forceinline__ uint32_t e2m1_byte(float lo, float hi) {
    uint32_t byte;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(byte) : "f"(hi), "f"(lo));
    return byte & 0xffu;
}
__device__ __forceinline__ uint32_t e4m3_byte(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(x));
    return r & 0xffu;
}

// Zero has one code: where the conversion keeps the sign of a small negative number, 8, the sign is taken off.  (Seven added to a
// nibble's three low bits carries into its high bit where they are not zero, and never beyond.)
__device__ __forceinline__ uint32_t e2m1_one_zero(uint32_t w) { return w & (((w & 0x77777777u) + 0x77777777u) | 0x77777777u); }

// 16 bf16 elements times `up` (a power of two) -> 8 code bytes and a scale byte: scale = e4m3(amax / 6), code = e2m1(x / scale).
//
// What makes the codes those of exact arithmetic: x has 8 significant bits, the scale 4, a point half way between two codes 3.
// So x / scale is either exactly such a point or off it by more than 2^-16 of itself, and it is enough to have the quotient to
// 2^-20 and exactly where it is such a point.  q = x r with r = 1 / scale rounded is off by a few 2^-24; one correction with the
// exact remainder, q + (x - q scale) r, leaves the square of that, so a half-way point comes out as itself.  (amax / 6 is one
// division for the 16; the same argument holds for it.)  Blocks with NaN or infinities, and those whose products would leave
// fp32's range, take true divisions: NaN becomes 0, the rest saturates.
__device__ __noinline__ uint2 fp4_encode_slow(const uint4 w0, const uint4 w1, float up, uint32_t& scale_byte) {
    float x[16], amax = 0.0f;
    Elem<CADD_DTYPE_BF16>::unpack(w0, x);
    Elem<CADD_DTYPE_BF16>::unpack(w1, x + 8);
    for (int i = 0; i < 16; ++i) { x[i] *= up; amax = fmaxf(amax, fabsf(x[i])); }      // fmaxf ignores NaN
    scale_byte = e4m3_byte(__fdiv_rn(amax, 6.0f)) & 0x7fu;
    const float s = e4m3_value(scale_byte);
    uint32_t w[2] = {0u, 0u};
    for (int i = 0; i < 16 && scale_byte; i += 2) {
        float a = __fdiv_rn(x[i], s), b = __fdiv_rn(x[i + 1], s);
        a = a == a ? a : 0.0f;
        b = b == b ? b : 0.0f;
        w[i >> 3] |= e2m1_byte(a, b) << ((i & 7) * 4);
    }
    return make_uint2(e2m1_one_zero(w[0]), e2m1_one_zero(w[1]));
}
__device__ __forceinline__ uint2 fp4_encode(const uint4& w0, const uint4& w1, float up, uint32_t& scale_byte) {
    const uint32_t in[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
    uint32_t big = 0;                                    // the magnitudes' bits order like the magnitudes, NaN above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) big = __vmaxu2(big, in[i] & 0x7fff7fffu);
    big = max(big & 0xffffu, big >> 16);
    if (big >= 0x7000u) return fp4_encode_slow(w0, w1, up, scale_byte);                // 2^97 and more, infinities, NaN
    scale_byte = e4m3_byte(__fdiv_rn(__uint_as_float(big << 16) * up, 6.0f)) & 0x7fu;
    const float s = e4m3_value(scale_byte), r = scale_byte ? __frcp_rn(s) : 0.0f;      // a zero scale: zero codes
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __uint_as_float(in[i] << 16) * up, b = __uint_as_float(in[i] & 0xffff0000u) * up;
        const float qa = a * r, qb = b * r;
        w[i >> 2] |= e2m1_byte(fmaf(fmaf(-qa, s, a), r, qa), fmaf(fmaf(-qb, s, b), r, qb)) << ((i & 3) * 8);
    }
    return make_uint2(e2m1_one_zero(w[0]), e2m1_one_zero(w[1]));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A pair of fp16 numbers code * scale as bf16: exact, both hold six significant bits.
__device__ __forceinline__ uint32_t bf16_of_half(uint32_t x) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
    return pack_bf16(f.x, f.y);
}

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
    // A nibble times 2^6 + 2^12 (2^2 + 2^8 for the second of a byte) has its three low bits at 6..8 and its sign at 15, and
    // nothing is carried between the two copies: a product and two masks a pair, the product off the logic unit.
    constexpr uint32_t keep = 0x81c081c0u;
    const uint32_t h = w >> 8;
    uint4 r;
    r.x = mul_bf16x2(((w & 0x000f000fu) * 4160u) & keep, f);
    r.y = mul_bf16x2(((w & 0x00f000f0u) * 260u) & keep, f);
    r.z = mul_bf16x2(((h & 0x000f000fu) * 4160u) & keep, f);
    r.w = mul_bf16x2(((h & 0x00f000f0u) * 260u) & keep, f);
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
// The power of two that a row with this largest magnitude is divided by for fp16; 0 for a row of zeros or one with non-finite elements
// (which stay what they are).
__device__ __forceinline__ int half_row_exponent(float amax) {
    const int e = (int)((__float_as_uint(amax) >> 23) & 255u) - 127;
    return e < -126 || e > 127 ? 0 : e - 14;
}
constexpr int kHalfMaxExponent = 40;                     // scale * 2^(e - k_exp) stays a normal fp32 number
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// What a chunk meets on its way to fp16.
constexpr unsigned kHalfRounded = 1;                     // an element rounded, by at most 2^-25
constexpr unsigned kHalfUnfit = 2;                       // one that does not fit, or NaN
// Eight elements of a row with largest magnitude `amax`, times 2^-e as fp16; e is chosen here.
__device__ __forceinline__ uint4 half_row_chunk(const uint4& x, float amax, int& e, unsigned& met) {
    const int want = half_row_exponent(amax);
    e = min(max(want, -kHalfMaxExponent), kHalfMaxExponent);
    if (want > e) met |= kHalfUnfit;
    const float down = exp2i(-e);
    float f[8];
    Elem<CADD_DTYPE_BF16>::unpack(x, f);
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = pack_half(f[2 * i] * down, f[2 * i + 1] * down);
        const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&r[i]));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float was = f[2 * i + j] * down, is = j ? back.y : back.x;
            if (was != is) met |= fabsf(was - is) <= 0x1p-25f ? kHalfRounded : kHalfUnfit;
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}
// Is a row lost to fp16?  `rounded`, `unfit`: its chunks that met either; `scale`: of its scores.  Values of keys are at most 2688.
__device__ __forceinline__ bool half_row_lost(unsigned rounded, unsigned unfit, float scale) {
    return unfit || (float)(__popc(rounded) * 8) * (2688.0f * 0x1p-25f) * scale > 0x1p-20f;
}
__device__ __forceinline__ float chunk_amax(const uint4& x) {
    float f[8], m = 0.0f;
    Elem<CADD_DTYPE_BF16>::unpack(x, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = !(fabsf(f[i]) <= m) ? fabsf(f[i]) : m;            // NaN stays
    return m;
}

}  // namespace cadd
