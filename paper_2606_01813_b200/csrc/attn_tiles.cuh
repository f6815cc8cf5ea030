// Tree attention on the 5th-generation tensor cores: blocks of 128 rows, units of 128 keys.
//
// For each unit S = Q K^T goes to tensor memory (M 128 = rows, N 128 = keys, contraction over the head's elements), the
// softmax warps turn it into weights P = e^{s - m} in bf16, written over S, and O += P V is accumulated in tensor memory
// (A = P from tensor memory, B = V as it lies, [key][element], i.e. "MN-major").  m is a reference, not the exact maximum: it
// starts as the first unit's maximum and is raised, with O and l multiplied by e^{old - new}, only when a later score exceeds
// it by a factor of more than 2^40 in weight.  Weights above 1 lose nothing, since neither bf16's nor fp32's relative rounding
// depends on the size, and weights, sums and products stay below 2^40 x 2^24 (the 4-bit form's factor) x keys x values; so O
// is touched by the products alone, but for a few units.  l adds the weights before they are rounded.
//
// The 4-bit cache: a code's bits, moved to where bf16 keeps its low exponent bits and first fraction bit, are the number times
// 2^-126; one packed multiplication by scale * 2^118 gives code * scale * 2^-8, exact in bf16 (<= 6 significant bits), for two
// elements at once, and the missing power of two goes into the scores' factor and into the weights' exponent.  A
// 32-bit word holds elements 0..7 of a group; masking the same nibble of its halves pairs elements (j, j + 4), so keys,
// values and queries stand in shared memory in the order 0 4 1 5 2 6 3 7 within each eight (the product with the keys
// does not mind, the values' order is undone when O is written).
//
// Two CTAs share an SM and alternate on the tensor cores and the exponential units; within one, the next unit's keys are on their
// way while the softmax runs, its values while the scores are formed.  256 threads (four warps on each quarter of an SM, which
// leaves 128 registers a thread):
//   warps 0-3  softmax and epilogue, a row (tensor-memory lane) per thread.  Between a unit's weights and the next unit's scores
//              they have nothing else to do, so thread 0 also issues the products; warp 0 owns the tensor memory (256
//              columns: S/P 128, O up to 128);
//   warps 4-7  loaders: keys and values into the 128-byte swizzle, by asynchronous 16-byte copies (bf16), or through registers
//              one unit ahead (4 bits).
// Every wait has an iteration limit; a role that gives up sets an error word and all leave.
//
// A product of a weight 0 with a non-finite value that the row does not see would be NaN.  A range that meets a non-finite result
// says so, and the join does such rows once more, key by key over the keys that they see; that costs nothing otherwise.
#pragma once
#include "attn_plan.cuh"
#include "tcgen05.cuh"

namespace cadd {

constexpr int kTileBM = 128;
constexpr int kTileThreads = 256;
constexpr int kTileTmemCols = 256;
constexpr float kTileSlack = 40.0f;                      // log2 of how far weights may exceed 1 before m is raised

template <int D> struct alignas(1024) TileShared {
    unsigned char q[kTileBM * D * 2];                    // D/64 sub-tiles of 128 rows x 128 bytes
    unsigned char k[kUnit * D * 2];
    unsigned char v[kUnit * D * 2];
    int64_t key_row[2][kUnit];                           // bf16: byte offsets of the unit's rows, -1 for none
    uint64_t k_full, v_full, s_full, p_ready, pv_done, drained;
    PlanShared plan;
    WorkIter<kTileBM> it[kTileThreads / 32];             // a walk per warp: here, not in registers, which are scarce
    uint32_t key_bits[2][4];                             // keys of the unit that exist
    uint32_t tmem_base, error, odd;
};
template <int D> constexpr size_t tile_smem_bytes() { return sizeof(TileShared<D>) + 1024; }

// Bounded wait without a time hint.
__device__ __forceinline__ bool tile_try(uint64_t* bar, unsigned parity) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
template <class Shared>
__device__ __forceinline__ bool tile_wait(Shared& sh, uint64_t* bar, unsigned parity) {
    for (int it = 0; it < (1 << 22); ++it) {
        if (tile_try(bar, parity)) return true;
        if (*(volatile uint32_t*)&sh.error) return false;
    }
    sh.error = 1;
    return false;
}
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {       // whole warp: 32 lanes x 16 columns
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, unsigned bytes) {        // bytes 0: zeros
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
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

// Matrix descriptor of a tile [key][64 elements] of 128-byte rows under the 128-byte swizzle, taken with the elements as the
// leading (N) axis: the next 64 elements lie `tile_bytes` on (leading offset), the next eight keys 1024 bytes on (stride
// offset).  A k-step of 16 keys advances the start by 2048 bytes.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(const void* tile, int k16, uint32_t tile_bytes) {
    const uint32_t addr = smem_u32(tile) + (uint32_t)k16 * 2048u;
    return (uint64_t)((addr >> 4) & 0x3fffu) | ((uint64_t)(tile_bytes >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}
// Instruction descriptors (see kHeadIdesc for the fields): scores, both operands K-major; output, B with N as its leading axis (bit 16).
__host__ __device__ constexpr uint32_t tile_idesc(int n, int b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTileBM >> 4) << 24);
}

// Shared-memory offset of 16-byte chunk `ch` of row `row` in a tile of rows of D bf16 elements (sub-tiles of 64 elements).
__device__ __forceinline__ uint32_t tile_off(int row, int ch) {
    return (uint32_t)((ch >> 3) * (128 * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
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

template <int D> struct Fp4Row {                          // a row of codes and scales on its way
    uint4 w[D / 32];
    uint32_t s[D / 64];
};
template <int D>
__device__ __forceinline__ void fp4_row_load(Fp4Row<D>& x, const unsigned char* pool, const unsigned char* scales, int64_t row) {
    if (row >= 0) {
        const uint4* src = (const uint4*)(pool + row * (D / 2));
        const uint32_t* ss = (const uint32_t*)(scales + row * (D / 16));
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x.w[i] = __ldg(src + i);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) x.s[i] = __ldg(ss + i);
    } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x.w[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) x.s[i] = 0;
    }
}
template <int D>
__device__ __noinline__ void fp4_row_store(const Fp4Row<D> x, unsigned char* tile, int row) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {                   // 32 elements: a 16-byte word of codes, two scales
        uint32_t f0, f1;
        fp4_unit_scales((x.s[i >> 1] >> ((i & 1) * 16)) & 0xffffu, f0, f1);
        *(uint4*)(tile + tile_off(row, i * 4 + 0)) = fp4_unit_values(x.w[i].x, f0);
        *(uint4*)(tile + tile_off(row, i * 4 + 1)) = fp4_unit_values(x.w[i].y, f0);
        *(uint4*)(tile + tile_off(row, i * 4 + 2)) = fp4_unit_values(x.w[i].z, f1);
        *(uint4*)(tile + tile_off(row, i * 4 + 3)) = fp4_unit_values(x.w[i].w, f1);
    }
}

__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The wait names the registers that it makes valid, so that nothing that reads them can be moved in front of it.
__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
__device__ __forceinline__ void mask_scores(uint32_t (&x)[16], uint32_t (&y)[16], uint32_t see) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = (see >> i) & 1u ? x[i] : 0xff800000u;
        y[i] = (see >> (16 + i)) & 1u ? y[i] : 0xff800000u;
    }
}
// A row's scores of a unit lie in tensor memory at `ts`; a load takes some 200 cycles.  First the largest, 64 columns at a time:
__device__ __forceinline__ float tile_max(uint32_t ts, bool masked, const uint32_t (&see)[4]) {
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    uint32_t s[4][16];
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) tmem_ld16(ts + c * 64 + j * 16, s[j]);
        tmem_ld_wait16(s[0]); tmem_ld_wait16(s[1]); tmem_ld_wait16(s[2]); tmem_ld_wait16(s[3]);
        if (masked) {
            mask_scores(s[0], s[1], c ? see[2] : see[0]);
            mask_scores(s[2], s[3], c ? see[3] : see[1]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t (&x)[16] = s[j];
#pragma unroll
            for (int i = 0; i < 8; ++i) mx[i & 3] = max3(mx[i & 3], __uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
        }
    }
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}
// then the weights 2^(s sc + off), written over the scores (columns that have been read already) as packed bf16, and their sum:
// 32 columns are worked on, long enough for the next 32 to arrive.
__device__ __forceinline__ void weights_of(const uint32_t (&x)[16], uint64_t sc2, uint64_t off2, uint64_t (&sum)[2], uint32_t dst) {
    uint32_t pk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float e0, e1;
        unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), sc2, off2), e0, e1);
        e0 = ex2(e0);
        e1 = ex2(e1);
        sum[i & 1] = add2(sum[i & 1], pack2(e0, e1));
        pk[i] = pack_bf16(e0, e1);
    }
    tmem_st8(dst, pk);
}
__device__ __forceinline__ float tile_weights(uint32_t ts, bool masked, const uint32_t (&see)[4], float sc, float off) {
    const uint64_t sc2 = pack2(sc, sc), off2 = pack2(off, off);
    uint64_t sum[2] = {0, 0};
    uint32_t s[4][16];
    tmem_ld16(ts, s[0]);
    tmem_ld16(ts + 16, s[1]);
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
        tmem_ld_wait16(s[0]); tmem_ld_wait16(s[1]);
        tmem_ld16(ts + c * 64 + 32, s[2]);
        tmem_ld16(ts + c * 64 + 48, s[3]);
        if (masked) mask_scores(s[0], s[1], c ? see[2] : see[0]);
        weights_of(s[0], sc2, off2, sum, ts + c * 32);
        weights_of(s[1], sc2, off2, sum, ts + c * 32 + 8);
        tmem_ld_wait16(s[2]); tmem_ld_wait16(s[3]);
        if (c == 0) {
            tmem_ld16(ts + 64, s[0]);
            tmem_ld16(ts + 80, s[1]);
        }
        if (masked) mask_scores(s[2], s[3], c ? see[3] : see[1]);
        weights_of(s[2], sc2, off2, sum, ts + c * 32 + 16);
        weights_of(s[3], sc2, off2, sum, ts + c * 32 + 24);
    }
    float a, b;
    unpack2(add2(sum[0], sum[1]), a, b);
    return a + b;
}

// A warp's walk in shared memory goes on to the next item: one lane moves it, no lane still reads the old or already reads the new.
__device__ __forceinline__ bool tile_next(WorkIter<kTileBM>& it, const AttnParams& p) {
    __syncwarp();
    int more = 0;
    if ((threadIdx.x & 31) == 0) more = it.next(p);
    __syncwarp();
    return __shfl_sync(kFullMask, more, 0) != 0;
}

// The end of an item, a warp's rows: O out of tensor memory (`to`), divided and written, or with m and l to the range's record.  True
// where a row of the thread holds a non-finite number.  (A call of its own, once per item: inlined, its registers would cost the
// units' loop theirs.)
template <int D, bool FP4>
__device__ __noinline__ bool tile_finish(const AttnWork& w, const WorkIter<kTileBM>& it, uint32_t to, bool live, int r, int hq, float m, float l) {
    const AttnParams& p = w.p;
    const int tid = threadIdx.x;
    const bool whole = it.whole();
    const float inv = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
    float* rec = w.records + ((int64_t)blockIdx.x * 2 + (it.u0 > 0 ? 0 : 1)) * record_floats<kTileBM, D>() + tid;
    unsigned char* dst = p.out + ((int64_t)it.b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head) * 2;
    bool odd = false;
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
        uint32_t o[16];
        tmem_ld16(to + c * 16, o);
        tmem_ld_wait16(o);
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= (o[i] & 0x7f800000u) == 0x7f800000u;
        if constexpr (FP4) {                  // undo the order 0 4 1 5 2 6 3 7
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                const uint32_t t[8] = {o[j], o[j + 1], o[j + 2], o[j + 3], o[j + 4], o[j + 5], o[j + 6], o[j + 7]};
#pragma unroll
                for (int i = 0; i < 8; ++i) o[j + (i >> 1) + 4 * (i & 1)] = t[i];
            }
        }
        if (!live) continue;
        if (whole) {
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                uint4 x;
                x.x = pack_bf16(__uint_as_float(o[j]) * inv, __uint_as_float(o[j + 1]) * inv);
                x.y = pack_bf16(__uint_as_float(o[j + 2]) * inv, __uint_as_float(o[j + 3]) * inv);
                x.z = pack_bf16(__uint_as_float(o[j + 4]) * inv, __uint_as_float(o[j + 5]) * inv);
                x.w = pack_bf16(__uint_as_float(o[j + 6]) * inv, __uint_as_float(o[j + 7]) * inv);
                *(uint4*)(dst + c * 32 + j * 2) = x;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) rec[(c * 16 + i) * kTileBM] = __uint_as_float(o[i]);
        }
    }
    if (live && !whole) { rec[D * kTileBM] = m; rec[(D + 1) * kTileBM] = l; }
    if (live && whole && p.lse) p.lse[((int64_t)it.b * p.R + r) * p.heads_q + hq] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
    return odd && live;
}

template <int D, bool FP4>
__global__ void __launch_bounds__(kTileThreads, 2) attn_tiles_kernel(const __grid_constant__ AttnWork w) {
    extern __shared__ __align__(16) unsigned char tile_smem_raw[];
    TileShared<D>& sh = *reinterpret_cast<TileShared<D>*>(tile_smem_raw + ((1024u - (smem_u32(tile_smem_raw) & 1023u)) & 1023u));
    const AttnParams& p = w.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) sh.error = sh.odd = 0;
    WorkIter<kTileBM> begin;
    if (!begin.init(p, sh.plan, blockIdx.x, gridDim.x)) {
        if (tid == 0) { w.items[blockIdx.x] = make_int4(0, 0, 0, kRangeEmpty); w.odd[blockIdx.x] = 0; }
        return;
    }
    WorkIter<kTileBM>& it = sh.it[warp];
    if (lane == 0) it = begin;
    __syncwarp();
    if (tid == 0) {
        w.items[blockIdx.x] = make_int4(it.b, it.h, it.mb, (it.u0 > 0 ? kRangeInside : 0) | (it.u1 == it.n_units ? kRangeEnds : 0));
        mbar_init(&sh.k_full, 4);
        mbar_init(&sh.v_full, 4);
        mbar_init(&sh.s_full, 1);
        mbar_init(&sh.p_ready, 4);
        mbar_init(&sh.pv_done, 1);
        mbar_init(&sh.drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc(&sh.tmem_base, kTileTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm_s = *(volatile uint32_t*)&sh.tmem_base, tm_o = tm_s + kUnit;
    constexpr int kCh = D / 8;                            // 16-byte chunks of a bf16 row

    if (warp >= 4) {
        // ---------------- loaders ----------------
        const int lt = tid - 128;                         // the thread's key (and row of Q)
        unsigned n = 0;
        bool ok = true;
        Fp4Row<D> kx, vx;
        do {
            const int64_t kv0 = ((int64_t)it.b * p.kvs_b + (int64_t)it.h * p.kvs_head) * 2;
            auto row_of = [&](int u) -> int64_t {         // of the thread's key: cache row (4 bits), or byte offset; -1: none
                const int key = it.first_key(u) + lt;
                if (it.is_tree(u)) return key < it.live ? kv0 + (int64_t)key * p.kvs_row * 2 : -1;
                if (key >= it.len) return -1;
                const int64_t row = cache_row(p.c, it.b, it.h, key);
                return FP4 || row < 0 ? row : row * (D * 2);
            };
            int64_t row = row_of(it.u0);
            bool held = false;                            // kx, vx hold unit u's rows
            for (int u = it.u0; u < it.u1; ++u, ++n) {
                const bool tree = it.is_tree(u);
                const uint32_t there = __ballot_sync(kFullMask, row >= 0);
                if constexpr (FP4) {
                    if (!tree && !held) { fp4_row_load<D>(kx, p.c.k, p.c.ks, row); fp4_row_load<D>(vx, p.c.v, p.c.vs, row); }
                } else {
                    sh.key_row[n & 1][lt] = row;
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                }
                if (n > 0) ok = tile_wait(sh, &sh.s_full, (n - 1) & 1);            // the product with the keys before is done
                if (!__all_sync(kFullMask, ok)) { ok = false; break; }
                if (lane == 0) sh.key_bits[n & 1][warp - 4] = there;
                if (u == it.u0) {                         // the item's queries
                    const int m0 = it.mb * kTileBM + lt, r = m0 / p.group, g = m0 - r * p.group;
                    const uint4* src = (const uint4*)(p.q + ((int64_t)it.b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)(it.h * p.group + g) * p.qs_head) * 2);
                    const bool live = r < it.live;
#pragma unroll 4
                    for (int ch = 0; ch < kCh; ++ch) {
                        uint4 x = live ? __ldg(src + ch) : make_uint4(0, 0, 0, 0);
                        if constexpr (FP4) x = order_pairs(x);
                        *(uint4*)(sh.q + tile_off(lt, ch)) = x;
                    }
                }
                const bool more = u + 1 < it.u1;
                int64_t next_row = -1;
                if constexpr (FP4) {
                    const bool ahead = more && !it.is_tree(u + 1);
                    if (more) next_row = row_of(u + 1);
                    if (!tree) {
                        fp4_row_store<D>(kx, sh.k, lt);
                    } else {
#pragma unroll 4
                        for (int ch = 0; ch < kCh; ++ch)
                            *(uint4*)(sh.k + tile_off(lt, ch)) = row >= 0 ? order_pairs(__ldg((const uint4*)(p.k + row) + ch)) : make_uint4(0, 0, 0, 0);
                    }
                    if (ahead) fp4_row_load<D>(kx, p.c.k, p.c.ks, next_row);
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.k_full);
                    if (n > 0) ok = tile_wait(sh, &sh.pv_done, (n - 1) & 1);
                    if (!__all_sync(kFullMask, ok)) { ok = false; break; }
                    if (!tree) {
                        fp4_row_store<D>(vx, sh.v, lt);
                    } else {
#pragma unroll 4
                        for (int ch = 0; ch < kCh; ++ch)
                            *(uint4*)(sh.v + tile_off(lt, ch)) = row >= 0 ? order_pairs(__ldg((const uint4*)(p.v + row) + ch)) : make_uint4(0, 0, 0, 0);
                    }
                    if (ahead) fp4_row_load<D>(vx, p.c.v, p.c.vs, next_row);
                    held = ahead;
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.v_full);
                } else {
                    const unsigned char* kb = tree ? p.k : p.c.k;
                    const unsigned char* vb = tree ? p.v : p.c.v;
                    const int ch = lt % kCh;
#pragma unroll 4
                    for (int i = lt / kCh; i < kUnit; i += 128 / kCh) {
                        const int64_t off = sh.key_row[n & 1][i];
                        cp_async16(smem_u32(sh.k) + tile_off(i, ch), kb + (off < 0 ? 0 : off + ch * 16), off < 0 ? 0u : 16u);
                    }
                    cp_async_commit();
                    if (more) next_row = row_of(u + 1);
                    if (n > 0) ok = tile_wait(sh, &sh.pv_done, (n - 1) & 1);
                    if (!__all_sync(kFullMask, ok)) { ok = false; break; }
#pragma unroll 4
                    for (int i = lt / kCh; i < kUnit; i += 128 / kCh) {
                        const int64_t off = sh.key_row[n & 1][i];
                        cp_async16(smem_u32(sh.v) + tile_off(i, ch), vb + (off < 0 ? 0 : off + ch * 16), off < 0 ? 0u : 16u);
                    }
                    cp_async_commit();
                    cp_async_wait<1>();
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.k_full);
                    cp_async_wait<0>();
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.v_full);
                }
                row = next_row;
            }
        } while (ok && tile_next(it, p));
        cp_async_wait<0>();
    } else {
        // ---------------- softmax and epilogue ----------------
        const uint32_t ts = tm_s + ((uint32_t)(warp * 32) << 16), to = tm_o + ((uint32_t)(warp * 32) << 16);
        // what the 4-bit form leaves to be put right: scores of cached keys times 2^(8 - k_exp), weights times 2^(8 - v_exp)
        const float sc_ctx = FP4 ? p.scale_log2 * exp2i(8 - p.c.k_exp) : p.scale_log2;
        const float up_ctx = FP4 ? (float)(8 - p.c.v_exp) : 0.0f, down_ctx = FP4 ? exp2i(p.c.v_exp - 8) : 1.0f;
        unsigned n = 0;
        bool ok = true;
        // thread 0: the scores of unit number i, once its keys are there
        auto scores = [&](unsigned i) {
            ok = tile_wait(sh, &sh.k_full, i & 1);
            if (!ok) return;
            tc_fence_after();
            // rolled, as all of this kernel's loops that need not be unrolled: code that one warp runs once per unit is otherwise
            // fetched anew from beyond the instruction caches each time
            const uint64_t dq = umma_desc_k_sw128(sh.q, 0), dk = umma_desc_k_sw128(sh.k, 0);
#pragma unroll 1
            for (int kk = 0; kk < D / 16; ++kk) {
                const int at = (kk >> 2) * 1024 + (kk & 3) * 2;
                umma_bf16(tm_s, dq + at, dk + at, tile_idesc(kUnit, 0), kk != 0);
            }
            umma_commit(&sh.s_full);
        };
        if (tid == 0) scores(0);
        __syncwarp();
        do {
            const int m0 = it.mb * kTileBM + tid, M = it.live * p.group;           // at most 2^24
            const bool live = m0 < M;
            const bool warp_live = it.mb * kTileBM + warp * 32 < M;
            const int r = live ? m0 / p.group : 0, hq = it.h * p.group + (m0 - r * p.group);
            const int dr = attn_depth(p, it.b, r);
            float m = -INFINITY, l = 0.0f;
            for (int u = it.u0; u < it.u1; ++u, ++n) {
                ok = __all_sync(kFullMask, ok && tile_wait(sh, &sh.s_full, n & 1));
                if (!ok) break;
                tc_fence_after();
                if (warp_live) {
                    const bool tree = it.is_tree(u);
                    const float sc = tree ? p.scale_log2 : sc_ctx, up = tree ? 0.0f : up_ctx, down = tree ? 1.0f : down_ctx;
                    uint32_t see[4];
                    unit_bits(p, tree, it.b, it.len, it.live, r, dr, it.first_key(u), see);
                    bool all = true;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        see[i] &= sh.key_bits[n & 1][i];
                        all = all && see[i] == ~0u;
                    }
                    const bool masked = !__all_sync(kFullMask, all || !live);
                    const float mx = tile_max(ts, masked, see) * sc;
                    if (__any_sync(kFullMask, mx > m + kTileSlack || (m == -INFINITY && mx > m))) {
                        const float mn = fmaxf(m, mx), a = m == -INFINITY ? 0.0f : ex2(m - mn);
                        m = mn;
                        l *= a;
                        if (u > it.u0) {
#pragma unroll 1
                            for (int c = 0; c < D / 16; ++c) {
                                uint32_t o[16];
                                tmem_ld16(to + c * 16, o);
                                tmem_ld_wait16(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
                                tmem_st16(to + c * 16, o);
                            }
                        }
                    }
                    l = fmaf(tile_weights(ts, masked, see, sc, up - (m == -INFINITY ? 0.0f : m)), down, l);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_ready);
                if (tid == 0) {                           // O += P V, then the next unit's scores in P's place
                    ok = tile_wait(sh, &sh.p_ready, n & 1) && tile_wait(sh, &sh.v_full, n & 1);
                    if (ok) {
                        tc_fence_after();
                        const uint64_t dv = umma_desc_mn_sw128(sh.v, 0, 16384);
                        const bool more = u > it.u0;
#pragma unroll 1
                        for (int kk = 0; kk < kUnit / 16; ++kk)
                            umma_bf16_ts(tm_o, tm_s + kk * 8, dv + kk * 128, tile_idesc(D, 1), (more || kk != 0) ? 1u : 0u);
                        umma_commit(&sh.pv_done);
                        if (u + 1 < it.u1 || it.left > 0) {
                            ok = tile_wait(sh, &sh.pv_done, n & 1);
                            if (ok) scores(n + 1);
                        }
                    }
                }
                __syncwarp();                             // the warp's other lanes wait here: polling, they would hold lane 0 up
            }
            if (!ok) break;
            // ---- epilogue ----
            ok = __all_sync(kFullMask, ok && tile_wait(sh, &sh.pv_done, (n - 1) & 1));
            if (!ok) break;
            tc_fence_after();
            if (warp_live && tile_finish<D, FP4>(w, it, to, live, r, hq, m, l)) sh.odd = 1;
            tc_fence_before();
        } while (tile_next(it, p));
        if (tid == 0) {                                   // no product is in flight when the tensor memory is given back
            umma_commit(&sh.drained);
            for (int i = 0; i < (1 << 20) && !mbar_try_wait(&sh.drained, 0); ++i) {}
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tm_s, kTileTmemCols);
    }
    if (tid == 0) w.odd[blockIdx.x] = (int)sh.odd;
    if (tid == 0 && sh.error && p.status)
        for (int b = 0; b < p.c.batch; ++b) atomicOr(&p.status[b], CADD_STATUS_INTERNAL_TIMEOUT);
}

}  // namespace cadd
