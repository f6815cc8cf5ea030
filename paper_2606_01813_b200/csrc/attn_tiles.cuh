// Tree attention on the 5th-generation tensor cores: blocks of 128 rows, units of 64 keys.
//
// For each unit S = Q K^T goes to tensor memory (M 128 = rows, N 64 = keys, contraction over the head's elements), the
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
// 32-bit word holds elements 0..7 of a group; taking the same nibble of its halves pairs elements (j, j + 4), so keys,
// values and queries stand in shared memory in the order 0 4 1 5 2 6 3 7 within each eight (the product with the keys
// does not mind, the values' order is undone when O is written).  (The fp16 form of fp4.cuh takes fewer logic instructions, but
// the tree's own rows are bf16 and one product has one type: with fp16 queries for cached units and bf16 ones for the
// tree's, the larger kernel spilled and came to 1055 us where this one took 887.)
//
// Keys, values and scores are double-buffered: the scores of unit n + 1 are formed and the values of unit n - 1 multiplied while
// the softmax works on unit n.  (With one buffer of 128 keys the three followed one another, and a unit of 128 keys cost 7000
// cycles of a CTA; measured on a B200.)  Two CTAs share an SM.  288 threads:
//   warps 0-3  softmax and epilogue, a row (tensor-memory lane) per thread;
//   warps 4-5  keys, warps 6-7 values: into the 128-byte swizzle, 32 keys a warp, by asynchronous 16-byte copies (bf16), or
//              a row a thread through registers, one unit ahead (4 bits); all four load the item's queries;
//   warp 8     issues the products and owns the tensor memory (256 columns: S/P 2 x 64, O up to 128).
//
// What bounds it (a thousand-node tree over up to 16k tokens in 4 bits, 850 us, 630 TFLOP/s, 0.38 of the measured rate): no unit
// alone.  The shared-memory pipe, which serves the loaders, tensor memory's reads and writes and the products' operands, is
// at 61 % without the operands, logic at 48 %, issue at 57 %, the tensor pipe at 34 %.  Per unit and CTA that is 256 + 128
// cycles of tensor memory, 256 of stores, 512 of operands (the queries are read again for every 64 keys) and some 300 others.
// Two blocks of rows to a CTA with 128 keys a unit would halve most of that; built, it was bound by the longer way from
// softmax to products and back (3050 cycles for 128 rows x 128 keys against 2900 here) and was not kept, nor were two
// threads to a row (929 us).  96 registers a thread, 20 (4 bits) and 28 bytes spilled.
// At head dimension 64 (a prompt chunk of 2000 rows over up to 6001 places, 12 heads, bf16: 175 us, 0.22 of the measured rate)
// there are half as many products to the same exponentials: issue 53 %, exponential unit 40 %, logic 38 %, tensor pipe 21 %.
// Every wait has an iteration limit; a role that gives up sets an error word and all leave.
//
// A product of a weight 0 with a non-finite value that the row does not see would be NaN.  A range that meets a non-finite result
// says so, and the join does such rows once more, key by key over the keys that they see; that costs nothing otherwise.
#pragma once
#include "attn_plan.cuh"
#include "tcgen05.cuh"
#include "fp4.cuh"

namespace cadd {

constexpr int kTileBM = 128;
constexpr int kTileThreads = 288;
constexpr int kTileTmemCols = 256;
constexpr int kTileWaitLimit = 1 << 19, kTileTestWaitLimit = 1 << 12;     // tries of a wait, 3.9 us each (measured): 2 s, 16 ms
constexpr float kTileSlack = 40.0f;                      // log2 of how far weights may exceed 1 before m is raised

template <int D> struct alignas(1024) TileShared {
    unsigned char q[kTileBM * D * 2];                    // D/64 sub-tiles of 128 rows x 128 bytes
    unsigned char k[2][kUnit * D * 2];                   // D/64 sub-tiles of 64 rows x 128 bytes
    unsigned char v[2][kUnit * D * 2];
    uint64_t q_full, k_full[2], v_full[2], s_full[2], p_ready[2], pv_done[2], drained;
    PlanShared plan;
    WorkIter<kTileBM> it[kTileThreads / 32];             // a walk per warp: here, not in registers, which are scarce
    uint32_t key_bits[4][2];                             // keys of the unit that exist
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
__device__ __forceinline__ bool tile_wait(Shared& sh, uint64_t* bar, unsigned parity, int limit) {
    for (int it = 0; it < limit; ++it) {
        if (tile_try(bar, parity)) return true;
        if (*(volatile uint32_t*)&sh.error) return false;
    }
    sh.error = 1;
    return false;
}
// The products, issued by the lane with `one` set of a warp that runs them together: the operands stay in uniform registers.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void umma_ss(uint32_t one, uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %0, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%1], %2, %3, %4, p;\n\t}"
                 ::"r"(one), "r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t one, uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %0, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], %3, %4, p;\n\t}"
                 ::"r"(one), "r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_commit_one(uint32_t one, uint64_t* bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %0, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}"
                 ::"r"(one), "r"(smem_u32(bar)) : "memory");
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

// Shared-memory offset of 16-byte chunk `ch` of row `row` in a tile of ROWS rows of bf16 elements (sub-tiles of 64 elements).
template <int ROWS>
__device__ __forceinline__ uint32_t tile_off(int row, int ch) {
    return (uint32_t)((ch >> 3) * (ROWS * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
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
__device__ __forceinline__ void fp4_row_store(const Fp4Row<D>& x, unsigned char* tile, int row) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {                   // 32 elements: a 16-byte word of codes, two scales
        uint32_t f0, f1;
        fp4_unit_scales((x.s[i >> 1] >> ((i & 1) * 16)) & 0xffffu, f0, f1);
        *(uint4*)(tile + tile_off<kUnit>(row, i * 4 + 0)) = fp4_unit_values(x.w[i].x, f0);
        *(uint4*)(tile + tile_off<kUnit>(row, i * 4 + 1)) = fp4_unit_values(x.w[i].y, f0);
        *(uint4*)(tile + tile_off<kUnit>(row, i * 4 + 2)) = fp4_unit_values(x.w[i].z, f1);
        *(uint4*)(tile + tile_off<kUnit>(row, i * 4 + 3)) = fp4_unit_values(x.w[i].w, f1);
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
__device__ __forceinline__ void tmem_ld_wait8(uint32_t (&r)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]) :: "memory");
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
// 2^(s sc + off) of 16 scores, packed and written to tensor memory.
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
    float* rec = w.records + ((int64_t)blockIdx.x * 2 + (it.u0 > 0 ? 0 : 1)) * record_floats<kTileBM, D>();
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
            for (int i = 0; i < 16; i += 4)
                *(float4*)(rec + tid * D + c * 16 + i) = make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
        }
    }
    if (live && !whole) { rec[kTileBM * D + tid] = m; rec[kTileBM * (D + 1) + tid] = l; }
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
        mbar_init(&sh.q_full, 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.k_full[i], p.test_drop && i == min(it.u1 - it.u0 - 1, 1) ? 3 : 2);       // test hook: an arrival that never comes
            mbar_init(&sh.v_full[i], 2);
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_ready[i], 4);
            mbar_init(&sh.pv_done[i], 1);
        }
        mbar_init(&sh.drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(&sh.tmem_base, kTileTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm_s = *(volatile uint32_t*)&sh.tmem_base, tm_o = tm_s + 2 * kUnit;
    constexpr int kCh = D / 8;                            // 16-byte chunks of a bf16 row

    // Units are numbered through the CTA's whole range: unit n uses buffer n & 1, in its (n >> 1)-th turn.
    if (warp == 8) {
        // ---------------- products ----------------
        const uint32_t one = elect_one();
        unsigned n = 0, items = 0;
        bool ok = true;
        auto output = [&](unsigned i, bool first) {       // O (+)= P V of unit i
            ok = tile_wait(sh, &sh.p_ready[i & 1], (i >> 1) & 1, p.wait_limit) && tile_wait(sh, &sh.v_full[i & 1], (i >> 1) & 1, p.wait_limit);
            if (!(ok = __all_sync(kFullMask, ok))) return;
            tc_fence_after();
            const uint64_t dv = umma_desc_mn_sw128(sh.v[i & 1], 0, kUnit * 128);
            const uint32_t pm = tm_s + (i & 1) * kUnit;
#pragma unroll
            for (int kk = 0; kk < kUnit / 16; ++kk) umma_ts(one, tm_o, pm + kk * 8, dv + kk * 128, tile_idesc(D, 1), (!first || kk != 0) ? 1u : 0u);
            umma_commit_one(one, &sh.pv_done[i & 1]);
        };
        do {
            if (!(ok = __all_sync(kFullMask, tile_wait(sh, &sh.q_full, items & 1, p.wait_limit)))) break;
            ++items;
            // The scores of a unit take the place of the weights of the unit two before, right behind the product that reads those:
            // products of one kind and accumulator type run in the order in which they are issued.
            const unsigned first = n, end = n + (it.u1 - it.u0);
            for (; n < end + 2; ++n) {
                if (n >= first + 2) output(n - 2, n == first + 2);
                if (!ok) break;
                if (n < end) {
                    ok = __all_sync(kFullMask, tile_wait(sh, &sh.k_full[n & 1], (n >> 1) & 1, p.wait_limit));
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dq = umma_desc_k_sw128(sh.q, 0), dk = umma_desc_k_sw128(sh.k[n & 1], 0);
                    const uint32_t sm = tm_s + (n & 1) * kUnit;
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        umma_ss(one, sm, dq + (kk >> 2) * 1024 + (kk & 3) * 2, dk + (kk >> 2) * (kUnit * 8) + (kk & 3) * 2, tile_idesc(kUnit, 0), kk != 0);
                    umma_commit_one(one, &sh.s_full[n & 1]);
                }
            }
            n = end;
        } while (ok && tile_next(it, p));
        umma_commit_one(one, &sh.drained);                // no product is in flight when the tensor memory is given back
        for (int i = 0; i < (1 << 20) && !mbar_try_wait(&sh.drained, 0); ++i) {}
    } else if (warp >= 4) {
        // ---------------- loaders ----------------
        const bool values = warp >= 6;
        const int kt = (warp & 1) * 32 + lane;            // the thread's key of a unit
        const unsigned char* pool = values ? p.c.v : p.c.k;
        const unsigned char* scales = values ? p.c.vs : p.c.ks;
        const unsigned char* own = values ? p.v : p.k;    // the tree's rows
        uint64_t* full = values ? sh.v_full : sh.k_full;
        uint64_t* freed = values ? sh.pv_done : sh.s_full;                         // the product that reads a buffer is done
        unsigned n = 0;
        bool ok = true;
        Fp4Row<D> x;
        do {
            const int64_t kv0 = ((int64_t)it.b * p.kvs_b + (int64_t)it.h * p.kvs_head) * 2;
            auto row_of = [&](int u) -> int64_t {         // of the thread's key: cache row (4 bits), or byte offset; -1: none
                const int key = it.first_key(u) + kt;
                if (it.is_tree(u)) return key < it.live ? kv0 + (int64_t)key * p.kvs_row * 2 : -1;
                if (key >= it.len) return -1;
                const int64_t row = cache_row(p.c, it.b, it.h, key);
                return FP4 || row < 0 ? row : row * (D * 2);
            };
            int64_t row = row_of(it.u0);
            if constexpr (FP4) { if (!it.is_tree(it.u0)) fp4_row_load<D>(x, pool, scales, row); }
            {   // the item's queries, once the last product with those before is done
                const int m0 = it.mb * kTileBM + (tid - 128), r = m0 / p.group, g = m0 - r * p.group;
                const uint4* src = (const uint4*)(p.q + ((int64_t)it.b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)(it.h * p.group + g) * p.qs_head) * 2);
                const bool live = r < it.live;
                if (n > 0) ok = tile_wait(sh, &sh.s_full[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_limit);
                if (!(ok = __all_sync(kFullMask, ok))) break;
#pragma unroll 4
                for (int ch = 0; ch < kCh; ++ch) {
                    uint4 t = live ? __ldg(src + ch) : make_uint4(0, 0, 0, 0);
                    if constexpr (FP4) t = order_pairs(t);
                    *(uint4*)(sh.q + tile_off<kTileBM>(tid - 128, ch)) = t;
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.q_full);
            }
            for (int u = it.u0; u < it.u1; ++u, ++n) {
                const bool tree = it.is_tree(u), more = u + 1 < it.u1;
                unsigned char* tile = values ? sh.v[n & 1] : sh.k[n & 1];
                const uint32_t there = __ballot_sync(kFullMask, row >= 0);
                if (n >= 2) ok = tile_wait(sh, &freed[n & 1], ((n >> 1) - 1) & 1, p.wait_limit);
                if (!(ok = __all_sync(kFullMask, ok))) break;
                if (!values && lane == 0) sh.key_bits[n & 3][warp & 1] = there;
                int64_t next_row = -1;
                if constexpr (FP4) {
                    if (!tree) {
                        fp4_row_store<D>(x, tile, kt);
                    } else {
#pragma unroll 4
                        for (int ch = 0; ch < kCh; ++ch)
                            *(uint4*)(tile + tile_off<kUnit>(kt, ch)) = row >= 0 ? order_pairs(__ldg((const uint4*)(own + row) + ch)) : make_uint4(0, 0, 0, 0);
                    }
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&full[n & 1]);
                    if (more) {
                        next_row = row_of(u + 1);
                        if (!it.is_tree(u + 1)) fp4_row_load<D>(x, pool, scales, next_row);
                    }
                } else {
                    const unsigned char* base = tree ? own : pool;
                    const int ch = lane % kCh;
#pragma unroll 4
                    for (int i = lane / kCh; i < 32; i += 32 / kCh) {
                        const int64_t off = __shfl_sync(kFullMask, row, i);
                        cp_async16(smem_u32(tile) + tile_off<kUnit>((warp & 1) * 32 + i, ch), base + (off < 0 ? 0 : off + ch * 16), off < 0 ? 0u : 16u);
                    }
                    cp_async_commit();
                    if (u > it.u0) {                      // unit n - 1 has landed
                        cp_async_wait<1>();
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&full[(n - 1) & 1]);
                    }
                    if (more) next_row = row_of(u + 1);
                }
                row = next_row;
            }
            if constexpr (!FP4) {                         // the item's last unit
                cp_async_wait<0>();
                fence_async_shared();
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&full[(n - 1) & 1]);
            }
        } while (ok && tile_next(it, p));
    } else {
        // ---------------- softmax and epilogue ----------------
        const uint32_t to = tm_o + ((uint32_t)(warp * 32) << 16);
        // what the 4-bit form leaves to be put right: scores of cached keys times 2^(8 - k_exp), weights times 2^(8 - v_exp)
        const float sc_ctx = FP4 ? p.scale_log2 * exp2i(8 - p.c.k_exp) : p.scale_log2;
        const float up_ctx = FP4 ? (float)(8 - p.c.v_exp) : 0.0f, down_ctx = FP4 ? exp2i(p.c.v_exp - 8) : 1.0f;
        unsigned n = 0;
        bool ok = true;
        do {
            const int m0 = it.mb * kTileBM + tid, M = it.live * p.group;           // at most 2^24
            const bool live = m0 < M;
            const bool warp_live = it.mb * kTileBM + warp * 32 < M;
            const int r = live ? m0 / p.group : 0, hq = it.h * p.group + (m0 - r * p.group);
            const int dr = attn_depth(p, it.b, r);
            float m = -INFINITY, l = 0.0f;
            for (int u = it.u0; u < it.u1; ++u, ++n) {
                ok = __all_sync(kFullMask, tile_wait(sh, &sh.s_full[n & 1], (n >> 1) & 1, p.wait_limit));
                if (!ok) break;
                tc_fence_after();
                if (warp_live) {
                    const uint32_t ts = tm_s + (n & 1) * kUnit + ((uint32_t)(warp * 32) << 16);
                    uint32_t s[4][16];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_ld16(ts + j * 16, s[j]);
                    const bool tree = it.is_tree(u);
                    uint32_t see[2] = {sh.key_bits[n & 3][0], sh.key_bits[n & 3][1]};
                    bool masked = false;                  // a whole cached unit without a window is seen by all
                    if (tree || p.window > 0 || (see[0] & see[1]) != ~0u) {
                        uint32_t bits[2];
                        unit_bits(p, tree, it.b, it.len, it.live, r, dr, it.first_key(u), bits);
                        see[0] &= bits[0];
                        see[1] &= bits[1];
                        masked = !__all_sync(kFullMask, (see[0] & see[1]) == ~0u || !live);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_ld_wait16(s[j]);
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < kUnit; ++i) s[i >> 4][i & 15] = (see[i >> 5] >> (i & 31)) & 1u ? s[i >> 4][i & 15] : 0xff800000u;
                    }
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < kUnit; i += 2) mx4[(i >> 1) & 3] = max3(mx4[(i >> 1) & 3], __uint_as_float(s[i >> 4][i & 15]), __uint_as_float(s[i >> 4][(i & 15) + 1]));
                    const float sc = tree ? p.scale_log2 : sc_ctx;
                    const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * sc;
                    if (__any_sync(kFullMask, mx > m + kTileSlack || (m == -INFINITY && mx > m))) {
                        const float mn = fmaxf(m, mx), a = m == -INFINITY ? 0.0f : ex2(m - mn);
                        m = mn;
                        l *= a;
                        if (u > it.u0) {                  // the product before must be done with O
                            ok = __all_sync(kFullMask, tile_wait(sh, &sh.pv_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_limit));
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 8; ++c) {
                                uint32_t o[8];
                                tmem_ld8(to + c * 8, o);
                                tmem_ld_wait8(o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
                                tmem_st8(to + c * 8, o);
                            }
                        }
                    }
                    const float off = (tree ? 0.0f : up_ctx) - (m == -INFINITY ? 0.0f : m);
                    const uint64_t sc2 = pack2(sc, sc), off2 = pack2(off, off);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j) weights_of(s[j], sc2, off2, sum, ts + j * 8);
                    float sa, sb;
                    unpack2(add2(sum[0], sum[1]), sa, sb);
                    l = fmaf(sa + sb, tree ? 1.0f : down_ctx, l);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_ready[n & 1]);
            }
            if (!ok) break;
            // ---- epilogue ----
            ok = __all_sync(kFullMask, tile_wait(sh, &sh.pv_done[(n - 1) & 1], ((n - 1) >> 1) & 1, p.wait_limit));
            if (!ok) break;
            tc_fence_after();
            if (warp_live && tile_finish<D, FP4>(w, it, to, live, r, hq, m, l)) sh.odd = 1;
            tc_fence_before();
        } while (tile_next(it, p));
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tm_s, kTileTmemCols);
    }
    if (tid == 0) w.odd[blockIdx.x] = (sh.odd ? kRangeOdd : 0) | (sh.error ? kRangeTimedOut : 0);
}

}  // namespace cadd
