// Warp-level products (16 rows x 8 keys x 16 elements) whose key operand comes from the cache's rows straight into registers.
#pragma once
#include "cache.cuh"

namespace cadd {

template <bool HALF>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A truth value as a type, for loops that exist once for either value.
template <bool B> struct Flag { static constexpr bool value = B; };

template <int D, bool FP4> struct WKeys;                 // eight keys' rows as a lane holds them
template <int D> struct WKeys<D, true> { uint32_t w[D / 32]; uint32_t s; };
template <int D> struct WKeys<D, false> { uint4 w[D / 32]; };

template <int D, bool FP4>
__device__ __forceinline__ void wkeys_load(WKeys<D, FP4>& x, const CacheView& c, int64_t row, int t) {
    if constexpr (FP4) {
        x.s = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x.w[i] = 0;
        if (row >= 0) {
            if constexpr (D == 128) {
                const uint4 v = __ldg((const uint4*)(c.k + row * (D / 2)) + t);
                x.w[0] = v.x; x.w[1] = v.y; x.w[2] = v.z; x.w[3] = v.w;
                x.s = __ldg((const unsigned short*)(c.ks + row * (D / 16)) + t);
            } else {
                const uint2 v = __ldg((const uint2*)(c.k + row * (D / 2)) + t);
                x.w[0] = v.x; x.w[1] = v.y;
                x.s = __ldg(c.ks + row * (D / 16) + t);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x.w[i] = row >= 0 ? __ldg((const uint4*)(c.k + row * (D * 2)) + i * 4 + t) : make_uint4(0, 0, 0, 0);
    }
}
// Word m of lane t holds chunk t * W + m (4 bits) or 4 m + t (bf16) of its key's row, W = D / 32; rows keep that chunk in slot
// 4 m + t, so that a key's four lanes read neighbouring slots.
template <int D, bool FP4> __device__ __forceinline__ int wkeys_slot(int chunk) { return FP4 ? (chunk % (D / 32)) * 4 + chunk / (D / 32) : chunk; }

// Rows of the lane's four keys k0 + 8 j + g; pages of 32 slots and more hold 32 aligned keys next to one another: one look-up.
__device__ __forceinline__ void wkeys_rows(const CacheView& c, int b, int h, int k0, int g, int end, int64_t (&row)[4]) {
    if (c.page_shift >= 5) {
        const int64_t first = k0 < end ? cache_row(c, b, h, k0) : -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) row[j] = first >= 0 && k0 + j * 8 + g < end ? first + (int64_t)(j * 8 + g) * c.stride_slot : -1;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) row[j] = k0 + j * 8 + g < end ? cache_row(c, b, h, k0 + j * 8 + g) : -1;
    }
}

// The same in two steps: table entries, and, a step later when those have come, rows.  (The weights kernel gains by it, 245 -> 234 us;
// the few-rows kernel, short of registers, loses: 170 -> 203 us for 16 tokens over up to 32k.)
__device__ __forceinline__ void wkeys_pages(const CacheView& c, int b, int k0, int g, int end, int (&page)[4]) {
    const int32_t* table = c.block_table + (int64_t)b * c.max_pages;
    if (c.page_shift >= 5) {
        page[0] = k0 < end ? table[k0 >> c.page_shift] : -1;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) page[j] = k0 + j * 8 + g < end ? table[(k0 + j * 8 + g) >> c.page_shift] : -1;
    }
}
__device__ __forceinline__ void wkeys_rows(const CacheView& c, int h, int k0, int g, int end, const int (&page)[4], int64_t (&row)[4]) {
    const int slots = (1 << c.page_shift) - 1;
    if (c.page_shift >= 5) {
        int64_t first = -1;
        if ((unsigned)page[0] < (uint64_t)c.n_pages)
            first = (int64_t)page[0] * c.stride_page + (int64_t)h * c.stride_head + (int64_t)(k0 & slots) * c.stride_slot;
#pragma unroll
        for (int j = 0; j < 4; ++j) row[j] = first >= 0 && k0 + j * 8 + g < end ? first + (int64_t)(j * 8 + g) * c.stride_slot : -1;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            row[j] = (unsigned)page[j] < (uint64_t)c.n_pages
                         ? (int64_t)page[j] * c.stride_page + (int64_t)h * c.stride_head + (int64_t)((k0 + j * 8 + g) & slots) * c.stride_slot : -1;
    }
}

}  // namespace cadd
