// Paged key/value cache (cadd_cache in cadd.h): addressing, the 4-bit form, and the kernels that write rows to it
// (cadd_cache_append) and read them back (cadd_cache_read).
//
// The 4-bit form stores 16 neighbouring elements of a row as e2m1 codes and one e4m3 scale.  What it stands for,
// code * scale, has at most 2 + 4 significant bits and lies in [2^-10, 2688], so bf16 (8 bits) holds it exactly: the
// attention kernels multiply exact numbers.
#pragma once
#include "common.cuh"
#include "fp4.cuh"

namespace cadd {

struct CacheView {
    unsigned char *k, *v;                  // rows of row_bytes
    unsigned char *ks, *vs;                // FP4: rows of head_dim / 16 scale bytes
    const int32_t* block_table;
    const int32_t* length;
    int64_t stride_page, stride_head, stride_slot;
    int64_t n_pages;
    int batch, heads, head_dim, page_shift, max_pages;
    int fp4;
    int k_exp, v_exp;
    int row_bytes;
};

__device__ __forceinline__ int cache_capacity(const CacheView& c) { return c.max_pages << c.page_shift; }
__device__ __forceinline__ int cache_clamped(const CacheView& c, int n) { return min(max(n, 0), cache_capacity(c)); }
__device__ __forceinline__ int cache_length(const CacheView& c, int b) { return cache_clamped(c, c.length[b]); }

// Row number of place `pos` (already inside the capacity) of request b in head h; -1 where block_table points outside the pool.
__device__ __forceinline__ int64_t cache_row(const CacheView& c, int b, int h, int pos) {
    const int page = c.block_table[(int64_t)b * c.max_pages + (pos >> c.page_shift)];
    if ((unsigned)page >= (uint64_t)c.n_pages) return -1;
    return (int64_t)page * c.stride_page + (int64_t)h * c.stride_head + (int64_t)(pos & ((1 << c.page_shift) - 1)) * c.stride_slot;
}

// Whole CTA: is any table entry of the places [from, to) outside the pool?  (Barrier inside; every thread gets the answer.)
__device__ __forceinline__ int cache_bad_pages(const CacheView& c, int b, int from, int to) {
    int bad = 0;
    if (to > from)
        for (int i = (from >> c.page_shift) + (int)threadIdx.x; i <= (to - 1) >> c.page_shift; i += (int)blockDim.x)
            bad |= (unsigned)c.block_table[(int64_t)b * c.max_pages + i] >= (uint64_t)c.n_pages;
    return __syncthreads_or(bad);
}

// Which rows a round's calls take: with a path row 0 and then path[0..], else rows 0, 1, ...
struct RowList {
    const int32_t *n_rows, *path, *path_len;
    int R, L;
};
__device__ __forceinline__ int row_count(const RowList& r, int b, int* out_of_range) {
    const int hi = r.path ? r.L : r.R;
    const int n = r.path ? r.path_len[b] : (r.n_rows ? r.n_rows[b] : r.R);
    const int m = min(max(n, 0), hi);
    *out_of_range = n != m;
    return r.path ? m + 1 : m;
}
// Source row of list entry i, -1 if the path names none.
__device__ __forceinline__ int row_at(const RowList& r, int b, int i) {
    if (!r.path) return i;
    const int j = i == 0 ? 0 : r.path[(int64_t)b * r.L + i - 1];
    return (unsigned)j < (unsigned)r.R ? j : -1;
}

// Item `it` of [rows][heads][head_dim / 16], head_dim / 16 being 4 or 8; a 64-bit division is only taken where it is needed.
__device__ __forceinline__ void cache_item(int64_t it, int64_t items, const CacheView& c, int& i, int& h, int& q) {
    const int shift = c.head_dim == 128 ? 3 : 2;
    q = (int)it & ((1 << shift) - 1);
    const int64_t rest = it >> shift;
    i = items <= 0xffffffffll ? (int)((unsigned)rest / (unsigned)c.heads) : (int)(rest / c.heads);
    h = (int)(rest - (int64_t)i * c.heads);
}

struct AppendParams {
    CacheView c;
    const unsigned char *k, *v;
    int64_t stride_b, stride_row, stride_head;           // elements
    RowList rows;
    int32_t* new_length;                                 // NULL: written by a kernel of its own (it is c.length)
    int32_t* status;
    int ctas_per_request;
};
constexpr int kCopyThreads = 256;

// Rows into the cache: one thread moves 16 elements of one row of one head, of k and of v.  Prompts of 37k rows in all, 8 heads of
// 128, to 4 bits and read back take 93 us together on a B200, 0.61 of the copy rate: writing 48 (issue active 74 % of the time, by
// the quotients and conversions), reading 45 (16 issue slots of waiting for loads to each instruction).  A round's few rows are
// bound by the launch.
// The first CTA of a request also writes its new length and status.
template <bool FP4>
__global__ void __launch_bounds__(kCopyThreads) cache_append_kernel(const AppendParams p) {
    const int b = blockIdx.x / p.ctas_per_request, part = blockIdx.x - b * p.ctas_per_request;
    const CacheView& c = p.c;
    int clamped = 0;
    const int base = cache_length(c, b), want = row_count(p.rows, b, &clamped);
    const int n = min(want, cache_capacity(c) - base);
    const int blocks = c.head_dim >> 4, per_row = c.heads * blocks;
    const int64_t items = (int64_t)n * per_row;
    for (int64_t it = (int64_t)part * kCopyThreads + threadIdx.x; it < items; it += (int64_t)p.ctas_per_request * kCopyThreads) {
        int i, h, q;
        cache_item(it, items, c, i, h, q);
        const int src = row_at(p.rows, b, i);
        const int64_t row = cache_row(c, b, h, base + i);
        if (src < 0 || row < 0) continue;
        const int64_t at = ((int64_t)b * p.stride_b + (int64_t)src * p.stride_row + (int64_t)h * p.stride_head + q * 16) * 2;
        uint4 w[4];
        w[0] = __ldg((const uint4*)(p.k + at)); w[1] = __ldg((const uint4*)(p.k + at) + 1);
        w[2] = __ldg((const uint4*)(p.v + at)); w[3] = __ldg((const uint4*)(p.v + at) + 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            unsigned char* pool = s ? c.v : c.k;
            if constexpr (!FP4) {
                uint4* dst = (uint4*)(pool + row * c.row_bytes + q * 32);
                dst[0] = w[2 * s];
                dst[1] = w[2 * s + 1];
            } else {
                uint32_t scale;
                const uint2 codes = fp4_encode(w[2 * s], w[2 * s + 1], exp2i(s ? c.v_exp : c.k_exp), scale);
                *(uint2*)(pool + row * c.row_bytes + q * 8) = codes;
                (s ? c.vs : c.ks)[row * blocks + q] = (unsigned char)scale;
            }
        }
    }
    if (part) return;
    if (threadIdx.x == 0 && p.new_length) p.new_length[b] = base + n;
    if (!p.status) return;
    int bad = cache_bad_pages(c, b, base, base + n) ? CADD_STATUS_BAD_PAGE : 0, path = 0;
    for (int i = threadIdx.x; i < want; i += kCopyThreads) path |= row_at(p.rows, b, i) < 0;
    path = __syncthreads_or(path);
    if (threadIdx.x == 0)
        p.status[b] = bad | (path ? CADD_STATUS_BAD_PATH : 0) | (n < want ? CADD_STATUS_CACHE_FULL : 0) |
                      ((clamped || c.length[b] != base) ? CADD_STATUS_BAD_LENGTH : 0);
}

// new_length is the array the other kernel reads: written once that kernel is done.
__global__ void cache_advance_kernel(const CacheView c, RowList rows, int32_t* new_length) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= c.batch) return;
    int clamped;
    const int base = cache_length(c, b);
    new_length[b] = base + min(row_count(rows, b, &clamped), cache_capacity(c) - base);
}

struct ReadParams {
    CacheView c;
    unsigned char *k, *v;
    int64_t stride_b, stride_row, stride_head;
    const int32_t *start, *count;
    int n_max;
    int32_t* status;
    int ctas_per_request;
};

// Rows out of the cache, 16 elements of k and v a thread.
template <bool FP4>
__global__ void __launch_bounds__(kCopyThreads) cache_read_kernel(const ReadParams p) {
    const int b = blockIdx.x / p.ctas_per_request, part = blockIdx.x - b * p.ctas_per_request;
    const CacheView& c = p.c;
    const int len = cache_length(c, b);
    const int s0 = p.start ? p.start[b] : 0, from = min(max(s0, 0), len);
    const int room = min(p.n_max, len - from), asked = p.count ? p.count[b] : room, n = min(max(asked, 0), room);
    const int blocks = c.head_dim >> 4, per_row = c.heads * blocks;
    const int64_t items = (int64_t)n * per_row;
    for (int64_t it = (int64_t)part * kCopyThreads + threadIdx.x; it < items; it += (int64_t)p.ctas_per_request * kCopyThreads) {
        int i, h, q;
        cache_item(it, items, c, i, h, q);
        const int64_t row = cache_row(c, b, h, from + i);
        if (row < 0) continue;
        const int64_t at = ((int64_t)b * p.stride_b + (int64_t)i * p.stride_row + (int64_t)h * p.stride_head + q * 16) * 2;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const unsigned char* pool = s ? c.v : c.k;
            uint4* dst = (uint4*)((s ? p.v : p.k) + at);
            if constexpr (!FP4) {
                const uint4* src = (const uint4*)(pool + row * c.row_bytes + q * 32);
                dst[0] = src[0];
                dst[1] = src[1];
            } else {
                const uint2 codes = *(const uint2*)(pool + row * c.row_bytes + q * 8);
                uint32_t f0, f1;
                fp4_half_scales((s ? c.vs : c.ks)[row * blocks + q], f0, f1);
                const float down = exp2i(-(s ? c.v_exp : c.k_exp));
                const uint4 lo = fp4_half_values(codes.x, f0), hi = fp4_half_values(codes.y, f0);
                const uint32_t in[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 two = __half22float2(*reinterpret_cast<const __half2*>(&in[j]));
                    w[j] = pack_bf16(two.x * down, two.y * down);
                }
                dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
    if (part || !p.status) return;
    const int bad = cache_bad_pages(c, b, from, from + n) ? CADD_STATUS_BAD_PAGE : 0;
    if (threadIdx.x == 0)
        p.status[b] = bad | ((c.length[b] != len || s0 != from || n < min(asked, p.n_max) || asked < 0) ? CADD_STATUS_BAD_LENGTH : 0);
}

}  // namespace cadd
