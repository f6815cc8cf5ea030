// What decides which cached places stay: the weight that accepted rows spend on them (cadd_cache_weights), and the choice
// of the heaviest with the copy of their rows (cadd_cache_evict).
#pragma once
#include "cache.cuh"
#include "tree_attention.cuh"

namespace cadd {

struct WeightsParams {
    CacheView c;
    const unsigned char* q;
    int64_t qs_b, qs_row, qs_head;
    const float* lse;
    RowList rows;
    const int32_t* base_length;
    const float* w_in;
    float* w_out;
    int64_t w_stride;
    int32_t* status;
    int heads_q, group, window, n_sinks;
    float scale_log2;
    int ctas_per_head;
};

// Simplest form: a warp per (request, head, place) goes over the accepted rows and the heads of the group.
template <int D, bool FP4>
__global__ void __launch_bounds__(128) weights_kernel(const WeightsParams p) {
    const int lane = threadIdx.x & 31;
    const int64_t bh = blockIdx.x / p.ctas_per_head;
    const int part = (int)(blockIdx.x - bh * p.ctas_per_head), b = (int)(bh / p.c.heads), h = (int)(bh - (int64_t)b * p.c.heads);
    const int len = cache_length(p.c, b), base = min(max(p.base_length[b], 0), len);
    int clamped;
    const int n = min(row_count(p.rows, b, &clamped), len - base);
    for (int pos = part * 4 + (threadIdx.x >> 5); pos < len; pos += p.ctas_per_head * 4) {
        const int64_t row = cache_row(p.c, b, h, pos);
        float sum = 0.0f;
        if (row >= 0) {
            float k[D / 32], q[D / 32];
            load_row_cache<D, FP4>(p.c, p.c.k, p.c.ks, p.c.k_exp, row, lane, k);
            for (int i = 0; i < n; ++i) {
                const int r = row_at(p.rows, b, i);
                if (r < 0 || pos > base + i || !(p.window == 0 || pos < p.n_sinks || base + i - pos < p.window)) continue;
                for (int g = 0; g < p.group; ++g) {
                    const int hq = h * p.group + g;
                    load_row_bf16<D>(p.q + ((int64_t)b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)hq * p.qs_head) * 2, lane, q);
                    float s = 0.0f;
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) s = fmaf(q[j], k[j], s);
#pragma unroll
                    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFullMask, s, o);
                    const float lse = p.lse[((int64_t)b * p.rows.R + r) * p.heads_q + hq];
                    if (fabsf(lse) != INFINITY) sum += exp2f(s * p.scale_log2 - lse * kLog2e);
                }
            }
        }
        if (lane == 0) {
            const int64_t at = bh * p.w_stride + pos;
            p.w_out[at] = (pos < base ? p.w_in[at] : 0.0f) + sum;
        }
    }
}
__global__ void __launch_bounds__(128) weights_status_kernel(const WeightsParams p) {
    const int b = blockIdx.x, len = cache_length(p.c, b), base = min(max(p.base_length[b], 0), len);
    const int bad = cache_bad_pages(p.c, b, 0, len);
    int clamped, path = 0;
    const int n = row_count(p.rows, b, &clamped);
    for (int i = threadIdx.x; i < n; i += blockDim.x) path |= row_at(p.rows, b, i) < 0;
    path = __syncthreads_or(path);
    if (threadIdx.x == 0)
        p.status[b] = (bad ? CADD_STATUS_BAD_PAGE : 0) | (path ? CADD_STATUS_BAD_PATH : 0) |
                      ((clamped || n > len - base || p.c.length[b] != len || p.base_length[b] != base) ? CADD_STATUS_BAD_LENGTH : 0);
}

struct EvictParams {
    CacheView c;
    const float* weights;
    int64_t w_stride;
    const int32_t* new_table;
    int32_t *new_length, *kept, *status;
    float* w_out;
    int64_t w_out_stride;
    int budget, n_sinks, n_recent, new_max_pages;
};
constexpr int kSelectThreads = 1024;

// Order of weights as integers, NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w == w ? ord32(__float_as_uint(w + 0.0f)) : 0u; }

// Choice: one CTA per (request, head).  Of the n - sinks - recent places between, the `left` heaviest stay.  Four passes over
// the keys' bytes, highest first, count how often each byte value occurs among the keys that share the bytes found so far
// and so find the left-th largest key T and how many places with exactly T stay; a last pass in place order writes
// them down (greater than T, or among the first of the equal ones).
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const EvictParams p) {
    __shared__ unsigned hist[256];
    __shared__ unsigned warp_keep[32], warp_tie[32];
    __shared__ unsigned sh_prefix, sh_left, sh_keep0, sh_tie0;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / p.c.heads), h = (int)(bh - (int64_t)b * p.c.heads);
    const int n = cache_length(p.c, b), keep = min(n, p.budget);
    const float* w = p.weights + bh * p.w_stride;
    int32_t* kept = p.kept + bh * p.budget;
    float* w_out = p.w_out ? p.w_out + bh * p.w_out_stride : nullptr;
    for (int i = keep + tid; i < p.budget; i += kSelectThreads) kept[i] = -1;
    if (h == 0 && p.status) {                                                      // (a uniform branch: barriers inside are met by all)
        int bad = cache_bad_pages(p.c, b, 0, n);
        for (int i = tid; i < (keep + (1 << p.c.page_shift) - 1) >> p.c.page_shift; i += kSelectThreads)
            bad |= (unsigned)p.new_table[(int64_t)b * p.new_max_pages + i] >= (uint64_t)p.c.n_pages;
        bad = __syncthreads_or(bad);
        if (tid == 0) p.status[b] = (bad ? CADD_STATUS_BAD_PAGE : 0) | (p.c.length[b] != n ? CADD_STATUS_BAD_LENGTH : 0);
    }
    if (h == 0 && tid == 0 && p.new_length) p.new_length[b] = keep;
    if (n <= p.budget) {
        for (int i = tid; i < n; i += kSelectThreads) {
            kept[i] = i;
            if (w_out) w_out[i] = w[i];
        }
        return;
    }
    const int lo = p.n_sinks, hi = n - p.n_recent;
    if (tid == 0) { sh_prefix = 0; sh_left = (unsigned)(p.budget - p.n_sinks - p.n_recent); sh_keep0 = 0; sh_tie0 = 0; }
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        const unsigned prefix = sh_prefix;
        for (int i = lo + tid; i < hi; i += kSelectThreads) {
            const unsigned key = weight_key(w[i]);
            if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            unsigned left = sh_left;
            int d = 255;
            for (; d > 0 && hist[d] < left; --d) left -= hist[d];
            sh_left = left;                                                        // of the keys that start like this, how many stay
            sh_prefix = prefix | ((unsigned)d << shift);
        }
        __syncthreads();
    }
    const unsigned T = sh_prefix, ties = sh_left;
    for (int i0 = 0; i0 < n; i0 += kSelectThreads) {
        const int i = i0 + tid;
        const float x = i < n ? w[i] : 0.0f;
        const unsigned key = weight_key(x);
        const bool inner = i >= lo && i < hi;
        const bool tie = inner && key == T;
        const unsigned tb = __ballot_sync(kFullMask, tie);
        if (lane == 0) warp_tie[warp] = __popc(tb);
        __syncthreads();
        unsigned tbase = sh_tie0;
        for (int j = 0; j < warp; ++j) tbase += warp_tie[j];
        const bool stay = i < n && (!inner || key > T || (tie && tbase + __popc(tb & ((1u << lane) - 1u)) < ties));
        const unsigned kb = __ballot_sync(kFullMask, stay);
        if (lane == 0) warp_keep[warp] = __popc(kb);
        __syncthreads();
        unsigned kbase = sh_keep0;
        for (int j = 0; j < warp; ++j) kbase += warp_keep[j];
        const unsigned at = kbase + __popc(kb & ((1u << lane) - 1u));
        if (stay && at < (unsigned)keep) {
            kept[at] = i;
            if (w_out) w_out[at] = x;
        }
        __syncthreads();
        if (tid == kSelectThreads - 1) { sh_tie0 = tbase + __popc(tb); sh_keep0 = kbase + __popc(kb); }
        __syncthreads();
    }
}

// Copy: 16 elements of k and v of one kept place a thread.
template <bool FP4>
__global__ void __launch_bounds__(kCopyThreads) evict_copy_kernel(const EvictParams p, int ctas_per_head) {
    const CacheView& c = p.c;
    const int64_t bh = blockIdx.x / ctas_per_head;
    const int part = (int)(blockIdx.x - bh * ctas_per_head), b = (int)(bh / c.heads), h = (int)(bh - (int64_t)b * c.heads);
    const int32_t* kept = p.kept + bh * p.budget;
    const int blocks = c.head_dim >> 4;
    CacheView to = c;
    to.block_table = p.new_table;
    to.max_pages = p.new_max_pages;
    for (int64_t it = (int64_t)part * kCopyThreads + threadIdx.x; it < (int64_t)p.budget * blocks; it += (int64_t)ctas_per_head * kCopyThreads) {
        const int i = (int)(it / blocks), q = (int)(it - (int64_t)i * blocks);
        const int pos = kept[i];
        if (pos < 0) return;                                                       // all behind it are -1 too
        const int64_t src = cache_row(c, b, h, pos), dst = cache_row(to, b, h, i);
        if (src < 0 || dst < 0) continue;
        if constexpr (FP4) {
            const uint2 k = *(const uint2*)(c.k + src * c.row_bytes + q * 8), v = *(const uint2*)(c.v + src * c.row_bytes + q * 8);
            const unsigned char ks = c.ks[src * blocks + q], vs = c.vs[src * blocks + q];
            *(uint2*)(c.k + dst * c.row_bytes + q * 8) = k;
            *(uint2*)(c.v + dst * c.row_bytes + q * 8) = v;
            c.ks[dst * blocks + q] = ks;
            c.vs[dst * blocks + q] = vs;
        } else {
            const uint4* k = (const uint4*)(c.k + src * c.row_bytes + q * 32);
            const uint4* v = (const uint4*)(c.v + src * c.row_bytes + q * 32);
            const uint4 a0 = k[0], a1 = k[1], b0 = v[0], b1 = v[1];
            uint4* dk = (uint4*)(c.k + dst * c.row_bytes + q * 32);
            uint4* dv = (uint4*)(c.v + dst * c.row_bytes + q * 32);
            dk[0] = a0; dk[1] = a1;
            dv[0] = b0; dv[1] = b1;
        }
    }
}
__global__ void evict_length_kernel(const CacheView c, int budget, int32_t* new_length) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < c.batch) new_length[b] = min(cache_length(c, b), budget);
}

}  // namespace cadd
