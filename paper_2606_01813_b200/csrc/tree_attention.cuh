// Attention of a draft tree's rows over a paged cache and over the tree itself (cadd_tree_attention).
//
// For a row r and a query head, over the keys that r sees:  o = sum_p e^{s_p - m} v_p / sum_p e^{s_p - m},
// s_p = scale q . k_p, m the largest s_p, lse = m + log of the denominator.
#pragma once
#include "cache.cuh"

namespace cadd {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnParams {
    CacheView c;
    const unsigned char *q, *k, *v;                      // bf16
    unsigned char* out;
    int64_t qs_b, qs_row, qs_head, kvs_b, kvs_row, kvs_head, os_b, os_row, os_head;      // elements
    const int32_t *n_nodes, *depth;
    const uint32_t* mask_bits;
    float* lse;
    int32_t* status;
    int R, heads_q, group, window, n_sinks, mask_words, item_cost;
    int test_drop, wait_limit;                           // of attn_tiles.cuh: a unit never comes; tries of a wait
    float scale_log2;                                    // scale * log2(e): scores are kept in units of log 2
};

// Rows in use of request b.
__device__ __forceinline__ int attn_live(const AttnParams& p, int b) {
    return min(max(p.n_nodes ? p.n_nodes[b] : p.R - 1, -1), p.R - 1) + 1;
}
__device__ __forceinline__ int attn_depth(const AttnParams& p, int b, int r) {
    return p.depth ? min(max(p.depth[(int64_t)b * p.R + r], 0), 1 << 20) : r;
}
// ---- one row at a time: a warp holds the row's query and sums, four (two) of the head's elements a lane ----
template <int D> struct RowSums {
    float m, l, o[D / 32];
};
template <int D>
__device__ __forceinline__ void load_row_bf16(const unsigned char* row, int lane, float (&x)[D / 32]) {
    const uint32_t* w = (const uint32_t*)(row + lane * (D / 32) * 2);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const uint32_t u = __ldg(w + i);
        x[2 * i] = __uint_as_float(u << 16);
        x[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
    }
}
template <int D, bool FP4>
__device__ __forceinline__ void load_row_cache(const CacheView& c, const unsigned char* pool, const unsigned char* scales, int exp, int64_t row, int lane, float (&x)[D / 32]) {
    if constexpr (!FP4) {
        load_row_bf16<D>(pool + row * (D * 2), lane, x);
    } else {
        const float f = e4m3_value(scales[row * (D / 16) + lane * (D / 32) / 16]) * exp2i(-exp);
        const unsigned char* w = pool + row * (D / 2) + lane * (D / 64);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint32_t two = w[i];
            x[2 * i] = e2m1_value(two & 15u) * f;
            x[2 * i + 1] = e2m1_value(two >> 4) * f;
        }
    }
}
template <int D>
__device__ __forceinline__ void row_add(RowSums<D>& st, float s, const float (&v)[D / 32]) {
    if (s == -INFINITY) return;
    const float m = fmaxf(st.m, s);                      // a NaN score leaves m and makes the sums NaN
    const float a = st.m == -INFINITY ? 0.0f : exp2f(st.m - m), e = exp2f(s - m);
    st.m = m;
    st.l = st.l * a + e;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) st.o[i] = fmaf(e, v[i], st.o[i] * a);
}
// Adds the keys of `see` (bits of the 32 from k0: cached places, or rows of the tree), as a warp: a lane looks up one key's row, and
// four rows at a time are fetched and multiplied side by side.
template <int D, bool FP4>
__device__ __forceinline__ void row_attend(const AttnParams& p, bool tree, int b, int h, uint32_t see, const float (&q)[D / 32], int k0, RowSums<D>& st) {
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x & 31;
    int64_t row = -1;                                    // cache row, or row of the tree
    if ((see >> lane) & 1u) row = tree ? k0 + lane : cache_row(p.c, b, h, k0 + lane);
    const int64_t kv0 = (int64_t)b * p.kvs_b + (int64_t)h * p.kvs_head;
    for (unsigned todo = __ballot_sync(kFullMask, row >= 0); todo;) {
        const int n = min(__popc(todo), kAtOnce);
        float k[kAtOnce][D / 32], v[kAtOnce][D / 32], s[kAtOnce];
        int src = 0;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (todo) src = __ffs(todo) - 1;             // past the end: the last key once more, not added
            todo &= todo - 1;
            const int64_t r = __shfl_sync(kFullMask, row, src);
            if (tree) {
                load_row_bf16<D>(p.k + (kv0 + r * p.kvs_row) * 2, lane, k[j]);
                load_row_bf16<D>(p.v + (kv0 + r * p.kvs_row) * 2, lane, v[j]);
            } else {
                load_row_cache<D, FP4>(p.c, p.c.k, p.c.ks, p.c.k_exp, r, lane, k[j]);
                load_row_cache<D, FP4>(p.c, p.c.v, p.c.vs, p.c.v_exp, r, lane, v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) s[j] = fmaf(q[i], k[j][i], s[j]);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1)
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) s[j] += __shfl_xor_sync(kFullMask, s[j], o);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (j < n) row_add<D>(st, s[j] * p.scale_log2, v[j]);
    }
}

}  // namespace cadd
