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
    float scale_log2;                                    // scale * log2(e): scores are kept in units of log 2
};

// Rows in use of request b.
__device__ __forceinline__ int attn_live(const AttnParams& p, int b) {
    return min(max(p.n_nodes ? p.n_nodes[b] : p.R - 1, -1), p.R - 1) + 1;
}
__device__ __forceinline__ int attn_depth(const AttnParams& p, int b, int r) {
    return p.depth ? min(max(p.depth[(int64_t)b * p.R + r], 0), 1 << 20) : r;
}
// Does a row at place len + depth see cached place pos?
__device__ __forceinline__ bool attn_sees_place(const AttnParams& p, int place, int pos) {
    return p.window == 0 || pos < p.n_sinks || place - pos < p.window;
}
// Does tree row r see tree row c?
__device__ __forceinline__ bool attn_sees_row(const AttnParams& p, int b, int len, int r, int dr, int c) {
    const bool link = p.mask_bits ? (p.mask_bits[((int64_t)b * p.R + r) * p.mask_words + (c >> 5)] >> (c & 31)) & 1u : c <= r;
    if (!link || p.window == 0) return link;
    const int dc = attn_depth(p, b, c);
    return dr - dc < p.window || len + dc < p.n_sinks;
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
__device__ __forceinline__ void row_add(RowSums<D>& st, const float (&q)[D / 32], const float (&k)[D / 32], const float (&v)[D / 32], float scale_log2) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFullMask, s, o);
    s *= scale_log2;
    if (s == -INFINITY) return;
    const float m = fmaxf(st.m, s);                      // a NaN score leaves m and makes the sums NaN
    const float a = st.m == -INFINITY ? 0.0f : exp2f(st.m - m), e = exp2f(s - m);
    st.m = m;
    st.l = st.l * a + e;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) st.o[i] = fmaf(e, v[i], st.o[i] * a);
}
// Adds the keys [from, to) that row r sees: cached places, or (TREE) rows of the tree.
template <int D, bool FP4, bool TREE>
__device__ __noinline__ void row_attend(const AttnParams& p, int b, int h, int len, int r, const float (&q)[D / 32], int from, int to, RowSums<D>& st) {
    const int lane = threadIdx.x & 31, dr = attn_depth(p, b, r);
    float k[D / 32], v[D / 32];
    for (int i = from; i < to; ++i) {
        if constexpr (TREE) {
            if (!attn_sees_row(p, b, len, r, dr, i)) continue;
            const int64_t at = ((int64_t)b * p.kvs_b + (int64_t)i * p.kvs_row + (int64_t)h * p.kvs_head) * 2;
            load_row_bf16<D>(p.k + at, lane, k);
            load_row_bf16<D>(p.v + at, lane, v);
        } else {
            if (!attn_sees_place(p, len + dr, i)) continue;
            const int64_t row = cache_row(p.c, b, h, i);
            if (row < 0) continue;
            load_row_cache<D, FP4>(p.c, p.c.k, p.c.ks, p.c.k_exp, row, lane, k);
            load_row_cache<D, FP4>(p.c, p.c.v, p.c.vs, p.c.v_exp, row, lane, v);
        }
        row_add<D>(st, q, k, v, p.scale_log2);
    }
}

}  // namespace cadd
