// Tree attention for few rows (16 and fewer: a decoded token's group of heads, a small tree) over a 4-bit cache.
//
// Such a call is a walk over the cache, 144 bytes a key and head at 128 elements, six cycles of an SM: blocks of 128 rows on the
// tensor memory's products would cost more than that for rows that are not there.  Here a warp takes 32 keys at a time from
// memory to registers, dequantises them there and multiplies by warp-level products, keys as in the weights' kernel
// (warp_product.cuh).  For the values a lane (g, t) holds elements g D/8 .. (g+1) D/8 - 1 of keys 2t and 2t + 1 of each group of
// eight: one nibble of each key side by side is what the conversion instruction turns into the operand's pair.  The four
// warps of a CTA work on different keys of the item, each with its own maximum, sum and output, joined in shared
// memory at the item's end; keys are shared out over the CTAs as in attn_plan.cuh.  The next keys are on their way from the
// moment the last are in their operands, the next values from the moment the last are multiplied.  Cached keys and values are
// multiplied in fp16 (fp4.cuh), the tree's rows in bf16.
//
// Measured on a B200, 8x4 heads of 128: 16 tokens over up to 32k places 180 us, 0.30 of the copy rate; 64 over up to 8191 places
// 211 us, one over 32k 37.  Latency and issue bound it: 255 registers leave eight warps an SM with one step of 32 keys each on its
// way; issue is active 43 % of the time, logic 36 %, tensor pipe 22 %, DRAM 25 %, and a warp waits 1.5 issue slots for its own last
// instructions and 1.0 for memory for each one it issues.
#pragma once
#include "attn_plan.cuh"
#include "warp_product.cuh"

namespace cadd {

constexpr int kFewRows = 16;
constexpr int kFewThreads = 128;
// Weights are formed as 2^(s - m + kFewUp): up to 2^15 where a score exceeds the reference m by the slack, so that fp16 holds them to
// 2^-8 of themselves or better from 2^-25 of the reference's weight on (2^-17, an fp16 subnormal with seven bits).  A step of 32
// keys with a smaller one takes its products in bf16, which has fp32's range; the values, code * scale, are the same in both.
// (16 tokens over up to 32k places on a B200: 170 us without the look at the smallest score, 179 with it, 196 where nearly every
// step has one.)
constexpr float kFewSlack = 7.0f;                        // as kTileSlack for fp16 weights
constexpr int kFewUp = 8;
constexpr float kFewHalfRange = 25.0f;

template <int D> struct alignas(16) FewShared {
    uint4 qh[kFewRows][D / 8 + 1], qb[kFewRows][D / 8 + 1];                        // fp16 scaled, bf16; one chunk of padding
    float scale[kFewRows];                               // of the scores of cached keys
    int2 row_at[kFewRows];                               // tree row, depth
    float o[4][kFewRows][D + 4];
    float2 ml[4][kFewRows];
    int64_t spare[4];                                    // a cached row in use, of each warp's part
    PlanShared plan;
    int odd;
};

__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D> struct FewValues {                      // a lane's share of 32 keys' values: [group of eight][key 2t, 2t + 1]
    uint32_t w[4][2][D / 64];
    uint32_t s[4];                                       // the two scales as bytes
};
// Places of the lane's keys of group j: 8 j + 2 t + e.  Their rows are known to the lanes that hold those keys' rows for the scores.  A
// key that does not exist gets zeros; its loads, unconditional like all others, go to `spare`, a row in use.  (Loads under a
// condition: 212 us where this takes 180, 16 tokens over up to 32k places on a B200; so does leaving out the zero scale.)
template <int D>
__device__ __forceinline__ void few_values_load(FewValues<D>& x, const CacheView& c, const int64_t (&row)[4], int64_t spare, int g, int t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t s[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int64_t r = __shfl_sync(kFullMask, row[j], (2 * t + e) * 4), safe = r < 0 ? spare : r;
            if constexpr (D == 128) {
                const uint2 v = __ldg((const uint2*)(c.v + safe * (D / 2)) + g);
                x.w[j][e][0] = v.x;
                x.w[j][e][1] = v.y;
                s[e] = __ldg(c.vs + safe * (D / 16) + g);
            } else {
                x.w[j][e][0] = __ldg((const uint32_t*)(c.v + safe * (D / 2)) + g);
                s[e] = __ldg(c.vs + safe * (D / 16) + (g >> 1));
            }
            if (r < 0) s[e] = 0;                         // zero scale, zero values
        }
        x.s[j] = s[0] | (s[1] << 8);
    }
}
// Word i of both keys of a group: eight operand registers, elements 8 i .. 8 i + 7 of the lane's share.
__device__ __forceinline__ void few_value_pairs(uint32_t a, uint32_t b, uint32_t scales, uint32_t (&r)[8]) {
    const uint32_t m = 0x0f0f0f0fu, even = (a & m) | ((b << 4) & ~m), odd = ((a >> 4) & m) | (b & ~m);
    uint32_t f;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"((unsigned short)scales));
    const uint4 x = fp4_half_values(even, f), y = fp4_half_values(odd, f);
    r[0] = x.x; r[1] = y.x; r[2] = x.y; r[3] = y.y; r[4] = x.z; r[5] = y.z; r[6] = x.w; r[7] = y.w;
}

template <int D>
__global__ void __launch_bounds__(kFewThreads, 2) attn_few_kernel(const __grid_constant__ AttnWork w) {
    extern __shared__ __align__(16) unsigned char few_smem_raw[];
    FewShared<D>& sh = *reinterpret_cast<FewShared<D>*>(few_smem_raw);
    const AttnParams& p = w.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    constexpr int W = D / 32, NB = D / 8;                // words of a lane's share of a key; column groups of the output
    WorkIter<kFewRows> it;
    if (tid == 0) sh.odd = 0;
    if (!it.init(p, sh.plan, blockIdx.x, gridDim.x)) {
        if (tid == 0) { w.items[blockIdx.x] = make_int4(0, 0, 0, kRangeEmpty); w.odd[blockIdx.x] = 0; }
        return;
    }
    if (tid == 0) w.items[blockIdx.x] = make_int4(it.b, it.h, it.mb, (it.u0 > 0 ? kRangeInside : 0) | (it.u1 == it.n_units ? kRangeEnds : 0));
    do {
        __syncthreads();                                  // the last item's sums have been read
        const int M = min(it.live * p.group - it.mb * kFewRows, kFewRows);
        for (int i = tid; i < kFewRows * NB; i += kFewThreads) {
            const int m = i / NB, ch = i - m * NB, m0 = it.mb * kFewRows + m, r = m0 / p.group, hq = it.h * p.group + (m0 - r * p.group);
            uint4 x = make_uint4(0, 0, 0, 0);
            if (m < M) x = __ldg((const uint4*)(p.q + ((int64_t)it.b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)hq * p.qs_head) * 2) + ch);
            float amax = chunk_amax(x);
#pragma unroll
            for (int o = NB / 2; o; o >>= 1) {
                const float y = __shfl_xor_sync(kFullMask, amax, o);
                amax = !(y <= amax) ? y : amax;
            }
            int e;
            unsigned met = 0;
            sh.qb[m][ch] = x;
            sh.qh[m][wkeys_slot<D, true>(ch)] = half_row_chunk(x, amax, e, met);
            const unsigned mine = ((1u << NB) - 1) << (lane & ~(NB - 1));          // the row's lanes
            const unsigned rounded = __ballot_sync(kFullMask, met & kHalfRounded) & mine, unfit = __ballot_sync(kFullMask, met & kHalfUnfit) & mine;
            if (ch == 0) {
                // a row lost to fp16: NaN, which sends it to the join's rows that are done key by key
                const float scale = p.scale_log2 * exp2i(e - p.c.k_exp);
                sh.scale[m] = half_row_lost(rounded, unfit, scale) ? __int_as_float(0x7fc00000) : scale;
                sh.row_at[m] = make_int2(m < M ? r : 0, attn_depth(p, it.b, m < M ? r : 0));
            }
        }
        __syncthreads();
        float o[NB][4];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};                  // rows g, g + 8; l over the lane's keys
        const float scale[2] = {sh.scale[g], sh.scale[g + 8]};
        const int2 at[2] = {sh.row_at[g], sh.row_at[g + 8]};

        // scores -> weights times 2^up in their place, m, l and o following; `see` of a row: bits of the 32 keys.  True: a weight (or what
        // a score that is masked would weigh) lies below what fp16 holds.
        auto softmax = [&](float (&c)[4][4], const float (&sc)[2], bool masked, const uint32_t (&see)[2], int up) -> bool {
            float low[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                low[h] = fminf(c[0][2 * h], c[0][2 * h + 1]);
#pragma unroll
                for (int j = 1; j < 4; ++j) low[h] = min3(low[h], c[j][2 * h], c[j][2 * h + 1]);
            }
            if (masked) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[j][e] = (see[e >> 1] >> (j * 8 + 2 * t + (e & 1))) & 1u ? c[j][e] : -INFINITY;
            }
            float f[2];
            bool raise = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) mx = fmaxf(mx, fmaxf(c[j][2 * h], c[j][2 * h + 1]));
                mx = fmaxf(mx, __shfl_xor_sync(kFullMask, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(kFullMask, mx, 2)) * sc[h];
                raise |= mx > m[h] + kFewSlack || (m[h] == -INFINITY && mx > m[h]);
                f[h] = fmaxf(m[h], mx);
            }
            if (__any_sync(kFullMask, raise)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float mn = f[h];
                    f[h] = m[h] == -INFINITY ? 0.0f : ex2(m[h] - mn);
                    m[h] = mn;
                    l[h] *= f[h];
                }
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    o[i][0] *= f[0]; o[i][1] *= f[0];
                    o[i][2] *= f[1]; o[i][3] *= f[1];
                }
            }
            const float down = exp2i(-up);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float off = (float)up - (m[h] == -INFINITY ? 0.0f : m[h]);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[j][2 * h] = ex2(fmaf(c[j][2 * h], sc[h], off));
                    c[j][2 * h + 1] = ex2(fmaf(c[j][2 * h + 1], sc[h], off));
                    sum += c[j][2 * h] + c[j][2 * h + 1];
                }
                l[h] = fmaf(sum, down, l[h]);
            }
            return __any_sync(kFullMask, low[0] * sc[0] < m[0] - kFewHalfRange || low[1] * sc[1] < m[1] - kFewHalfRange);
        };

        const int ctx_end = min(it.u1, it.ctx.total);
        // ---- cached keys: the warp's steps of 32 are halves warp, warp + 4, ... of the part's ----
        {
            auto first_of = [&](int s) { return it.first_key(it.u0 + (s >> 1)) + (s & 1) * 32; };
            int steps = 2 * max(0, ctx_end - it.u0);
            if (steps && first_of(steps - 1) >= it.len) --steps;                   // (the last unit's second half)
            WKeys<D, true> kx[4];
            FewValues<D> vx;
            int64_t row[4];
            // A step's keys are fetched once the last ones are in their operands, its values once the last ones are multiplied, and its
            // rows are looked up a step before that.
            auto look_up = [&](int s) {
                if (s < steps) wkeys_rows(p.c, it.b, it.h, first_of(s), g, it.len, row);
            };
            auto exist_bits = [&]() -> unsigned {         // bit j: the lane's key (of the scores) of group j exists
                unsigned x = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) x |= row[j] >= 0 ? 1u << j : 0u;
                return x;
            };
            unsigned there = 0, there_next = 0;
            if (warp < steps) {
                // (row 0 where a table entry outside the pool leaves the warp's first key without one)
                if (lane == 0) sh.spare[warp] = max(cache_row(p.c, it.b, it.h, first_of(warp)), (int64_t)0);
                __syncwarp();
                look_up(warp);
                there = exist_bits();
#pragma unroll
                for (int j = 0; j < 4; ++j) wkeys_load<D, true>(kx[j], p.c, row[j], t);
                few_values_load<D>(vx, p.c, row, sh.spare[warp], g, t);
                look_up(warp + 4);
            }
            for (int s = warp; s < steps; s += 4, there = there_next) {
                float c[4][4] = {};
                {
                    uint32_t kf[4][W * 4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t f0, f1;
                        fp4_half_scales(kx[j].s, f0, f1);
#pragma unroll
                        for (int i = 0; i < W; ++i) {
                            const uint4 v = fp4_half_values(kx[j].w[i], (D == 128 && i >= 2) ? f1 : f0);
                            kf[j][4 * i] = v.x; kf[j][4 * i + 1] = v.y; kf[j][4 * i + 2] = v.z; kf[j][4 * i + 3] = v.w;
                        }
                    }
                    if (s + 4 < steps) {
                        there_next = exist_bits();
#pragma unroll
                        for (int j = 0; j < 4; ++j) wkeys_load<D, true>(kx[j], p.c, row[j], t);
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const uint4 lo = sh.qh[g][i * 4 + t], hi = sh.qh[g + 8][i * 4 + t];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            mma_16x8x16<true>(c[j], lo.x, hi.x, lo.y, hi.y, kf[j][4 * i], kf[j][4 * i + 1]);
                            mma_16x8x16<true>(c[j], lo.z, hi.z, lo.w, hi.w, kf[j][4 * i + 2], kf[j][4 * i + 3]);
                        }
                    }
                }
                const int k0 = first_of(s);
                uint32_t see[2] = {~0u, ~0u};
                const bool whole = __all_sync(kFullMask, there == 15u) && p.window == 0;
                if (!whole) {
                    // bits of the 32 keys that exist: lane (key, 0) knows four, one of each group
                    uint32_t exist = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t bl = __ballot_sync(kFullMask, (there >> j) & 1u);
#pragma unroll
                        for (int k = 0; k < 8; ++k) exist |= ((bl >> (4 * k)) & 1u) << (8 * j + k);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) see[h] = exist & attn_key_bits(p, false, it.b, it.len, it.live, at[h].x, at[h].y, k0);
                }
                const bool wide = softmax(c, scale, !whole, see, kFewUp);
                // O += P V, two steps of 16 keys
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t a[4];                        // rows g, g + 8 of keys 0..7, then of keys 8..15
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = c[2 * h + (e >> 1)][2 * (e & 1)], y = c[2 * h + (e >> 1)][2 * (e & 1) + 1];
                        a[e] = wide ? pack_bf16(x, y) : pack_half(x, y);
                    }
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) {
                        uint32_t b0[8], b1[8];
                        few_value_pairs(vx.w[2 * h][0][i], vx.w[2 * h][1][i], vx.s[2 * h], b0);
                        few_value_pairs(vx.w[2 * h + 1][0][i], vx.w[2 * h + 1][1][i], vx.s[2 * h + 1], b1);
                        if (!wide) {
#pragma unroll
                            for (int n = 0; n < 8; ++n) mma_16x8x16<true>(o[i * 8 + n], a[0], a[1], a[2], a[3], b0[n], b1[n]);
                        } else {
#pragma unroll
                            for (int n = 0; n < 8; ++n) mma_16x8x16<false>(o[i * 8 + n], a[0], a[1], a[2], a[3], bf16_of_half(b0[n]), bf16_of_half(b1[n]));
                        }
                    }
                }
                if (s + 4 < steps) {
                    few_values_load<D>(vx, p.c, row, sh.spare[warp], g, t);
                    look_up(s + 8);
                }
            }
        }
        // ---- the tree's rows, bf16 ----
        for (int s = 2 * max(0, it.ctx.total - it.u0) + warp; s < 2 * (it.u1 - it.u0); s += 4) {
            const int k0 = it.first_key(it.u0 + (s >> 1)) + (s & 1) * 32;
            if (k0 >= it.live) continue;
            const int64_t base = (int64_t)it.b * p.kvs_b + (int64_t)it.h * p.kvs_head;
            float c[4][4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = k0 + j * 8 + g;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const uint4 v = key < it.live ? __ldg((const uint4*)(p.k + (base + (int64_t)key * p.kvs_row) * 2) + i * 4 + t) : make_uint4(0, 0, 0, 0);
                    const uint4 lo = sh.qb[g][i * 4 + t], hi = sh.qb[g + 8][i * 4 + t];
                    mma_16x8x16<false>(c[j], lo.x, hi.x, lo.y, hi.y, v.x, v.y);
                    mma_16x8x16<false>(c[j], lo.z, hi.z, lo.w, hi.w, v.z, v.w);
                }
            }
            uint32_t see[2], a[4][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) see[h] = attn_key_bits(p, true, it.b, it.len, it.live, at[h].x, at[h].y, k0);
            const float sc[2] = {p.scale_log2, p.scale_log2};
            softmax(c, sc, true, see, kFewUp + p.c.v_exp);
#pragma unroll
            for (int j = 0; j < 4; ++j) { a[j][0] = pack_bf16(c[j][0], c[j][1]); a[j][1] = pack_bf16(c[j][2], c[j][3]); }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {        // eight elements of four keys
                    uint4 v[2][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int key = k0 + (2 * h + j) * 8 + 2 * t + e;
                            v[j][e] = key < it.live ? __ldg((const uint4*)(p.v + (base + (int64_t)key * p.kvs_row + g * NB + i * 8) * 2)) : make_uint4(0, 0, 0, 0);
                        }
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        auto word = [&](const uint4& x) { return n < 2 ? x.x : (n < 4 ? x.y : (n < 6 ? x.z : x.w)); };
                        const uint32_t pick = n & 1 ? 0x7632u : 0x5410u;
                        mma_16x8x16<false>(o[i * 8 + n], a[2 * h][0], a[2 * h][1], a[2 * h + 1][0], a[2 * h + 1][1],
                                           __byte_perm(word(v[0][0]), word(v[0][1]), pick), __byte_perm(word(v[1][0]), word(v[1][1]), pick));
                    }
                }
            }
        }
        // ---- the four warps' sums ----
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(kFullMask, l[h], 1);
            l[h] += __shfl_xor_sync(kFullMask, l[h], 2);
            if (t == 0) sh.ml[warp][g + 8 * h] = make_float2(m[h], l[h]);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                sh.o[warp][g + 8 * h][2 * t * NB + i] = o[i][2 * h];
                sh.o[warp][g + 8 * h][(2 * t + 1) * NB + i] = o[i][2 * h + 1];
            }
        }
        __syncthreads();
        const int row = tid >> 3, c0 = (tid & 7) * NB;    // a thread: D / 8 elements of a row
        if (row < M) {
            float ml = -INFINITY, sum = 0.0f, f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) ml = fmaxf(ml, sh.ml[k][row].x);
            const float ref = ml == -INFINITY ? 0.0f : ml;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[k] = ex2(sh.ml[k][row].x - ref);
                sum = fmaf(sh.ml[k][row].y, f[k], sum);
            }
            const bool whole = it.whole();
            const float post = exp2i(-kFewUp - p.c.v_exp) * (whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f);
            const int m0 = it.mb * kFewRows + row, r = m0 / p.group, hq = it.h * p.group + (m0 - r * p.group);
            float* rec = w.records + ((int64_t)blockIdx.x * 2 + (it.u0 > 0 ? 0 : 1)) * record_floats<kFewRows, D>();
            unsigned char* dst = p.out + ((int64_t)it.b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head) * 2;
            bool odd = false;
#pragma unroll
            for (int i = 0; i < NB; i += 8) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int d = c0 + i + j;
                    x[j] = (sh.o[0][row][d] * f[0] + sh.o[1][row][d] * f[1] + sh.o[2][row][d] * f[2] + sh.o[3][row][d] * f[3]) * post;
                    odd |= !(fabsf(x[j]) <= 3.4e38f);
                }
                if (whole) {
                    *(uint4*)(dst + (c0 + i) * 2) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
                } else {
                    *(float4*)(rec + row * D + c0 + i) = make_float4(x[0], x[1], x[2], x[3]);
                    *(float4*)(rec + row * D + c0 + i + 4) = make_float4(x[4], x[5], x[6], x[7]);
                }
            }
            if (odd) sh.odd = 1;
            if (c0 == 0) {
                if (!whole) { rec[kFewRows * D + row] = ml; rec[kFewRows * (D + 1) + row] = sum; }
                else if (p.lse) p.lse[((int64_t)it.b * p.R + r) * p.heads_q + hq] = sum == 0.0f ? -INFINITY : (ml + log2f(sum)) * kLn2;
            }
        }
    } while (it.next(p));
    __syncthreads();
    if (tid == 0) w.odd[blockIdx.x] = sh.odd ? kRangeOdd : 0;
}

}  // namespace cadd
