// What decides which cached places stay: the weight that accepted rows spend on them (cadd_cache_weights), and the choice
// of the heaviest with the copy of their rows (cadd_cache_evict).
#pragma once
#include "cache.cuh"
#include "tree_attention.cuh"
#include "fp4.cuh"
#include "warp_product.cuh"
#include "tile_ring.cuh"

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
    int ctas_per_head, keys_per_cta;
};

// Weights of the accepted rows on the cached keys.  Few rows (the path times the group's heads, 16 to some 70) meet long
// caches, so the keys are read once and everything else has to keep up with that: 72 bytes a key and head in 4 bits are three
// cycles of an SM.  Warp-level products (16 rows x 8 keys x 16 elements) take a key's elements from registers as they come from
// memory, without a detour over shared memory: which element stands in which place of the contraction is free as long as
// rows and keys agree, so lane t of a key's four lanes holds a contiguous quarter of its row (4 bits: one 16-byte load, D 128),
// and word m of it, eight elements, feeds contraction steps 2m and 2m + 1.  The rows stand in shared memory as 16-byte chunks in
// the same order (in fp16 for a 4-bit cache: fp4.cuh).  A warp takes 32 keys at a time, the next 32 being on their way; sums
// over rows stay in registers and are joined across the lanes at the end, in a fixed order.  More than 128 rows are done in
// groups, the later ones adding to what the earlier ones wrote.
// Measured on a B200 (32 requests of up to 32k places, 4 to 52 rows a head, 4 bits): 202 us, 0.29 of the measured copy rate (236
// where every row is in bf16; bf16 cache: 360 us, 0.53, with 176 bytes of spills a thread, 4 bits 12).  Twelve warps an SM hide
// little: table entries and totals are fetched a step before their use (245 -> 201 us; four CTAs an SM, with spills, came to
// 270); issue is then active 50 % of the time, logic 33 %, tensor pipe 28 %, DRAM 20 %.  By count: 190 instructions to dequantise a
// warp's 32 keys, and per 16 rows 32 products, 16 exponentials a thread and their sums.
constexpr int kWThreads = 128;
constexpr int kWRows = 128;                              // rows in shared memory at a time
template <int D> struct alignas(16) WeightsShared {
    uint4 q[kWRows][D / 8 + 1];                          // one chunk of padding: rows eight apart lie in different banks
    float lse[kWRows];                                   // times log2(e); +Inf marks a row that adds nothing
    float scale[kWRows];                                 // of the row's scores
    int place[kWRows];
};

template <int D, bool FP4>
__global__ void __launch_bounds__(kWThreads, D == 128 ? 3 : 4) weights_kernel(const __grid_constant__ WeightsParams p) {
    extern __shared__ __align__(16) unsigned char weights_smem_raw[];
    WeightsShared<D>& sh = *reinterpret_cast<WeightsShared<D>*>(weights_smem_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int bh = blockIdx.x / p.ctas_per_head, part = blockIdx.x - bh * p.ctas_per_head, b = bh / p.c.heads, h = bh - b * p.c.heads;
    const int len = cache_length(p.c, b), begin = part * p.keys_per_cta, chunk_end = min(cache_capacity(p.c), begin + p.keys_per_cta), end = min(len, chunk_end);
    if (p.w_out != p.w_in) {                             // another array: places from the length on are copied
        const float* src = p.w_in + (int64_t)bh * p.w_stride;
        float* dst = p.w_out + (int64_t)bh * p.w_stride;
        for (int i0 = max(begin, len) + tid; i0 < chunk_end; i0 += 8 * kWThreads) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = i0 + j * kWThreads < chunk_end ? __ldg(src + i0 + j * kWThreads) : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i0 + j * kWThreads < chunk_end) dst[i0 + j * kWThreads] = x[j];
        }
    }
    if (begin >= end) return;
    const int base = min(max(p.base_length[b], 0), len);
    int clamped;
    const int rows = min(row_count(p.rows, b, &clamped), len - base) * p.group;
    const float* w_in = p.w_in + (int64_t)bh * p.w_stride;
    float* w_out = p.w_out + (int64_t)bh * p.w_stride;
    constexpr int W = D / 32;                            // words of a lane, two contraction steps each

    for (int m0 = 0; m0 == 0 || m0 < rows; m0 += kWRows) {
        const int here = min(rows - m0, kWRows), tiles = (here + 15) >> 4;
        if (m0) __syncthreads();
        // a row's D / 8 chunks by as many neighbouring lanes; true: a row is lost to fp16 (then once more, all of them as bf16)
        auto stage = [&](bool wide) -> bool {
            bool lost = false;
            for (int i = tid; i < tiles * 16 * (D / 8); i += kWThreads) {
                const int m = i / (D / 8), ch = i - m * (D / 8), li = (m0 + m) / p.group, hq = h * p.group + (m0 + m - li * p.group);
                const int r = m < here ? row_at(p.rows, b, li) : -1;
                const float lse = r >= 0 ? p.lse[((int64_t)b * p.rows.R + r) * p.heads_q + hq] : INFINITY;
                const bool out = fabsf(lse) == INFINITY;
                uint4 x = make_uint4(0, 0, 0, 0);        // a row that adds nothing: zeros, whatever it holds
                if (!out) x = __ldg((const uint4*)(p.q + ((int64_t)b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)hq * p.qs_head) * 2) + ch);
                float scale = p.scale_log2;
                if constexpr (FP4) {
                    float amax = chunk_amax(x);
#pragma unroll
                    for (int o = D / 16; o; o >>= 1) {   // (the loop's trip count is the same for all lanes of a row)
                        const float y = __shfl_xor_sync(kFullMask, amax, o);
                        amax = !(y <= amax) ? y : amax;
                    }
                    int e = 0;
                    unsigned met = 0;
                    if (!wide) x = half_row_chunk(x, amax, e, met);
                    scale *= exp2i(e - p.c.k_exp);
                    const unsigned mine = ((1u << (D / 8)) - 1) << (lane & ~(D / 8 - 1));      // the row's lanes
                    const unsigned rounded = __ballot_sync(kFullMask, met & kHalfRounded) & mine, unfit = __ballot_sync(kFullMask, met & kHalfUnfit) & mine;
                    lost |= half_row_lost(rounded, unfit, scale);
                }
                sh.q[m][wkeys_slot<D, FP4>(ch)] = x;
                if (ch == 0) {
                    sh.lse[m] = out ? INFINITY : lse * kLog2e;
                    sh.scale[m] = scale;
                    sh.place[m] = base + li;
                }
            }
            return __syncthreads_or(lost);
        };
        const bool wide = stage(false);
        if (FP4 && wide) stage(true);
        // (a loop for rows in fp16 and one for rows in bf16: a choice inside the loop, 232 us where this takes 201)
        auto cached = [&](auto wide_tag) {
            constexpr bool kHalf = FP4 && !decltype(wide_tag)::value;
            WKeys<D, FP4> x[4];
            int64_t row[4];
            int k0 = begin + warp * 32;
            auto exist_bits = [&]() -> unsigned {             // bit j: this lane's key of group j exists
                unsigned e = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) e |= row[j] >= 0 ? 1u << j : 0u;
                return e;
        };
        int page[4];
        wkeys_pages(p.c, b, k0, g, end, page);
        wkeys_rows(p.c, h, k0, g, end, page, row);
#pragma unroll
        for (int j = 0; j < 4; ++j) wkeys_load<D, FP4>(x[j], p.c, row[j], t);
        unsigned there = exist_bits(), there_next;
        wkeys_pages(p.c, b, k0 + kWThreads, g, end, page);                         // looked up a step before the keys are fetched
        const int mine = (g >> 1) * 8 + 2 * t + (g & 1);    // the key of each 32 whose sum this lane ends with
        const float* totals = m0 ? w_out : w_in;
        const int counted = m0 ? end : min(base, end);      // places that have a total
        auto total_of = [&](int key) { return key < counted ? totals[key] : 0.0f; };
        float before = total_of(k0 + mine), before_next;    // (and so are the totals: what a step waits for has been under way for a step)
        for (; k0 < end; k0 += kWThreads, there = there_next, before = before_next) {
            const int key = k0 + mine;
            before_next = total_of(key + kWThreads);
            uint32_t kf[4][W * 4];                       // the 32 keys as operands: [key group of 8][word][two steps x two registers]
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                [[maybe_unused]] uint32_t f0 = 0, f1 = 0;
                if constexpr (FP4) fp4_half_scales(x[j].s, f0, f1);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    uint4 v;
                    if constexpr (FP4) v = fp4_half_values(x[j].w[i], (D == 128 && i >= 2) ? f1 : f0);
                    else v = x[j].w[i];
                    kf[j][4 * i] = v.x; kf[j][4 * i + 1] = v.y; kf[j][4 * i + 2] = v.z; kf[j][4 * i + 3] = v.w;
                }
            }
            if constexpr (FP4 && !kHalf) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < W * 4; ++i) kf[j][i] = bf16_of_half(kf[j][i]);
            }
            wkeys_rows(p.c, h, k0 + kWThreads, g, end, page, row);
#pragma unroll
            for (int j = 0; j < 4; ++j) wkeys_load<D, FP4>(x[j], p.c, row[j], t);            // the next keys
            there_next = exist_bits();
            wkeys_pages(p.c, b, k0 + 2 * kWThreads, g, end, page);
            float sum[4][2] = {};
            if (p.window == 0 || k0 < p.n_sinks || k0 + 31 > base - p.window) {
                const bool plain = p.window == 0 && k0 + 31 <= base;               // every row sees all 32
#pragma unroll 1
                for (int mt = 0; mt < tiles; ++mt) {
                    float c[4][4] = {};
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const uint4 lo = sh.q[mt * 16 + g][i * 4 + t], hi = sh.q[mt * 16 + g + 8][i * 4 + t];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            mma_16x8x16<kHalf>(c[j], lo.x, hi.x, lo.y, hi.y, kf[j][4 * i], kf[j][4 * i + 1]);
                            mma_16x8x16<kHalf>(c[j], lo.z, hi.z, lo.w, hi.w, kf[j][4 * i + 2], kf[j][4 * i + 3]);
                        }
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int m = mt * 16 + half * 8 + g, place = sh.place[m];
                        const float lse = sh.lse[m], sc = sh.scale[m];
                        if (FP4 && plain) {              // codes are finite: a row with lse = +Inf gives 2^-Inf by itself
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                sum[j][0] += ex2(fmaf(c[j][half * 2], sc, -lse));
                                sum[j][1] += ex2(fmaf(c[j][half * 2 + 1], sc, -lse));
                            }
                        } else {
                            const bool out = lse == INFINITY;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int at = k0 + j * 8 + 2 * t + e;
                                    const bool see = !out && at <= place && (p.window == 0 || at < p.n_sinks || place - at < p.window);
                                    const float v = ex2(fmaf(c[j][half * 2 + e], sc, -lse));
                                    sum[j][e] += see ? v : 0.0f;
                                }
                            }
                        }
                    }
                }
            }
            // sums over the eight lanes of equal t; each round halves what a lane goes on with
            float a[4], c2[2], v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {                // g's high bit chooses between key groups 0, 1 and 2, 3
                const float keep = g & 4 ? sum[2 + (i >> 1)][i & 1] : sum[i >> 1][i & 1], give = g & 4 ? sum[i >> 1][i & 1] : sum[2 + (i >> 1)][i & 1];
                a[i] = keep + __shfl_xor_sync(kFullMask, give, 16);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float keep = g & 2 ? a[2 + i] : a[i], give = g & 2 ? a[i] : a[2 + i];
                c2[i] = keep + __shfl_xor_sync(kFullMask, give, 8);
            }
            v = (g & 1 ? c2[1] : c2[0]) + __shfl_xor_sync(kFullMask, g & 1 ? c2[0] : c2[1], 4);
            // whether that key exists is known to the lanes with g' = mine & 7, as bit mine >> 3
            const unsigned known = __shfl_sync(kFullMask, there, (mine & 7) * 4);
            if (!((known >> (mine >> 3)) & 1u)) v = 0.0f;                          // on no page: nothing to be seen
            if (key < end) w_out[key] = before + v;
        }
        };
        if constexpr (FP4) {
            if (!wide) cached(Flag<false>{});
            else cached(Flag<true>{});
        } else {
            cached(Flag<false>{});
        }
        if (rows <= kWRows) break;
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
    int budget, room, n_sinks, n_recent, new_max_pages;  // budget: columns of kept; room: places that stay at most
};
constexpr int kSelectThreads = 1024;

// Order of weights as integers, NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w == w ? ord32(__float_as_uint(w + 0.0f)) : 0u; }

// Choice: one CTA per (request, head).  Of the n - sinks - recent places between, the `left` heaviest stay.  Three passes
// over the keys' digits of 11, 11 and 10 bits, highest first, count how often each digit occurs among the keys that share the digits
// found so far and so find the left-th largest key T and how many places with exactly T stay.  (Weights lie close together: their
// first eight bits take a handful of values, and counting in shared memory then waits for the same few words.)  Then each warp takes a contiguous part of the
// places, counts what stays there, and after one scan over the warps writes it down without further barriers.  The weights come
// from L2 after the first pass.
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
    constexpr int kWarps = kSelectThreads / 32;
    __shared__ unsigned hist[2048];
    __shared__ unsigned warp_sure[kWarps], warp_tie[kWarps];
    __shared__ unsigned sh_prefix, sh_left;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / p.c.heads), h = (int)(bh - (int64_t)b * p.c.heads);
    const int n = cache_length(p.c, b), keep = min(n, p.room);
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
    if (n <= p.room) {
        for (int i = tid; i < n; i += kSelectThreads) {
            kept[i] = i;
            if (w_out) w_out[i] = w[i];
        }
        return;
    }
    const int lo = p.n_sinks, hi = n - p.n_recent;
    unsigned left = (unsigned)(p.room - p.n_sinks - p.n_recent), prefix = 0;
    constexpr int kBins = 2048 / kSelectThreads;                                   // a thread has neighbouring digits, the last thread the largest
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), above_shift = pass == 0 ? 32 : (pass == 1 ? 21 : 10);
        const unsigned mask = pass == 2 ? 1023u : 2047u;
#pragma unroll
        for (int i = 0; i < kBins; ++i) hist[tid * kBins + i] = 0;
        __syncthreads();
#pragma unroll 8
        for (int i = lo + tid; i < hi; i += kSelectThreads) {
            const unsigned key = weight_key(__ldg(w + i));
            if (pass == 0 || (key >> above_shift) == (prefix >> above_shift)) atomicAdd(&hist[(key >> shift) & mask], 1u);
        }
        __syncthreads();
        unsigned mine[kBins], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins; ++i) { mine[i] = hist[tid * kBins + i]; sum += mine[i]; }
        unsigned above = sum;                                                      // keys with a digit of this thread's or more
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned x = __shfl_down_sync(kFullMask, above, o);
            if (lane + o < 32) above += x;
        }
        if (lane == 0) warp_sure[warp] = above;
        __syncthreads();
        above -= sum;                                                              // of higher threads'
        for (int k = warp + 1; k < kWarps; ++k) above += warp_sure[k];
        // the left-th largest is here (left = 0: nothing between stays; the largest digit takes T's place)
        if ((left > above && left <= above + sum) || (left == 0 && tid == kSelectThreads - 1)) {
            unsigned rest = left - above;
            int d = kBins - 1;
            if (left == 0) rest = 0;
            else for (; d > 0 && mine[d] < rest; --d) rest -= mine[d];
            sh_left = rest;
            sh_prefix = prefix | ((unsigned)(tid * kBins + d) << shift);
        }
        __syncthreads();
        left = sh_left;                                                            // of the keys that start like this, how many stay
        prefix = sh_prefix;
        __syncthreads();
    }
    const unsigned T = prefix, ties = left;
    const int per = (((n + kWarps - 1) / kWarps) + 31) & ~31, from = min(n, warp * per), to = min(n, from + per);
    unsigned sure = 0, tie_n = 0;                                                  // of a lane's places: stay whatever happens, have key T
#pragma unroll 4
    for (int i = from + lane; i < to; i += 32) {
        const bool inner = i >= lo && i < hi;
        const unsigned key = weight_key(__ldg(w + i));
        sure += !inner || key > T;
        tie_n += inner && key == T;
    }
    sure = __reduce_add_sync(kFullMask, sure);
    tie_n = __reduce_add_sync(kFullMask, tie_n);
    if (lane == 0) { warp_sure[warp] = sure; warp_tie[warp] = tie_n; }
    __syncthreads();
    unsigned at = 0, tie_at = 0;                                                   // kept places and ties of the warps before
    {
        const unsigned s = lane < warp ? warp_sure[lane] : 0, t = lane < warp ? warp_tie[lane] : 0;
        at = __reduce_add_sync(kFullMask, s);
        tie_at = __reduce_add_sync(kFullMask, t);
        at += min(tie_at, ties);
    }
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < to ? __ldg(w + i) : 0.0f;
        const unsigned key = weight_key(x);
        const bool inner = i >= lo && i < hi;
        const bool tie = i < to && inner && key == T;
        const unsigned before = (1u << lane) - 1u, tb = __ballot_sync(kFullMask, tie);
        const bool stay = i < to && (!inner || key > T || (tie && tie_at + __popc(tb & before) < ties));
        const unsigned kb = __ballot_sync(kFullMask, stay);
        const unsigned slot = at + __popc(kb & before);
        if (stay && slot < (unsigned)keep) {
            kept[slot] = i;
            if (w_out) w_out[slot] = x;
        }
        at += __popc(kb);
        tie_at += __popc(tb);
    }
}

// Copy: a thread moves 32 bytes of a kept place's key and value rows in bf16, 16 bytes of each and their two scales in 4 bits.
// Bound by memory traffic: 453 MB read and written in 84 us, 5.4 TB/s (0.82 of the measured copy rate).
template <bool FP4>
__global__ void __launch_bounds__(kCopyThreads) evict_copy_kernel(const __grid_constant__ EvictParams p, int ctas_per_head) {
    grid_dependency_wait();
    const CacheView& c = p.c;
    const int64_t bh = blockIdx.x / ctas_per_head;
    const int part = (int)(blockIdx.x - bh * ctas_per_head), b = (int)(bh / c.heads), h = (int)(bh - (int64_t)b * c.heads);
    const int32_t* kept = p.kept + bh * p.budget;
    const int per_row = FP4 ? c.head_dim >> 5 : c.head_dim >> 4;
    CacheView to = c;
    to.block_table = p.new_table;
    to.max_pages = p.new_max_pages;
    const int64_t items = (int64_t)p.room * per_row, step = (int64_t)ctas_per_head * kCopyThreads;
    for (int64_t it = (int64_t)part * kCopyThreads + threadIdx.x; it < items; it += step) {
        const int i = (int)(it / per_row), q = (int)(it - (int64_t)i * per_row);
        const int pos = kept[i];
        if (pos < 0) return;                                                       // all behind it are -1 too
        const int64_t src = cache_row(c, b, h, pos), dst = cache_row(to, b, h, i);
        if (src < 0 || dst < 0) continue;
        if constexpr (FP4) {
            const uint4 k = __ldcs((const uint4*)(c.k + src * c.row_bytes) + q), v = __ldcs((const uint4*)(c.v + src * c.row_bytes) + q);
            const unsigned short ks = *((const unsigned short*)(c.ks + src * (c.head_dim >> 4)) + q), vs = *((const unsigned short*)(c.vs + src * (c.head_dim >> 4)) + q);
            *((uint4*)(c.k + dst * c.row_bytes) + q) = k;
            *((uint4*)(c.v + dst * c.row_bytes) + q) = v;
            *((unsigned short*)(c.ks + dst * (c.head_dim >> 4)) + q) = ks;
            *((unsigned short*)(c.vs + dst * (c.head_dim >> 4)) + q) = vs;
        } else {
            const uint4* k = (const uint4*)(c.k + src * c.row_bytes + q * 32);
            const uint4* v = (const uint4*)(c.v + src * c.row_bytes + q * 32);
            const uint4 a0 = __ldcs(k), a1 = __ldcs(k + 1), b0 = __ldcs(v), b1 = __ldcs(v + 1);
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
