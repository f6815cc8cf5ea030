// How the attention kernels share out their work.
//
// An item is (request, key/value head, block of BM rows), a row being one (tree row, query head of the group) pair: all
// query heads of a group use the same keys, so they stand in one block.  An item's keys are cut into units of 64: the
// cached places that any of its rows can see (all, or with a window the sinks' units and the window's), then the tree's
// rows.  All units of all items, one after the other, are cut into equal ranges, one per CTA, whatever the requests'
// lengths (an item's beginning and end, its queries and its results, count as kItemCost units more, in front of its own: without
// that, a request with an empty cache and a tree of 256 nodes, whose items have a few units each, kept one CTA busy for 660 us
// where the others took 340; measured on a B200): a CTA works through the ends and wholes of items that its range covers.  An item that lies in one range is
// finished there; of an item that does not, every range leaves sums (m, l, o) relative to its own maximum, and
// attn_join_kernel adds them up in range order: the same inputs give the same bits.
#pragma once
#include "cache.cuh"
#include "tile_ring.cuh"
#include "tree_attention.cuh"

namespace cadd {

constexpr int kUnit = 64;                                // keys per unit

constexpr int kItemCost = 5;                             // units' worth of time that an item takes besides its units (0 where every unit gets a CTA)

struct AttnWork {
    AttnParams p;
    float* records;                                      // [grid][2] partial records of BM x (D + 2) floats
    int4* items;                                         // [grid] what each range begins with
    int* odd;                                            // [grid] what the range met: kRangeOdd, kRangeTimedOut
};

// The cached units of an item: `sink_units` from place 0 on, then up to the length from unit `win_first` on.
struct CtxUnits {
    int sink_units, win_first, total;
};
__device__ __forceinline__ CtxUnits ctx_units(const AttnParams& p, int len) {
    CtxUnits c;
    const int all = (len + kUnit - 1) / kUnit;
    c.sink_units = 0;
    c.win_first = 0;
    if (p.window > 0) {
        const int lowest = max(0, len - p.window + 1);                  // no row of depth >= 0 sees below it but for the sinks
        const int sinks = (min(p.n_sinks, lowest) + kUnit - 1) / kUnit;
        if (sinks < lowest / kUnit) { c.sink_units = sinks; c.win_first = lowest / kUnit; }
    }
    c.total = c.sink_units + all - c.win_first;
    return c;
}
// Tree rows that row block mb can see: all live ones, or without a mask those up to its last row.
template <int BM>
__device__ __forceinline__ int tree_rows(const AttnParams& p, int live, int mb) {
    if (p.mask_bits) return live;
    return min(live, ((mb + 1) * BM - 1) / p.group + 1);                // rows times group: at most 2^24
}
template <int BM>
__device__ __forceinline__ int row_blocks(const AttnParams& p, int live) { return (live * p.group + BM - 1) / BM; }
// Units of one head of a request, the items' cost included.
template <int BM>
__device__ __forceinline__ int64_t units_per_head(const AttnParams& p, int len, int live) {
    const int mbs = row_blocks<BM>(p, live), ctx = ctx_units(p, len).total;
    if (p.mask_bits) return (int64_t)mbs * (p.item_cost + ctx + (live + kUnit - 1) / kUnit);
    int64_t n = (int64_t)mbs * (p.item_cost + ctx);
    for (int mb = 0; mb < mbs; ++mb) n += (tree_rows<BM>(p, live, mb) + kUnit - 1) / kUnit;
    return n;
}

struct PlanShared {
    int64_t part[32];
    int64_t first_off;
    int first_b;
};

// Range c of G: [T c / G, T (c+1) / G).
__device__ __forceinline__ int64_t range_begin(int64_t total, int c, int G) { return total * c / G; }

// The CTA's walk through its range; every warp keeps one of its own and all of them agree.
template <int BM>
struct WorkIter {
    int64_t left;                // units of the range not yet handed out
    int b, h, mb, mbs, live, len;
    CtxUnits ctx;
    int n_units;                 // of the item
    int u0, u1;                  // the CTA's part of it

    __device__ __forceinline__ void item_size(const AttnParams& p) {
        n_units = ctx.total + (tree_rows<BM>(p, live, mb) + kUnit - 1) / kUnit;
    }
    __device__ __forceinline__ void load_request(const AttnParams& p) {
        len = cache_length(p.c, b);
        live = attn_live(p, b);
        ctx = ctx_units(p, len);
        mbs = row_blocks<BM>(p, live);
    }
    // Whole CTA (barriers inside).  False: the range is empty.
    __device__ __forceinline__ bool init(const AttnParams& p, PlanShared& sh, int range, int ranges) {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = (int)blockDim.x >> 5;
        int64_t mine = 0;
        for (int i = tid; i < p.c.batch; i += (int)blockDim.x) mine += p.c.heads * units_per_head<BM>(p, cache_length(p.c, i), attn_live(p, i));
#pragma unroll
        for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(kFullMask, mine, o);
        if (lane == 0) sh.part[warp] = mine;
        __syncthreads();
        int64_t total = 0;
        for (int i = 0; i < nw; ++i) total += sh.part[i];
        const int64_t begin = range_begin(total, range, ranges);
        left = range_begin(total, range + 1, ranges) - begin;
        __syncthreads();
        int64_t base = 0;                                            // units of the requests before this chunk of requests
        for (int i0 = 0; i0 < p.c.batch && base <= begin; i0 += (int)blockDim.x) {
            const int i = i0 + tid;
            const int64_t n = i < p.c.batch ? p.c.heads * units_per_head<BM>(p, cache_length(p.c, i), attn_live(p, i)) : 0;
            int64_t upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(kFullMask, upto, o);
                if (lane >= o) upto += x;
            }
            if (lane == 31) sh.part[warp] = upto;
            __syncthreads();
            int64_t before = base, all = 0;
            for (int j = 0; j < nw; ++j) {
                if (j < warp) before += sh.part[j];
                all += sh.part[j];
            }
            upto += before;
            if (begin < upto && begin >= upto - n) { sh.first_b = i; sh.first_off = begin - (upto - n); }
            base += all;
            __syncthreads();
        }
        if (left <= 0) return false;
        b = sh.first_b;
        int64_t off = sh.first_off;
        load_request(p);
        const int64_t per_head = units_per_head<BM>(p, len, live);
        h = (int)(off / per_head);
        off -= h * per_head;
        mb = 0;
        item_size(p);
        while (off >= n_units + p.item_cost) { off -= n_units + p.item_cost; ++mb; item_size(p); }
        const int v1 = (int)min((int64_t)n_units + p.item_cost, off + left);
        left -= v1 - off;
        u0 = max(0, (int)off - p.item_cost);
        u1 = max(0, v1 - p.item_cost);
        return u1 > u0 || next(p);                       // (of an item whose cost alone lies in the range another range does all)
    }
    // On to the next item with units in the range; false at the range's end.
    __device__ __forceinline__ bool next(const AttnParams& p) {
        if (left <= p.item_cost) return false;
        if (++mb >= mbs) {
            mb = 0;
            if (++h >= p.c.heads) {
                h = 0;
                do { ++b; load_request(p); } while (mbs == 0);
            }
        }
        item_size(p);
        u0 = 0;
        u1 = (int)min((int64_t)n_units, left - p.item_cost);
        left -= u1 + p.item_cost;
        return true;
    }
    __device__ __forceinline__ bool is_tree(int u) const { return u >= ctx.total; }
    // First key of unit u: a cached place, or a tree row.
    __device__ __forceinline__ int first_key(int u) const {
        if (u >= ctx.total) return (u - ctx.total) * kUnit;
        return (u < ctx.sink_units ? u : ctx.win_first + u - ctx.sink_units) * kUnit;
    }
    __device__ __forceinline__ bool whole() const { return u0 == 0 && u1 == n_units; }
};

// Which of 64 keys from `key0` on row r (place len + dr) sees, as far as lengths, masks and windows say.
__device__ __forceinline__ uint32_t bits_from(int x) { return x <= 0 ? ~0u : (x >= 32 ? 0u : ~0u << x); }       // bits x.. of a word
__device__ __forceinline__ uint32_t attn_key_bits(const AttnParams& p, bool tree, int b, int len, int live, int r, int dr, int k);
__device__ __forceinline__ void unit_bits(const AttnParams& p, bool tree, int b, int len, int live, int r, int dr, int key0, uint32_t (&w)[kUnit / 32]) {
#pragma unroll
    for (int i = 0; i < kUnit / 32; ++i) w[i] = attn_key_bits(p, tree, b, len, live, r, dr, key0 + 32 * i);
}

// The same for 32 keys from `k`, a multiple of 32.
__device__ __forceinline__ uint32_t attn_key_bits(const AttnParams& p, bool tree, int b, int len, int live, int r, int dr, int k) {
    uint32_t m;
    if (!tree) {
        m = ~bits_from(len - k);
        if (p.window > 0) m &= bits_from(len + dr - p.window + 1 - k) | ~bits_from(p.n_sinks - k);
        return m;
    }
    m = 0;
    if (k < live) {
        m = p.mask_bits ? __ldg(p.mask_bits + ((int64_t)b * p.R + r) * p.mask_words + (k >> 5)) : ~bits_from(r + 1 - k);
        m &= ~bits_from(live - k);
    }
    if (p.window > 0) {
        for (uint32_t t = m; t; t &= t - 1) {
            const int c = k + __ffs(t) - 1, dc = attn_depth(p, b, c);
            if (!(dr - dc < p.window || len + dc < p.n_sinks)) m &= ~(1u << (c - k));
        }
    }
    return m;
}

// ---- what the ranges leave of an item that they share, and how it is joined ----
// A record: o [BM][D], then m [BM], then l [BM].
template <int BM, int D> __host__ __device__ constexpr int record_floats() { return BM * (D + 2); }

// What a range begins with: its first item's (b, h, mb) and flags.
constexpr int kRangeInside = 1;      // the range begins inside that item (its sums are record 0 of the range)
constexpr int kRangeEnds = 2;        // that item ends in the range
constexpr int kRangeEmpty = 4;
constexpr int kRangeOdd = 1;         // non-finite results
constexpr int kRangeTimedOut = 2;    // a wait ran out

// ---- rows done once more, key by key ----
constexpr int kJoinRows = 16;                            // rows of an item that a CTA of the join takes
// What a product of a weight 0 with a non-finite value that the row does not see has made NaN, and what the sums of large weights
// have made infinite, is right when it is computed from the row's own keys alone; so are rows that a kernel gave up (all NaN, lse
// too).  A row goes once through its keys, 32 at a time shared out over the warps of the CTA, whose sums are joined in warp
// order; elements that came out finite stay.  A row stops as soon as all that is asked for is NaN.  Measured on a B200: 16 rows
// over 8192 places, one row of Inf that all see, 5 ms (7 over 4 bits); 65 rows and 32 heads of one request over 32k places 33 ms,
// where the call takes 0.76 ms without.  (A walk for each eight elements of a row by one warp took 175 ms for the 16 rows.)
template <int D, int T> struct RedoShared {
    uint32_t want[kJoinRows][D / 32];                    // elements asked for, as bits
    float o[T / 32][D];
    float2 ml[T / 32];
    int stop;
};
// Whole CTA of T threads.  A thread has looked at eight elements, from 8 (tid % (D / 8)) on, of row tid / (D / 8) of the item's rows from
// blockIdx.y * kJoinRows on; `bad`: bits of those to be done again.
template <int D, bool FP4, int BM, int T>
__device__ __noinline__ void redo_rows(const AttnParams& p, const WorkIter<BM>& it, unsigned bad, RedoShared<D, T>& sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (!__syncthreads_or(bad != 0)) return;             // (and no one reads `sh` of the last call any more)
    reinterpret_cast<unsigned char*>(sh.want[tid / (D / 8)])[tid % (D / 8)] = (unsigned char)bad;
    __syncthreads();
    for (int row = 0; row < kJoinRows; ++row) {
        unsigned any = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) any |= sh.want[row][i];
        if (!any) continue;
        const int m0 = it.mb * BM + (int)blockIdx.y * kJoinRows + row, r = m0 / p.group, hq = it.h * p.group + (m0 - r * p.group);
        const int dr = attn_depth(p, it.b, r), d0 = lane * (D / 32);
        const uint32_t mine = sh.want[row][d0 >> 5] >> (d0 & 31);                  // of the lane's D / 32 elements
        float* lse = p.lse ? p.lse + ((int64_t)it.b * p.R + r) * p.heads_q + hq : nullptr;
        const bool want_lse = lse && *lse != *lse;
        if (tid == 0) sh.stop = 0;
        __syncthreads();
        float q[D / 32];
        load_row_bf16<D>(p.q + ((int64_t)it.b * p.qs_b + (int64_t)r * p.qs_row + (int64_t)hq * p.qs_head) * 2, lane, q);
        RowSums<D> st;
        st.m = -INFINITY;
        st.l = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) st.o[i] = 0.0f;
        for (int s = warp; s < 2 * it.n_units; s += T / 32) {
            const bool tree = it.is_tree(s >> 1);
            const int k0 = it.first_key(s >> 1) + (s & 1) * 32;
            const uint32_t see = attn_key_bits(p, tree, it.b, it.len, it.live, r, dr, k0);
            if (!see) continue;
            row_attend<D, FP4>(p, tree, it.b, it.h, see, q, k0, st);
            bool number = want_lse && st.l == st.l;      // something asked for is not NaN so far
#pragma unroll
            for (int i = 0; i < D / 32; ++i) number |= ((mine >> i) & 1u) && st.o[i] == st.o[i];
            if (!__any_sync(kFullMask, number) && lane == 0) *(volatile int*)&sh.stop = 1;
            if (__shfl_sync(kFullMask, *(volatile int*)&sh.stop, 0)) break;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) sh.o[warp][d0 + i] = st.o[i];
        if (lane == 0) sh.ml[warp] = make_float2(st.m, st.l);
        __syncthreads();
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int k = 0; k < T / 32; ++k) m = fmaxf(m, sh.ml[k].x);
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int k = 0; k < T / 32; ++k) l = fmaf(exp2f(sh.ml[k].x - ref), sh.ml[k].y, l);
        if (want_lse && tid == 0) *lse = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
        for (int d = tid; d < D; d += T) {
            if (!((sh.want[row][d >> 5] >> (d & 31)) & 1u)) continue;
            float o = 0.0f;
#pragma unroll
            for (int k = 0; k < T / 32; ++k) o = fmaf(exp2f(sh.ml[k].x - ref), sh.o[k][d], o);
            __nv_bfloat16* out = (__nv_bfloat16*)p.out + (int64_t)it.b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head;
            out[d] = __float2bfloat16_rn(l == 0.0f ? 0.0f : o / l);
        }
        __syncthreads();                                 // the sums have been read
    }
}
__device__ __forceinline__ unsigned not_finite(const float (&x)[8]) {
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bad |= !(fabsf(x[i]) <= 3.4e38f) ? 1u << i : 0u;
    return bad;
}

// Eight elements of a row whose range gave up on a wait: NaN, and its lse.
__device__ __forceinline__ void give_up_row(const AttnParams& p, int b, int r, int hq, int dc) {
    *(uint4*)(p.out + ((int64_t)b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head + dc * 8) * 2) =
        make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
    if (p.lse && dc == 0) p.lse[((int64_t)b * p.R + r) * p.heads_q + hq] = __int_as_float(0x7fffffff);
}

// The join.  blockIdx.x is a range: the one in which a shared item begins (its sums are record 1 there) joins it, blockIdx.y takes
// 16 of its rows.  Threads first find the ranges that share the item, then the rows' maxima over them, 16 ranges at a time; then
// a thread adds up eight elements of one row, in range order.  Rows whose joined result, or whose result in a whole item of
// a range that met non-finite numbers, is not finite are done once more.  Rows of items in which a range gave up on a wait get NaN.
template <int BM, int D, bool FP4>
__global__ void __launch_bounds__(kJoinRows * D / 8) attn_join_kernel(const __grid_constant__ AttnWork w, int grid) {
    constexpr int T = kJoinRows * D / 8, kPer = T / kJoinRows;                     // threads; ranges looked at in one go
    __shared__ int list[512];                                                      // ranges are at most 512 (kMaxGrid)
    __shared__ int count, any_odd, found[T / 32];
    __shared__ float part[kPer][kJoinRows];
    __shared__ PlanShared plan;
    __shared__ RedoShared<D, T> redo;
    grid_dependency_wait();
    const AttnParams& p = w.p;
    const int c0 = blockIdx.x, tid = threadIdx.x;
    if (p.status && blockIdx.y == 0) {                                             // the requests' status, shared out over the ranges
        int late = 0;
        for (int i = tid; i < grid; i += T) late |= w.odd[i] & kRangeTimedOut;
        late = __syncthreads_or(late);
        for (int b = c0; b < p.c.batch; b += (int)gridDim.x) {
            const int len = cache_length(p.c, b), bad = cache_bad_pages(p.c, b, 0, len), n = p.n_nodes ? p.n_nodes[b] : p.R - 1;
            if (tid == 0)
                p.status[b] = (bad ? CADD_STATUS_BAD_PAGE : 0) | (p.c.length[b] != len ? CADD_STATUS_BAD_LENGTH : 0) |
                              ((n < -1 || n > p.R - 1) ? CADD_STATUS_BAD_N_NODES : 0) | (late ? CADD_STATUS_INTERNAL_TIMEOUT : 0);
        }
    }
    const int4 mine = w.items[c0];
    if (mine.w & kRangeEmpty) return;
    const int dc = tid % (D / 8), row = blockIdx.y * kJoinRows + tid / (D / 8);    // a row's chunks in neighbouring lanes
    if (w.odd[c0]) {                                                               // the range's whole items
        WorkIter<BM> it;
        if (it.init(p, plan, c0, grid)) {
            do {
                if (!it.whole()) continue;
                const int m0 = it.mb * BM + row, r = m0 / p.group, hq = it.h * p.group + (m0 - r * p.group);
                unsigned bad = 0;
                if (w.odd[c0] & kRangeTimedOut) {
                    if (m0 < it.live * p.group) give_up_row(p, it.b, r, hq, dc);
                    continue;
                }
                if (m0 < it.live * p.group) {
                    const uint4 x = *(const uint4*)(p.out + ((int64_t)it.b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head + dc * 8) * 2);
                    float f[8];
                    Elem<CADD_DTYPE_BF16>::unpack(x, f);
                    bad = not_finite(f);
                }
                redo_rows<D, FP4, BM, T>(p, it, bad, redo);
            } while (it.next(p));
        }
    }
    if ((mine.w & kRangeInside) && !(mine.w & kRangeEnds)) return;                 // no item begins here and goes on
    int c = c0 + 1;
    while (c < grid && (w.items[c].w & kRangeEmpty)) ++c;
    if (c >= grid) return;
    const int4 item = w.items[c];
    if (!(item.w & kRangeInside)) return;
    const int b = item.x, h = item.y, mb = item.z, live = attn_live(p, b);
    if (mb * BM + (int)blockIdx.y * kJoinRows >= live * p.group) return;
    // the ranges that share it, in order
    if (tid == 0) { list[0] = c0; count = 1; any_odd = w.odd[c0]; }
    __syncthreads();
    for (int i0 = c; i0 < grid; i0 += T) {
        const int i = i0 + tid;
        bool in = false, behind = false;                                           // behind: an item after this one
        if (i < grid) {
            const int4 e = w.items[i];
            in = (e.w & kRangeInside) && !(e.w & kRangeEmpty) && e.x == b && e.y == h && e.z == mb;
            behind = !in && !(e.w & kRangeEmpty);
        }
        const unsigned ballot = __ballot_sync(kFullMask, in);
        if ((tid & 31) == 0) found[tid >> 5] = __popc(ballot);
        __syncthreads();
        int at = count + __popc(ballot & ((1u << (tid & 31)) - 1u));
        for (int k = 0; k < tid >> 5; ++k) at += found[k];
        if (in) {
            list[at] = i;
            if (w.odd[i]) atomicOr(&any_odd, w.odd[i]);
        }
        const bool last = __syncthreads_or(behind);
        if (tid == 0)
            for (int k = 0; k < T / 32; ++k) count += found[k];
        __syncthreads();
        if (last) break;
    }
    const int n = count, odd = any_odd & kRangeOdd, rec = record_floats<BM, D>();
    auto record = [&](int i) -> const float* { return w.records + ((int64_t)list[i] * 2 + (i == 0 ? 1 : 0)) * rec; };
    const int lr = tid % kJoinRows, li = tid / kJoinRows, grow = blockIdx.y * kJoinRows + lr;
    float mx = -INFINITY;
    for (int i = li; i < n; i += kPer) mx = fmaxf(mx, record(i)[BM * D + grow]);
    part[li][lr] = mx;
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) M = fmaxf(M, part[i][tid / (D / 8)]);
    const int m0 = mb * BM + row, r = m0 / p.group, hq = h * p.group + (m0 - r * p.group);
    const bool there = m0 < live * p.group;
    if (any_odd & kRangeTimedOut) {
        if (there) give_up_row(p, b, r, hq, dc);
        return;
    }
    unsigned bad = 0;
    if (there) {
        const float ref = M == -INFINITY ? 0.0f : M;
        float l = 0.0f, o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = 0.0f;
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float* rp = record(i);
            const float a = exp2f(rp[BM * D + row] - ref);
            const float4 x = *(const float4*)(rp + row * D + dc * 8), y = *(const float4*)(rp + row * D + dc * 8 + 4);
            l = fmaf(a, rp[BM * (D + 1) + row], l);
            o[0] = fmaf(a, x.x, o[0]); o[1] = fmaf(a, x.y, o[1]); o[2] = fmaf(a, x.z, o[2]); o[3] = fmaf(a, x.w, o[3]);
            o[4] = fmaf(a, y.x, o[4]); o[5] = fmaf(a, y.y, o[5]); o[6] = fmaf(a, y.z, o[6]); o[7] = fmaf(a, y.w, o[7]);
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint4 out;
        out.x = pack_bf16(o[0] * inv, o[1] * inv);
        out.y = pack_bf16(o[2] * inv, o[3] * inv);
        out.z = pack_bf16(o[4] * inv, o[5] * inv);
        out.w = pack_bf16(o[6] * inv, o[7] * inv);
        *(uint4*)(p.out + ((int64_t)b * p.os_b + (int64_t)r * p.os_row + (int64_t)hq * p.os_head + dc * 8) * 2) = out;
        if (p.lse && dc == 0) p.lse[((int64_t)b * p.R + r) * p.heads_q + hq] = l == 0.0f ? -INFINITY : (M + log2f(l)) * kLn2;
        if (odd) bad = not_finite(o);
    }
    if (odd) {
        WorkIter<BM> it;
        it.b = b; it.h = h; it.mb = mb;
        it.load_request(p);
        it.item_size(p);
        redo_rows<D, FP4, BM, T>(p, it, bad, redo);
    }
}

}  // namespace cadd
