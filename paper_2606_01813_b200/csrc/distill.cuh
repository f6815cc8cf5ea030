// Distillation of the drafter from the target's top tokens: losses and gradients (cadd_distill_args has the definition).
//
// One CTA an SM walks through the rows of drafter's logits (few rows: a cluster of CTAs, each with a contiguous segment of every row), which
// come to a ring of 40 KB tiles in shared memory by bulk copies.  The warps of a CTA have roles, so that no row waits for another's
// small steps:
//   producer   sends for the tiles, row after row, as stages fall free;
//   prepare    a row's list, a row ahead: the target's probabilities, the drafter's logits of the listed tokens, where they lie in the segment;
//   compute    (20 warps) adds up the exponentials of the tokens that are not listed, relative to a power of two near the
//              largest (see DistillSum): a listed token counts as -Inf there, and goes into the row's statistics by itself, in fp64, so the
//              rest's probability is right even where the listed tokens leave all but nothing; then, where the gradient is
//              wanted, forms it from the tiles: the row's last ones have stayed, as many as the ring holds, and the others come once more,
//              from L2, where there are never more rows than SMs;
//   finish     joins the warps' sums, exchanges them within the cluster (distributed shared memory), and makes of the statistics the
//              loss and the two factors that the gradient needs.
// The gradient alone (statistics given, no exchange) passes over the tiles once.
//
// What bounds it.  Losses alone: 1728 rows of 151936 in bf16 (526 MB) take 102 us, 5.2 TB/s; the exponential unit has 16 ex2 a clock of an SM, which
// is 66 % busy over the whole launch (DRAM 59 % of nominal).  Doing an eighth of them or more on the FMA pipes instead, as polynomials
// in packed fp32, was slower (103 -> 111: packed operations have only half of those pipes), and so was more CTAs an SM.  With the gradient:
// 2048 rows, 1245 MB, 246 us, 5.1 TB/s; the unit 60 % busy, and writes, which alone reach 3.8 to 4.0 TB/s here.  Both exponentials of an element
// are computed: kept ones would need fp32 tiles twice as large.  512 rows of 100003 in fp32: 88 to 93 us, 4.5 TB/s, of which a sixth
// is that 512 rows are not a multiple of the SMs.  Few rows: chains of loads and 64-bit steps, 9.4 us.  (All as replayed from a graph; called one
// after another with other inputs each time, 103 to 108 and 249 to 259 us for the first two.)
// All waits are bounded; a CTA in which one runs out leaves NaN in its rows from there on.
#pragma once
#include "common.cuh"
#include "tile_ring.cuh"
#include "packed.cuh"

namespace cadd {

constexpr int kDistillWarps = 20;                                   // that compute (step of 2048 rows: 281 us with 20, 292 with 24 of half as many chunks, 305 with 16, 293 with 28)
constexpr int kDistillCompute = 32 * kDistillWarps;
constexpr int kDistillThreads = kDistillCompute + 96;               // and producer, prepare, finish
constexpr int kDistillStatusThreads = 256;
constexpr int kDistillMaxC = 4;                                     // CTAs a row at most
constexpr int kDistillEach = 4;                                     // 16-byte chunks of a tile that a thread has
constexpr int kDistillTile = kDistillEach * kDistillCompute;
constexpr int kDistillMaxStages = 216 * 1024 / (kDistillTile * 16);
constexpr int kDistillMaxV = 2000000;
constexpr int kDistillK = CADD_DISTILL_MAX_K;
constexpr float kDistillLowest = -1.0e30f;                          // logits below count as -Inf
constexpr float kDistillUnder = -0x1.93e596p+99f;                   // the next float below that
constexpr float kDistillNear = 262144.0f;                           // see DistillSum
constexpr double kRestRounding = 0x1p-20;

struct DistillParams {
    const char* logits;
    char* grad;
    int64_t V, in_b, in_row, out_b, out_row;
    int rows, batch, L, R, K, path_cols, rest;
    int C, clusters, chunks_max, stages;          // CTAs a row; clusters; chunks of a segment at most; tiles of the ring
    float c, over_c;                              // log2(e) / T and its inverse
    double inv_t;
    const int32_t *token, *path, *path_len, *n_rows;
    const double *value, *lse;
    const float *weight, *grad_loss;
    float *loss, *stats;
    int32_t* status;
    int drop;                                     // test hook: this tile of every segment is never copied (-1: none)
};

// A row on its way through the roles; two of them are.
struct DistillRow {
    double p_rest, entropy, mass, cross;          // entropy, cross: sum p log p, sum p (s - m_list) / T over the entries; mass: sum p
    double z_list;                                // sum of e over tokens (not entries)
    double factor;                                // of the exponentials in the gradient of tokens that are not listed
    double sum[kDistillWarps], peer_sum[kDistillMaxC];
    float max[kDistillWarps], ref[kDistillWarps], peer_max[kDistillMaxC], peer_ref[kDistillMaxC];
    float weight, upstream;                       // of the row; grad_loss
    unsigned row;                                 // batch * L + position
    float m_list;                                 // largest listed logit
    float grad_base, grad_ref;                    // reference of the gradient's exponentials
    int live;                                     // 0: left out from the start, nothing is read
    int left_out;                                 // by its list, after its tiles have been sent for
    int twice;                                    // some token is listed more than once
    int near;                                     // some logit beside the list is far above those that are far out below
};
constexpr int kDistillGroups = 512;
struct DistillMap {
    int before[kDistillGroups + 1];
    int scan[kDistillThreads / 32];
};
// The entries of a row's list; n: K rounded up to whole warps.
struct DistillList {
    double *prob, *e;                             // p; exp((s - m_list) / T), 0 below kDistillLowest
    float* g;                                     // gradient of the token
    int* token;                                   // -1 where there is none
    int16_t *next, *thread;                       // next entry of the same part, -1: none; the thread that has the token
    uint8_t *where, *once;                        // which of the thread's (four) chunks of the tile, * 8 + element of the chunk; 1: the token's first entry
    __device__ __forceinline__ DistillList(unsigned char* at, int n) {
        prob = reinterpret_cast<double*>(at);
        e = prob + n;
        g = reinterpret_cast<float*>(e + n);
        token = reinterpret_cast<int*>(g + n);
        next = reinterpret_cast<int16_t*>(token + n);
        thread = next + n;
        where = reinterpret_cast<uint8_t*>(thread + n);
        once = where + n;
    }
};
constexpr int kDistillEntry = 30;                 // bytes of an entry
// Behind this: two lists; int first_of[2][parts + 2], the first entry of each row's list in each part of the segment, what a warp has
// of a tile (-1: none; the last two parts are the row's scalar head and tail); the ring.
struct DistillShared {
    alignas(8) uint64_t full[kDistillMaxStages], empty[kDistillMaxStages];
    uint64_t listed[2], ready[2], done[2], summed[2], known[2], exchanged;
    int sent[kDistillMaxStages];                  // last tile sent for into each stage, -1: none
    int error;
    unsigned lost;                                // the first row in the cluster's order that some role has not finished
    DistillRow row[2];
    DistillMap map;
};
__host__ __device__ inline int distill_parts(int chunks) { return (chunks + kDistillTile - 1) / kDistillTile * kDistillWarps; }
__host__ __device__ inline size_t distill_first_bytes(int chunks) { return ((size_t)(distill_parts(chunks) + 2) * 8 + 127) & ~(size_t)127; }
__host__ __device__ inline size_t distill_shared_bytes() { return (sizeof(DistillShared) + 127) & ~(size_t)127; }
__host__ __device__ inline size_t distill_list_bytes(int K) { return (size_t)((K + 31) & ~31) * kDistillEntry; }
__host__ __device__ inline size_t distill_ring_at(int chunks, int K) { return distill_shared_bytes() + 2 * distill_list_bytes(K) + distill_first_bytes(chunks); }
inline size_t distill_smem_bytes(int chunks, int K, int stages) { return distill_ring_at(chunks, K) + (size_t)stages * kDistillTile * 16; }

__device__ __forceinline__ uint32_t peer_address(const void* p, unsigned rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
// 2^n for an integer n that is small or negative, 0 below the normal range.
__device__ __forceinline__ double pow2_down(float n) {
    return n > -1000.0f ? __hiloint2double((1023 + (int)n) << 20, 0) : (n == n ? 0.0 : (double)n);
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    return x;
}

// Positions of request b that are learnt from.
__device__ __forceinline__ int distill_live(const DistillParams& p, int b) {
    if (p.path) {
        const int n = p.path_len[b], most = min(p.L - 1, p.path_cols);
        return 1 + max(0, min(n, most));
    }
    return p.n_rows ? max(0, min(p.n_rows[b], p.L)) : p.L;
}

// -Inf in an element of a chunk in shared memory.
template <int DT>
__device__ __forceinline__ void hide_element(uint4* chunk, int e) {
    if constexpr (DT == CADD_DTYPE_BF16) reinterpret_cast<volatile uint16_t*>(chunk)[e] = 0xff80u;
    else reinterpret_cast<volatile uint32_t*>(chunk)[e] = 0xff800000u;
}
// factor * 2^((x - base) c - ref) of a chunk's elements, as a chunk; without kFar, base is 0.
template <int DT, bool kFar>
__device__ __forceinline__ uint4 gradient_chunk(const uint4& w, uint64_t c2, float nbase, uint64_t nref2, uint64_t factor2) {
    using E = Elem<DT>;
    float f[E::EPC];
    E::unpack(w, f);
    if constexpr (kFar) {
#pragma unroll
        for (int q = 0; q < E::EPC; ++q) f[q] += nbase;
    }
    uint4 r;
    uint32_t* x = &r.x;
#pragma unroll
    for (int q = 0; q < E::EPC; q += 2) {
        float t0, t1;
        unpack2(fma2(pack2(f[q], f[q + 1]), c2, nref2), t0, t1);
        unpack2(mul2(pack2(ex2_approx(t0), ex2_approx(t1)), factor2), t0, t1);
        if constexpr (DT == CADD_DTYPE_BF16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(t0, t1);
            x[q / 2] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            x[q] = __float_as_uint(t0);
            x[q + 1] = __float_as_uint(t1);
        }
    }
    return r;
}
// An element's bits.
template <int DT> __device__ __forceinline__ uint32_t element_bits(float x) {
    if constexpr (DT == CADD_DTYPE_BF16) return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x));
    else return __float_as_uint(x);
}
template <int DT> __device__ __forceinline__ void store_chunk(char* row, int64_t i, const uint4& w) {      // where it is not aligned
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (DT == CADD_DTYPE_BF16) {
            ((uint16_t*)row)[i + 2 * q] = (uint16_t)x[q];
            ((uint16_t*)row)[i + 2 * q + 1] = (uint16_t)(x[q] >> 16);
        } else ((uint32_t*)row)[i + q] = x[q];
    }
}
template <int DT> __device__ __forceinline__ void store_element(char* row, int64_t i, float x) {
    if constexpr (DT == CADD_DTYPE_BF16) ((__nv_bfloat16*)row)[i] = __float2bfloat16_rn(x);
    else ((float*)row)[i] = x;
}

// A thread's running sum of 2^((x - base) c - ref) over the elements it has seen.
// While the largest x c is within kDistillNear, base is 0 and ref an integer between 3 above and 4 below it, so that x c - ref is rounded once, and a step from
// one reference to another is a power of two.  The rounding then moves a term by 2^-23 ln 2 of the largest at most (between 2^-24 and 2^-23 below 4 in
// magnitude; further down terms get smaller as fast as their roundings grow), which is less than ex2's own error.  The room on either side is for
// speed: it saves most steps to another reference, one of which halts a warp's 32 threads (training step of 2048 rows 242.0 us, losses of 1728 rows 99.9; with the
// least reference always 247 and 103, with 16 more 241.4 and 98.2 and roundings of 2^-20).
// Beyond, fp32 has no integers fine enough to tell x c from ref by: then base is the largest logit itself and ref 0, the difference of two logits being
// as exact as a product.  Every tile then goes the long way (top is -Inf), unless the row has been seen to hold logits so far above (DistillRow::near) that
// these add exactly nothing: such a thread goes on as one that has seen nothing yet (rows with a finite mask: 2048 rows 347 us without that).
// A sum of nothing has ref Inf, from which all terms are 0.
constexpr float kDistillSpare = 2.0f, kDistillAbove = 3.75f;
struct DistillSum {
    float m;                                      // the largest logit
    float base, ref;
    float top;                                    // the largest logit that the reference serves
    double acc;
    __device__ __forceinline__ DistillSum() : m(-INFINITY), base(0.0f), ref(INFINITY), top(kDistillUnder), acc(0.0) {}
};
__device__ __forceinline__ float warp_max(float x) {                // NaN ignored
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ bool is_far(float x, float c) { return !(fabsf(x * c) <= kDistillNear); }
// s.m is above s.top: the reference follows.
__device__ __forceinline__ void distill_raise(const DistillParams& p, DistillSum& s, volatile int* near) {
    const float at = s.m * p.c;
    const bool far = is_far(s.m, p.c), none = s.base == 0.0f && s.ref == INFINITY;         // (none: acc is 0, or NaN)
    if (at >= 1200.0f - kDistillNear) *near = 1;                    // (2^-1000 and less count as 0)
    if (!far && s.base == 0.0f) {
        const float ref = ceilf(at) + kDistillSpare;
        s.acc *= none ? 0.0 : pow2_down(s.ref - ref);
        s.ref = ref;
        s.top = fmaxf(s.m, (ref + kDistillAbove) * p.over_c);
    } else if (far && at < 0.0f && *near) {
        s.acc *= 0.0;
        s.base = 0.0f;
        s.ref = INFINITY;
        s.top = -kDistillNear * p.over_c;
    } else if (s.base != s.m) {
        const float base = far ? s.m : 0.0f, ref = far ? 0.0f : ceilf(at) + kDistillSpare;
        const double step = ((double)s.base * (double)p.c + (double)s.ref) - ((double)base * (double)p.c + (double)ref);
        s.acc *= none || step < -1000.0 ? 0.0 : exp2(step);
        s.base = base;
        s.ref = ref;
        s.top = far ? -INFINITY : fmaxf(s.m, (ref + kDistillAbove) * p.over_c);
    }
}
// A sum's reference for others: the integer; +-Inf where it is the largest logit; -Inf where there is nothing.
__device__ __forceinline__ float told_reference(const DistillSum& s) {
    return s.base != 0.0f ? copysignf(INFINITY, s.base) : (s.ref == INFINITY ? -INFINITY : s.ref);
}
__device__ __forceinline__ double whole_reference(float m, float told, float c) { return isinf(told) ? (double)m * (double)c : (double)told; }
// The step from one reference to another where the latter is far out, or so near that it is not far from others that are.
__device__ __noinline__ double far_step(float m, float told, float m_all, float all, float c) {
    if (!(m >= kDistillLowest)) return 0.0;
    const double step = whole_reference(m, told, c) - whole_reference(m_all, all, c);
    return step < -1000.0 ? 0.0 : exp2(step);
}
// Sums of the lanes together, in every lane: m the largest logit of a lane's sum, told its reference.
__device__ __forceinline__ void distill_join(float c, float& m, float& told, double& acc) {
    const float m_all = warp_max(m), all = warp_max(told);
    acc *= fabsf(all) <= kDistillNear - 1200.0f ? pow2_down(told - all) : far_step(m, told, m_all, all, c);      // (told -Inf: 0)
    m = m_all;
    told = all;
    acc = warp_sum(acc);
}
// Packed sums of the exponentials of a chunk's even and odd elements.
template <int DT, bool kFar>
__device__ __forceinline__ uint64_t chunk_terms(const uint4& w, uint64_t c2, float nbase, uint64_t nref2) {
    using E = Elem<DT>;
    float f[E::EPC];
    E::unpack(w, f);
    uint64_t pr[E::EPC / 2];
#pragma unroll
    for (int q = 0; q < E::EPC; q += 2) {
        float t0, t1;
        if (kFar) unpack2(mul2(pack2(f[q] + nbase, f[q + 1] + nbase), c2), t0, t1);
        else unpack2(fma2(pack2(f[q], f[q + 1]), c2, nref2), t0, t1);
        pr[q / 2] = pack2(ex2_approx(t0), ex2_approx(t1));
    }
    uint64_t r = add2(pr[0], pr[1]);
    if constexpr (E::EPC == 8) r = add2(r, add2(pr[2], pr[3]));
    return r;
}
template <int DT, bool kFar>
__device__ __forceinline__ double tile_terms(const uint4 (&w)[kDistillEach], uint64_t c2, const DistillSum& s) {
    const uint64_t nref2 = pack2(-s.ref, -s.ref);
    const uint64_t sum2 = add2(add2(chunk_terms<DT, kFar>(w[0], c2, -s.base, nref2), chunk_terms<DT, kFar>(w[1], c2, -s.base, nref2)),
                               add2(chunk_terms<DT, kFar>(w[2], c2, -s.base, nref2), chunk_terms<DT, kFar>(w[3], c2, -s.base, nref2)));
    float a0, a1;
    unpack2(sum2, a0, a1);
    return (double)(a0 + a1);
}

// Where the CTA stands in a row: what all roles work out for themselves.
template <int DT>
struct DistillSegment {
    using E = Elem<DT>;
    int b, i;
    const char* in;
    RowSplit sp;
    int nc, n_tiles, scalars, head;               // head: of the scalars, those before the chunks (the others are behind them)
    int64_t e0;                                   // token of the first chunk
    __device__ __forceinline__ DistillSegment(const DistillParams& p, unsigned row, int rank) {
        b = (int)(row / (unsigned)p.L);
        i = (int)(row - (unsigned)b * (unsigned)p.L);
        in = p.logits + ((int64_t)b * p.in_b + (int64_t)i * p.in_row) * E::ES;
        sp = split_row<DT>(in, p.V);
        const int per = (int)((unsigned)(sp.n_chunks + p.C - 1) / (unsigned)p.C), s0 = min(sp.n_chunks, rank * per);
        nc = min(per, sp.n_chunks - s0);
        n_tiles = (nc + kDistillTile - 1) / kDistillTile;
        e0 = sp.head + (int64_t)s0 * E::EPC;
        head = rank == 0 ? sp.head : 0;
        scalars = head + (rank == p.C - 1 ? sp.tail : 0);
    }
    __device__ __forceinline__ int64_t scalar(const DistillParams& p, int k) const { return k < head ? k : p.V - sp.tail + (k - head); }
};
// Rows in the order in which clusters take them: those that path or n_rows leave in (they cost most, and are dealt out evenly), then the
// others.  In shared memory: how many rows the requests before each group of requests leave in.
__device__ __forceinline__ int group_size(const DistillParams& p) { return (p.batch + kDistillGroups - 1) / kDistillGroups; }
// The whole CTA.
__device__ __forceinline__ void distill_map(const DistillParams& p, DistillMap& m) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, size = group_size(p), groups = (p.batch + size - 1) / size;
    int carry = 0;
    for (int g0 = 0; g0 < groups; g0 += kDistillThreads) {
        const int g = g0 + tid;
        int n = 0;
        if (g < groups)
            for (int b = g * size; b < min(p.batch, (g + 1) * size); ++b) n += distill_live(p, b);
        int sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFullMask, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) m.scan[warp] = sum;
        __syncthreads();
        int before = carry, all = carry;
        for (int k = 0; k < kDistillThreads / 32; ++k) {
            before += k < warp ? m.scan[k] : 0;
            all += m.scan[k];
        }
        if (g < groups) m.before[g + 1] = before + sum;
        carry = all;
        __syncthreads();
    }
    if (tid == 0) m.before[0] = 0;
    __syncthreads();
}
// The k-th row that is left in (live) or out: batch * L + position.
__device__ __forceinline__ unsigned distill_row(const DistillParams& p, const DistillMap& m, unsigned k, bool live) {
    if (!p.path && !p.n_rows) return k;
    const int size = group_size(p), groups = (p.batch + size - 1) / size;
    auto before = [&](int g) { return live ? (unsigned)m.before[g] : (unsigned)min(g * size, p.batch) * (unsigned)p.L - (unsigned)m.before[g]; };
    int lo = 0, hi = groups - 1;                                     // the last group with before(g) <= k
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before(mid) <= k) lo = mid;
        else hi = mid - 1;
    }
    unsigned left = k - before(lo);
    for (int b = lo * size;; ++b) {
        const unsigned in = (unsigned)distill_live(p, b), here = live ? in : (unsigned)p.L - in;
        if (left < here) return (unsigned)b * (unsigned)p.L + (live ? left : in + left);
        left -= here;
    }
}
// The target's row for position i of request b, or -1 where the position is left out.
__device__ __forceinline__ int distill_teacher(const DistillParams& p, unsigned row, int b, int i) {
    const float weight = p.weight ? p.weight[row] : 1.0f;
    int r = p.path && i > 0 && i - 1 < p.path_cols ? p.path[(int64_t)b * p.path_cols + i - 1] : (p.path ? 0 : i);
    if (i >= distill_live(p, b) || weight == 0.0f || r < 0 || r >= p.R) r = -1;
    return r;
}

// kLoss: statistics and loss are computed here; otherwise they are given.  kGrad: the gradient is written.
template <int DT, bool kLoss, bool kGrad>
__global__ void __launch_bounds__(kDistillThreads, 1) distill_kernel(DistillParams p) {
    using E = Elem<DT>;
    extern __shared__ __align__(128) unsigned char distill_smem_raw[];
    DistillShared& sh = *reinterpret_cast<DistillShared*>(distill_smem_raw);
    const int parts_max = distill_parts(p.chunks_max);
    const int list_size = (p.K + 31) & ~31;
    unsigned char* const list_all = distill_smem_raw + distill_shared_bytes();
    int* const first_all = reinterpret_cast<int*>(list_all + 2 * distill_list_bytes(p.K));
    uint4* ring = reinterpret_cast<uint4*>(distill_smem_raw + distill_ring_at(p.chunks_max, p.K));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned C = (unsigned)p.C, cluster = blockIdx.x / C;
    const int rank = (int)(blockIdx.x - cluster * C);
    if (tid == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], kDistillWarps); sh.sent[s] = -1; }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sh.listed[s], 1);
            mbar_init(&sh.ready[s], 1);
            mbar_init(&sh.done[s], kDistillWarps + 1);
            mbar_init(&sh.summed[s], kDistillWarps);
            mbar_init(&sh.known[s], 1);
        }
        mbar_init(&sh.exchanged, C);
        sh.error = 0;
        sh.lost = 0xffffffffu;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    unsigned n_live = (unsigned)p.rows;
    if (p.path || p.n_rows) {
        distill_map(p, sh.map);
        n_live = (unsigned)sh.map.before[(p.batch + group_size(p) - 1) / group_size(p)];
    } else __syncthreads();
    if (C > 1) { cluster_arrive(); cluster_wait(); }                 // every CTA's barriers are ready for the others
    // Waits of one warp; false: the time is up, here or in another role (then everybody leaves).
    volatile int* error = &sh.error;
    const unsigned nap = warp == kDistillWarps || warp == kDistillWarps + 1 ? 200u : 32u;
    auto wait = [&](uint64_t* bar, unsigned parity, int limit) {
        bool ok = false;
        for (int it = 0; it < limit && !ok; ++it) {
            ok = mbar_try_wait_cluster(bar, parity);
            if (ok) break;
            if (*error) break;
            __nanosleep(nap);                                        // a waiting warp must not take issue slots from those that compute
        }
        ok = __all_sync(kFullMask, ok);
        if (!ok) *error = 1;
        return ok;
    };
    auto arrive = [&](uint64_t* bar) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    // tile number g of the CTA (all rows' tiles in turn): its stage and the parity of that stage's barrier
    const unsigned S = (unsigned)p.stages;

    if (warp == kDistillWarps) {
        // ---------------- producer ----------------
        unsigned stage = 0, turn = 0;                                // turn: how often the ring has gone round
        bool going = true;
        const uint64_t keep = l2_keep(), drop_it = l2_drop();
        for (unsigned at = cluster; going && at < n_live; at += p.clusters) {
            const unsigned row = distill_row(p, sh.map, at, true);
            const DistillSegment<DT> seg(p, row, rank);
            if (distill_teacher(p, row, seg.b, seg.i) < 0) continue;
            const int drop = p.drop < 0 ? -1 : min(p.drop, seg.n_tiles - 1);
            // both loss and gradient: those that do not stay come twice, and are kept in L2 meanwhile
            const int again = kLoss && kGrad ? max(0, seg.n_tiles - (int)S) : 0;
            for (int u = 0; u < seg.n_tiles + again; ++u) {
                const int t = u < seg.n_tiles ? u : u - seg.n_tiles;
                if (turn > 0 && !wait(&sh.empty[stage], (turn - 1) & 1u, kSpinLimit)) { going = false; break; }
                if (lane == 0 && u != drop) {
                    const unsigned bytes = (unsigned)min(kDistillTile, seg.nc - t * kDistillTile) * 16u;
                    sh.sent[stage] = (int)turn;
                    mbar_arrive_expect_tx(&sh.full[stage], bytes);
                    bulk_load_hint((void*)(ring + stage * kDistillTile), seg.in + seg.e0 * E::ES + (int64_t)t * kDistillTile * 16, bytes, &sh.full[stage],
                                   u < again ? keep : drop_it);
                }
                if (++stage == S) { stage = 0; ++turn; }
            }
        }
        // no CTA leaves with a copy of its own in flight
        if (lane == 0)
            for (unsigned s = 0; s < S; ++s)
                if (sh.sent[s] >= 0) mbar_wait_bounded(&sh.full[s], (unsigned)sh.sent[s] & 1u);
    } else if (warp == kDistillWarps + 1) {
        // ---------------- prepare ----------------
        unsigned n = 0;
        for (unsigned order = cluster; order < n_live; order += p.clusters, ++n) {
            const unsigned row = distill_row(p, sh.map, order, true);
            DistillRow& k = sh.row[n & 1u];
            const DistillList l(list_all + (n & 1u) * distill_list_bytes(p.K), list_size);
            int* first_of = first_all + (n & 1u) * (parts_max + 2);
            const DistillSegment<DT> seg(p, row, rank);
            const int r = distill_teacher(p, row, seg.b, seg.i), parts = seg.n_tiles * kDistillWarps;
            if (n >= 2 && !wait(&sh.done[n & 1u], (n / 2 - 1) & 1u, kSpinLimit)) break;
            if (lane == 0) k.row = row;
            if (r < 0) {
                if (lane == 0) k.live = 0;
                arrive(&sh.listed[n & 1u]);
                arrive(&sh.ready[n & 1u]);
                continue;
            }
            for (int o = lane; o < parts + 2; o += 32) first_of[o] = -1;
            __syncwarp();                                            // (below, any lane's token may lie in any part)
            const float weight = p.weight ? p.weight[row] : 1.0f, upstream = p.grad_loss ? p.grad_loss[row] : 1.0f;
            if (lane == 0) { k.live = 1; k.near = 0; k.weight = weight; k.upstream = upstream; }
            const int64_t at = ((int64_t)seg.b * p.R + r) * p.K;
            double top = p.rest && p.lse ? p.lse[(int64_t)seg.b * p.R + r] / p.inv_t : (p.rest ? 0.0 : -INFINITY);
            float m_list = -INFINITY;
            bool any = false, twice = false;
            // tokens, and where they lie: all that the sums need
            for (int o = lane; o < list_size; o += 32) {
                int tok = o < p.K ? p.token[at + o] : -1;
                if (tok < 0 || tok >= p.V) tok = -1;
                l.token[o] = tok;
                int part = -1, thread = 0, where = 0;
                if (tok >= seg.e0 && tok < seg.e0 + (int64_t)seg.nc * E::EPC) {
                    const unsigned c = (unsigned)(tok - seg.e0) / E::EPC, t = c / kDistillTile, in_tile = c - t * kDistillTile;
                    thread = (int)(in_tile % kDistillCompute);
                    where = (int)(in_tile / kDistillCompute * 8 + (unsigned)(tok - seg.e0) % E::EPC);
                    part = (int)t * kDistillWarps + thread / 32;
                } else if (tok >= 0 && tok < seg.head) { thread = tok; part = parts; }
                else if (tok >= 0 && tok >= p.V - seg.sp.tail && seg.scalars > seg.head) { thread = (int)(tok - (p.V - seg.sp.tail)) + seg.head; part = parts + 1; }
                l.thread[o] = (int16_t)thread;
                l.where[o] = (uint8_t)where;
                if (part >= 0) l.next[o] = (int16_t)atomicExch(&first_of[part], o);
                // a token's first entry: none before it among the 32 of this turn, nor in the turns before
                const unsigned same = __match_any_sync(kFullMask, tok);
                bool once = tok >= 0 && __ffs(same) - 1 == lane;
                for (int f = 0; f < o - lane; f += 4) {
                    const int4 x = *reinterpret_cast<const int4*>(&l.token[f]);
                    once = once && x.x != tok && x.y != tok && x.z != tok && x.w != tok;
                }
                l.once[o] = once;
                twice = twice || (tok >= 0 && !once);
                // (the gradient alone may be written over logits by the other CTAs meanwhile: only this CTA's are read)
                l.e[o] = tok >= 0 && (kLoss || part >= 0) ? 1.0 : 0.0;
                __syncwarp();
            }
            arrive(&sh.listed[n & 1u]);
            // the target's and the drafter's logits
            for (int o = lane; o < p.K; o += 32) {
                const int tok = l.token[o];
                const double v = p.value[at + o];
                const float x = l.e[o] != 0.0 ? E::load(seg.in, tok) : -INFINITY;
                l.prob[o] = v;
                l.e[o] = (double)x;
                m_list = fmaxf(m_list, x);
                if (tok >= 0) {
                    if (!p.rest) top = fmax(top, v);
                    any = any || p.rest || !(v == -INFINITY);       // (NaN counts: it shows in the sum)
                }
            }
            m_list = warp_max(m_list);
            if (!(m_list >= kDistillLowest)) m_list = -INFINITY;
            any = __any_sync(kFullMask, any);
            twice = __any_sync(kFullMask, twice);
            if (!p.rest) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmax(top, __shfl_xor_sync(kFullMask, top, o));
            }
            // the target's probabilities, up to their sum, and the drafter's exponentials
            double sum = 0.0, z = 0.0, entropy = 0.0, cross = 0.0;
#pragma unroll 1
            for (int o = lane; o < p.K; o += 32) {
                double q = 0.0, e = 0.0;
                if (l.token[o] >= 0) {
                    const double x = l.e[o], lp = (l.prob[o] - top) * p.inv_t;
                    const bool none = x < (double)kDistillLowest;
                    q = exp(lp);
                    const double below = (x - (double)m_list) * p.inv_t;
                    if (!none) e = exp(below);
                    if (q != 0.0) {
                        entropy += q * lp;
                        cross += none ? -INFINITY : q * below;
                    }
                    sum += q;
                    if (l.once[o]) z += e;
                }
                l.prob[o] = q;
                l.e[o] = e;
            }
            sum = warp_sum(sum);
            z = warp_sum(z);
            entropy = warp_sum(entropy);
            cross = warp_sum(cross);
            double mass = sum;
            if (!p.rest) {
                const double scale = 1.0 / sum;
                for (int o = lane; o < p.K; o += 32) l.prob[o] *= scale;
                mass = sum * scale;
                entropy = entropy * scale - log(sum) * mass;
                cross *= scale;
            }
            if (lane == 0) {
                k.entropy = entropy;
                k.mass = mass;
                k.cross = cross;
                k.z_list = z;
                k.m_list = m_list;
                k.p_rest = !p.rest ? 0.0 : (sum < 1.0 ? 1.0 - sum : (sum == sum ? 0.0 : sum));
                k.left_out = any ? 0 : 1;
                k.twice = twice;
            }
            arrive(&sh.ready[n & 1u]);
        }
    } else if (warp == kDistillWarps + 2) {
        // ---------------- finish ----------------
        unsigned n = 0, lives = 0, order = cluster;                  // lives: rows read so far, per slot, a bit each: the parity of what only they pass
        for (; order < n_live; order += p.clusters, ++n) {
            const unsigned slot = n & 1u;
            DistillRow& k = sh.row[slot];
            const DistillList l(list_all + slot * distill_list_bytes(p.K), list_size);
            if (!wait(&sh.ready[slot], (n / 2) & 1u, kSpinLimit)) break;
            const unsigned row = k.row;
            float4* stats = reinterpret_cast<float4*>(p.stats) + row;
            if (!k.live) {
                if (kLoss && rank == 0 && lane == 0) {
                    if (p.loss) p.loss[row] = 0.0f;
                    if (p.stats) *stats = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
                arrive(&sh.done[slot]);
                continue;
            }
            const unsigned phase = (lives >> slot) & 1u;
            lives ^= 1u << slot;
            const double nan = __longlong_as_double(0x7ff8000000000000ll);
            float m_rest, m_all, ref = 0.0f;                         // an exponential of the gradient is exp((s - m_rest) / T) / up, where up is 2^(ref - m_rest c),
            double z_rest, z_all, a_list, a_rest, up;                // or, far out, 1
            bool far;
            const float m_list = k.m_list;
            if constexpr (kLoss) {
                if (!wait(&sh.summed[slot], phase, kSpinLimit)) break;
                bool in_use = lane < kDistillWarps;
                float m = in_use ? k.max[lane] : -INFINITY, told = in_use ? k.ref[lane] : -INFINITY;
                double acc = in_use ? k.sum[lane] : 0.0;
                distill_join(p.c, m, told, acc);
                if (C > 1) {                                         // (the cluster's only row: there are at least as many clusters as rows)
                    if (lane < (int)C) {
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_address(&k.peer_max[rank], lane)), "f"(m) : "memory");
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_address(&k.peer_ref[rank], lane)), "f"(told) : "memory");
                        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(peer_address(&k.peer_sum[rank], lane)), "d"(acc) : "memory");
                        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_address(&sh.exchanged, lane)) : "memory");
                    }
                    __syncwarp();
                    if (!wait(&sh.exchanged, 0u, kSpinLimit)) break;
                    in_use = lane < (int)C;
                    m = in_use ? k.peer_max[lane] : -INFINITY;
                    told = in_use ? k.peer_ref[lane] : -INFINITY;
                    acc = in_use ? k.peer_sum[lane] : 0.0;
                    distill_join(p.c, m, told, acc);
                }
                m_rest = m >= kDistillLowest ? m : -INFINITY;
                m_all = fmaxf(m_rest, m_list);
                // three exponentials at once: of the list's and the rest's largest, and of the step from the rest's reference to its largest
                const double x = lane == 0 ? ((double)m_list - (double)m_all) * p.inv_t : lane == 1 ? ((double)m_rest - (double)m_all) * p.inv_t
                                                                                            : (whole_reference(m_rest, told, p.c) - (double)m_rest * (double)p.c) * 0.693147180559945309;
                const double y = exp(x);
                a_list = m_list > -INFINITY ? __shfl_sync(kFullMask, y, 0) : 0.0;
                a_rest = __shfl_sync(kFullMask, y, 1);
                up = __shfl_sync(kFullMask, y, 2);
                z_rest = up * acc * kEx2BiasFix;
                far = m_rest > -INFINITY && is_far(m_rest, p.c);
                if (!(m_rest > -INFINITY)) {
                    a_rest = 0.0;
                    z_rest = acc == acc ? 0.0 : acc;
                } else if (far) up = 1.0;
                else {
                    ref = ceilf(m_rest * p.c);                       // the least that serves, so that small gradients stay
                    up *= pow2_down(ref - told);
                }
                z_all = k.z_list * a_list + z_rest * a_rest;
                if (!(m_all > -INFINITY) || !(acc == acc) || !(k.z_list == k.z_list)) z_all = nan;
            } else {
                const float4 st = *stats;
                m_all = st.x; z_all = (double)st.y; m_rest = st.z; z_rest = (double)st.w;
                far = m_rest > -INFINITY && is_far(m_rest, p.c);
                if (m_rest > -INFINITY && !far) ref = ceilf(m_rest * p.c);
                const double x = lane == 0 ? ((double)m_list - (double)m_all) * p.inv_t : lane == 1 ? ((double)m_rest - (double)m_all) * p.inv_t
                                                                                            : (far ? 0.0 : ((double)ref - (double)m_rest * (double)p.c) * 0.693147180559945309);
                const double y = exp(x);
                a_list = m_list > -INFINITY ? __shfl_sync(kFullMask, y, 0) : 0.0;
                a_rest = m_rest > -INFINITY ? __shfl_sync(kFullMask, y, 1) : 0.0;
                up = __shfl_sync(kFullMask, y, 2);
                if (!(m_all > -INFINITY)) z_all = nan;
            }
            const bool empty = !(m_rest > -INFINITY);                // no token is left beside the list
            const double total = k.mass + k.p_rest, weight = (double)k.weight;
            if constexpr (kGrad) {
                const double w = (double)k.upstream * weight * p.inv_t, inv = 1.0 / (lane == 1 ? z_rest : z_all);
                const double inv_all = __shfl_sync(kFullMask, inv, 0), inv_rest = __shfl_sync(kFullMask, inv, 1);
                if (lane == 0) {
                    k.grad_base = far ? m_rest : 0.0f;
                    k.grad_ref = ref;
                    k.factor = empty ? w * (0.0 * z_all) : w * (total * a_rest * inv_all - (k.p_rest != 0.0 ? k.p_rest * inv_rest : 0.0)) * up;
                }
                const double q = w * total * a_list * inv_all;
                const bool twice = k.twice != 0;
#pragma unroll 1
                for (int o = lane; o < p.K; o += 32) {
                    double mine = l.prob[o];
                    if (twice)
                        for (int f = o + 1; f < p.K; ++f)
                            if (l.token[f] == l.token[o]) mine += l.prob[f];
                    l.g[o] = (float)(l.e[o] * q - w * mine);
                }
                arrive(&sh.known[slot]);
            }
            if (kLoss && rank == 0) {
                const double log_z = log(z_all);                     // of exp((s - m_all) / T)
                // entropy - sum p log q, with log q = s / T - m_all / T - log_z  (without a logit in the list, cross says all)
                double loss = k.entropy - k.cross + k.mass * ((m_list > -INFINITY ? ((double)m_all - (double)m_list) * p.inv_t : 0.0) + log_z);
                if (k.p_rest != 0.0) {
                    if (empty) loss = k.p_rest <= kRestRounding ? loss + 0.0 * z_all : loss + k.p_rest * (double)INFINITY;
                    else loss += k.p_rest * (log(k.p_rest) - (((double)m_rest - (double)m_all) * p.inv_t + log(z_rest) - log_z));
                }
                if (lane == 0) {
                    const bool out_of_it = k.left_out != 0;
                    if (p.loss) p.loss[row] = out_of_it ? 0.0f : (float)(weight * loss);
                    if (p.stats) *stats = out_of_it ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(z_all == z_all ? m_all : (float)nan, (float)z_all, m_rest, (float)z_rest);
                }
            }
            arrive(&sh.done[slot]);
        }
        if (lane == 0 && order < n_live) atomicMin(&sh.lost, order);
    } else {
        // ---------------- compute ----------------
        unsigned n = 0, stage = 0, turn = 0, lives = 0;
        const uint64_t c2 = pack2(p.c, p.c);
        unsigned order = cluster;
        for (; order < n_live; order += p.clusters, ++n) {
            const unsigned slot = n & 1u;
            DistillRow& k = sh.row[slot];
            const DistillList l(list_all + slot * distill_list_bytes(p.K), list_size);
            if (!wait(&sh.listed[slot], (n / 2) & 1u, kSpinLimit)) break;
            const DistillSegment<DT> seg(p, k.row, rank);
            const int* first_of = first_all + slot * (parts_max + 2);
            const int nc = seg.nc, parts = seg.n_tiles * kDistillWarps;
            char* out = kGrad ? p.grad + ((int64_t)seg.b * p.out_b + (int64_t)seg.i * p.out_row) * E::ES : nullptr;
            const bool same = kGrad && ((uintptr_t)seg.in & 15u) == ((uintptr_t)out & 15u);
            uint4* o4 = reinterpret_cast<uint4*>(out + seg.e0 * E::ES);
            const bool live = k.live != 0;
            const unsigned phase = (lives >> slot) & 1u;
            if (live) lives ^= 1u << slot;
            const int drop = p.drop < 0 ? -1 : min(p.drop, seg.n_tiles - 1);
            bool ok = true;
            const int again = kLoss && kGrad && live ? max(0, seg.n_tiles - (int)S) : seg.n_tiles;      // tiles that do not stay: the first ones
            unsigned stay_stage = 0;                                 // of the first that does
            if (kLoss && live) {
                DistillSum s;
                if (tid < seg.scalars) {
                    float x = E::load(seg.in, seg.scalar(p, tid));
                    for (int o = first_of[tid < seg.head ? parts : parts + 1]; o >= 0; o = l.next[o])
                        if (l.thread[o] == tid) x = -INFINITY;
                    s.m = fmaxf(s.m, x);
                    if (x > s.top) distill_raise(p, s, &k.near);
                    s.acc += (double)ex2_approx(fmaf(x - s.base, p.c, -s.ref));
                }
                for (int t = 0; t < seg.n_tiles; ++t) {
                    if (t == again) stay_stage = stage;
                    if (!wait(&sh.full[stage], turn & 1u, t == drop ? kTestSpinLimit : kSpinLimit)) { ok = false; break; }
                    uint4* tile = ring + stage * kDistillTile;
                    const int c0 = t * kDistillTile + tid;
                    constexpr uint32_t ninf = E::ES == 2 ? 0xff80ff80u : 0xff800000u;
                    const int first = first_of[t * kDistillWarps + warp];
                    if (first >= 0) {
                        // listed tokens of this warp's part: each becomes -Inf where it lies (its gradient does not come from there)
                        for (int o = first; o >= 0; o = l.next[o])
                            if (l.thread[o] == tid) {
                                hide_element<DT>(tile + (l.where[o] / 8) * kDistillCompute + tid, l.where[o] & 7);
                                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (the stage's next tile comes after this)
                            }
                    }
                    uint4 w[kDistillEach];
#pragma unroll
                    for (int u = 0; u < kDistillEach; ++u) w[u] = tile[u * kDistillCompute + tid];
                    if ((t + 1) * kDistillTile > nc) {               // the last tile: what lies behind the segment's end
#pragma unroll
                        for (int u = 0; u < kDistillEach; ++u)
                            if (c0 + u * kDistillCompute >= nc) w[u] = make_uint4(ninf, ninf, ninf, ninf);
                    }
                    if (!kGrad || t < again) arrive(&sh.empty[stage]);
                    if (++stage == S) { stage = 0; ++turn; }
                    if (c0 - lane >= nc) continue;                   // nothing of this tile for the warp
                    const float m = E::max4(w[0], w[1], w[2], w[3]);
                    s.m = fmaxf(s.m, m);
                    bool near = true;
                    if (m > s.top) {
                        distill_raise(p, s, &k.near);
                        near = s.base == 0.0f;
                        if (!near) s.acc += tile_terms<DT, true>(w, c2, s);
                    }
                    if (near) s.acc += tile_terms<DT, false>(w, c2, s);
                }
                if (!ok) break;
                float m = s.m, told = told_reference(s);
                double acc = s.acc;
                distill_join(p.c, m, told, acc);
                if (lane == 0) { k.max[warp] = m; k.ref[warp] = told; k.sum[warp] = acc; }
                arrive(&sh.summed[slot]);
            }
            if constexpr (kGrad) {
                if (live && !wait(&sh.known[slot], phase, kSpinLimit)) break;
                const bool zero = !live || k.left_out;
                const float nbase = live ? -k.grad_base : 0.0f, nref = live ? -k.grad_ref : 0.0f, factor = live ? (float)k.factor : 0.0f;
                const bool far = nbase != 0.0f;
                const uint64_t nref2 = pack2(nref, nref), factor2 = pack2(factor, factor);
                if (tid < seg.scalars) {
                    const int64_t v = seg.scalar(p, tid);
                    float g = 0.0f;
                    if (!zero) {
                        g = factor * ex2_approx(fmaf(E::load(seg.in, v) + nbase, p.c, nref));
                        for (int o = first_of[tid < seg.head ? parts : parts + 1]; o >= 0; o = l.next[o])
                            if (l.thread[o] == tid && l.once[o]) g = l.g[o];
                    }
                    store_element<DT>(out, v, g);
                }
                for (int o = 0; o < seg.n_tiles; ++o) {
                    // first those that have stayed, then the others, which come again meanwhile
                    const bool stayed = live && o < seg.n_tiles - again;
                    const int t = stayed ? again + o : o - (seg.n_tiles - again);
                    unsigned at = stage;
                    if (stayed) {
                        at = stay_stage;
                        if (++stay_stage == S) stay_stage = 0;
                    } else if (live) {
                        if (!wait(&sh.full[stage], turn & 1u, !kLoss && t == drop ? kTestSpinLimit : kSpinLimit)) { ok = false; break; }
                        if (++stage == S) { stage = 0; ++turn; }
                    }
                    const uint4* tile = ring + at * kDistillTile;
                    const int first = zero ? -1 : first_of[t * kDistillWarps + warp];
#pragma unroll
                    for (int u = 0; u < kDistillEach; ++u) {
                        const int c = t * kDistillTile + u * kDistillCompute + tid;
                        if (c >= nc) break;
                        uint4 w = make_uint4(0u, 0u, 0u, 0u);
                        if (!zero && far) w = gradient_chunk<DT, true>(tile[u * kDistillCompute + tid], c2, nbase, nref2, factor2);
                        else if (!zero) w = gradient_chunk<DT, false>(tile[u * kDistillCompute + tid], c2, 0.0f, nref2, factor2);
                        if (same) o4[c] = w;
                        else store_chunk<DT>(out, seg.e0 + (int64_t)c * E::EPC, w);
                    }
                    // listed tokens, over what this thread has written
                    for (int o = first; o >= 0; o = l.next[o])
                        if (l.thread[o] == tid && l.once[o])
                            store_element<DT>(out, seg.e0 + (int64_t)(t * kDistillTile + (l.where[o] / 8) * kDistillCompute + tid) * E::EPC + (l.where[o] & 7), l.g[o]);
                    if (live) arrive(&sh.empty[at]);
                }
                if (!ok) break;
            }
            arrive(&sh.done[slot]);
        }
        if (lane == 0 && order < n_live) atomicMin(&sh.lost, order);
    }
    __syncthreads();
    // ---- rows that path or n_rows leave out, and, where a wait ran out, NaN in all that the CTA has not finished ----
    const unsigned lost = sh.lost;
    auto fill = [&](unsigned row, float x) {
        const DistillSegment<DT> seg(p, row, rank);
        if constexpr (kGrad) {
            char* out = p.grad + ((int64_t)seg.b * p.out_b + (int64_t)seg.i * p.out_row) * E::ES;
            if (tid < seg.scalars) store_element<DT>(out, seg.scalar(p, tid), x);
            const uint32_t bits = element_bits<DT>(x), two = DT == CADD_DTYPE_BF16 ? bits | bits << 16 : bits;
            const uint4 w = make_uint4(two, two, two, two);
            const bool same = ((uintptr_t)seg.in & 15u) == ((uintptr_t)out & 15u);
            for (int c = tid; c < seg.nc; c += kDistillThreads) {
                if (same) reinterpret_cast<uint4*>(out + seg.e0 * E::ES)[c] = w;
                else store_chunk<DT>(out, seg.e0 + (int64_t)c * E::EPC, w);
            }
        }
        if (kLoss && rank == 0 && tid == 0) {
            if (p.loss) p.loss[row] = x;
            if (p.stats) reinterpret_cast<float4*>(p.stats)[row] = make_float4(x, x, x, x);
        }
        if (x != 0.0f && tid == 0 && p.status) atomicOr(&p.status[seg.b], CADD_STATUS_INTERNAL_TIMEOUT);
    };
    if constexpr (kGrad) {
        for (unsigned order = cluster; order < (unsigned)p.rows - n_live; order += p.clusters) fill(distill_row(p, sh.map, order, false), 0.0f);
    } else {
        for (unsigned order = blockIdx.x * kDistillThreads + tid; order < (unsigned)p.rows - n_live; order += gridDim.x * kDistillThreads) {
            const unsigned row = distill_row(p, sh.map, order, false);
            if (p.loss) p.loss[row] = 0.0f;
            if (p.stats) reinterpret_cast<float4*>(p.stats)[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    }
    for (unsigned order = lost; order < n_live; order += p.clusters) fill(distill_row(p, sh.map, order, true), __int_as_float(0x7fc00000));
    if (C > 1) { cluster_arrive(); cluster_wait(); }                 // nobody writes to a CTA that has left
}

// Status of one request, where it is asked for.
__global__ void __launch_bounds__(kDistillStatusThreads) distill_status_kernel(DistillParams p) {
    __shared__ int bits;
    const int b = blockIdx.x, tid = threadIdx.x;
    if (tid == 0) bits = 0;
    __syncthreads();
    int st = 0;
    if (p.path ? p.path_len[b] < 0 || p.path_len[b] > min(p.L - 1, p.path_cols) : p.n_rows && (p.n_rows[b] < 0 || p.n_rows[b] > p.L)) st |= CADD_STATUS_BAD_LENGTH;
    const int live = distill_live(p, b);
    for (int64_t n = tid; n < (int64_t)live * p.K; n += kDistillStatusThreads) {
        const int i = (int)(n / p.K), k = (int)(n - (int64_t)i * p.K);
        const int r = !p.path ? i : (i == 0 ? 0 : p.path[(int64_t)b * p.path_cols + i - 1]);
        if (r < 0 || r >= p.R) { st |= CADD_STATUS_BAD_PATH; continue; }
        const int tok = p.token[((int64_t)b * p.R + r) * p.K + k];
        if (tok < -1 || tok >= p.V) st |= CADD_STATUS_BAD_TOKEN;
    }
    if (st) atomicOr(&bits, st);
    __syncthreads();
    if (tid == 0) p.status[b] = bits;
}

}  // namespace cadd
