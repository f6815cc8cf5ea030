// Distillation of the drafter from the target's top tokens: losses and gradients (cadd_distill_args has the definition).
//
// A cluster of CTAs takes one row of drafter's logits, a CTA one contiguous segment of it, which comes to shared memory in tiles of
// 16 KB (bulk copies, each with a barrier).  As the tiles land, every thread adds up the exponentials of its elements that are
// not listed, relative to a power of two at or above its own largest; listed tokens are left out of that sum (their elements
// count as -Inf) and go into the row's statistics one by one, in fp64: the rest's probability is therefore right even where the
// listed tokens leave all but nothing.  The segments' (largest, sum) pairs cross the cluster through distributed shared memory.
// Where the gradient is wanted too, all tiles of the segment have room and stay, and with the statistics known it is formed from them:
// a row is read from memory once and written once.  The loss alone, and the gradient alone (statistics given, no exchange), need a
// tile once, so these walk through a ring of a few tiles and give a CTA more of the row.
#pragma once
#include "common.cuh"
#include "tile_ring.cuh"
#include "packed.cuh"

namespace cadd {

constexpr int kDistillThreads = 256;
constexpr int kDistillMaxC = 8;                                     // CTAs a row at most
constexpr int kDistillTile = 4 * kDistillThreads;                   // 16-byte chunks of one copy: four a thread
constexpr int kDistillMaxTiles = 13;                                // that stay in shared memory: 208 KB
constexpr int kDistillRing = 3;                                     // tiles of the ring, where they do not stay
constexpr int kDistillK = CADD_DISTILL_MAX_K;
static_assert(kDistillK <= kDistillThreads, "one thread an entry");
constexpr float kDistillLowest = -1.0e30f;                          // logits below count as -Inf; also the reference of an empty sum
constexpr double kRestRounding = 0x1p-20;

struct DistillParams {
    const char* logits;
    char* grad;
    int64_t V, in_b, in_row, out_b, out_row;
    int L, R, K, path_cols, rest;
    int C, chunks_max;                            // CTAs a row; chunks of a segment at most
    float c;                                      // log2(e) / T
    double inv_t;
    const int32_t *token, *path, *path_len, *n_rows;
    const double *value, *lse;
    const float *weight, *grad_loss;
    float *loss, *stats;
    int32_t* status;
    int drop;                                     // test hook: this tile of every segment is never copied (-1: none)
};

// Behind this: int first_of[groups + 2], the first entry of the list in each group of 32 consecutive chunks (-1: none; the last
// two groups are the row's scalar head and tail), then the segment.
struct DistillShared {
    alignas(8) uint64_t full[kDistillMaxTiles];
    int sent[kDistillMaxTiles];                   // last tile sent for into each stage, -1: none
    unsigned released[kDistillRing];              // ring: warps done with the stage's current tile
    double value[kDistillK];                      // entries of the list: target's logit
    double prob[kDistillK];                       // entries: p
    double peer_sum[kDistillMaxC];
    double warp_sum[kDistillThreads / 32];
    double factor;                                // of the exponentials in the gradient of tokens that are not listed
    float peer_max[kDistillMaxC], peer_ref[kDistillMaxC];
    float warp_max[kDistillThreads / 32], warp_ref[kDistillThreads / 32];
    float logit[kDistillK];                       // entries: drafter's logit
    float g[kDistillK];                           // entries: gradient of their token
    int token[kDistillK];                         // entries: token, -1 where there is none
    int chunk[kDistillK];                         // entries: chunk of the segment
    int16_t next[kDistillK];                      // next entry of the same group, -1: none
    uint8_t elem[kDistillK], once[kDistillK];     // element of the chunk; 1: the token's first entry
    float ref;                                    // reference exponent of the gradient's exponentials
    int twice;                                    // some token is listed more than once
    int left_out;
    int timeout;
};
__host__ __device__ inline size_t distill_first_bytes(int chunks) { return (((size_t)(chunks + 31) / 32 + 2) * 4 + 127) & ~(size_t)127; }
__host__ __device__ inline size_t distill_shared_bytes() { return (sizeof(DistillShared) + 127) & ~(size_t)127; }
inline size_t distill_smem_bytes(int chunks, int room) { return distill_shared_bytes() + distill_first_bytes(chunks) + (size_t)room * 16; }

__device__ __forceinline__ uint32_t peer_address(const void* p, unsigned rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
// 2^n for integer-valued n <= 0, 0 below the normal range.
__device__ __forceinline__ double pow2_down(float n) {
    return n > -1000.0f ? __hiloint2double((1023 + (int)n) << 20, 0) : (n == n ? 0.0 : (double)n);
}

// Positions of request b that are learnt from.
__device__ __forceinline__ int distill_live(const DistillParams& p, int b) {
    if (p.path) {
        const int n = p.path_len[b], most = min(p.L - 1, p.path_cols);
        return 1 + max(0, min(n, most));
    }
    return p.n_rows ? max(0, min(p.n_rows[b], p.L)) : p.L;
}

// -Inf in the elements of a chunk whose bit is set.
template <int DT>
__device__ __forceinline__ void blank(uint4& w, uint32_t bits) {
    uint32_t* x = &w.x;
    if constexpr (DT == CADD_DTYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t gone = ((bits >> (2 * i)) & 1u ? 0x0000ffffu : 0u) | ((bits >> (2 * i + 1)) & 1u ? 0xffff0000u : 0u);
            x[i] = (x[i] & ~gone) | (0xff80ff80u & gone);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (bits >> i) & 1u ? 0xff800000u : x[i];
    }
}
template <int DT>
__device__ __forceinline__ uint4 pack_chunk(const float* f) {
    if constexpr (DT == CADD_DTYPE_BF16) {
        uint4 w;
        uint32_t* x = &w.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            x[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return w;
    } else {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
}
template <int DT> __device__ __forceinline__ void store_element(char* row, int64_t i, float x) {
    if constexpr (DT == CADD_DTYPE_BF16) ((__nv_bfloat16*)row)[i] = __float2bfloat16_rn(x);
    else ((float*)row)[i] = x;
}

// A thread's running sum of 2^(x c - ref) over the elements it has seen, ref an integer at or above the largest x c.
struct DistillSum {
    float m, ref;
    double acc;
};
__device__ __forceinline__ void distill_raise(DistillSum& s, float m, float c) {
    s.m = m;
    const float ref = fmaxf(ceilf(m * c), kDistillLowest);
    if (ref > s.ref) {
        s.acc *= pow2_down(s.ref - ref);
        s.ref = ref;
    }
}
__device__ __forceinline__ float warp_max(float x) {                // NaN ignored
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
// The warp's sums together, in every lane.
__device__ __forceinline__ void distill_join(DistillSum& s) {
    const float m = warp_max(s.m), ref = warp_max(s.ref);
    s.acc *= pow2_down(s.ref - ref);
    s.m = m;
    s.ref = ref;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s.acc += __shfl_xor_sync(kFullMask, s.acc, o);
}
// Packed sums of the exponentials of a chunk's even and odd elements.
template <int DT>
__device__ __forceinline__ uint64_t chunk_terms(const uint4& w, uint64_t c2, uint64_t nref2) {
    using E = Elem<DT>;
    float f[E::EPC];
    E::unpack(w, f);
    uint64_t pr[E::EPC / 2];
#pragma unroll
    for (int q = 0; q < E::EPC; q += 2) {
        float t0, t1;
        unpack2(fma2(pack2(f[q], f[q + 1]), c2, nref2), t0, t1);
        pr[q / 2] = pack2(ex2_approx(t0), ex2_approx(t1));
    }
    uint64_t r = add2(pr[0], pr[1]);
    if constexpr (E::EPC == 8) r = add2(r, add2(pr[2], pr[3]));
    return r;
}

// kLoss: statistics and loss are computed here; otherwise they are given.  kGrad: the gradient is written.
template <int DT, bool kLoss, bool kGrad>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(DistillParams p) {
    using E = Elem<DT>;
    extern __shared__ __align__(128) unsigned char distill_smem_raw[];
    DistillShared& sh = *reinterpret_cast<DistillShared*>(distill_smem_raw);
    int* first_of = reinterpret_cast<int*>(distill_smem_raw + distill_shared_bytes());
    const uint4* seg = reinterpret_cast<const uint4*>(distill_smem_raw + distill_shared_bytes() + distill_first_bytes(p.chunks_max));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr bool kRing = !(kLoss && kGrad);
    const unsigned C = (unsigned)p.C, row = blockIdx.x / C, rank = blockIdx.x - row * C;
    const int b = (int)(row / (unsigned)p.L), i = (int)(row - (unsigned)b * (unsigned)p.L);

    // ---- the row, and the target's row for it ----
    const char* in = p.logits + ((int64_t)b * p.in_b + (int64_t)i * p.in_row) * E::ES;
    char* out = kGrad ? p.grad + ((int64_t)b * p.out_b + (int64_t)i * p.out_row) * E::ES : nullptr;
    const RowSplit sp = split_row<DT>(in, p.V);
    const int per = (sp.n_chunks + (int)C - 1) / (int)C;
    const int s0 = min(sp.n_chunks, (int)rank * per), nc = min(per, sp.n_chunks - s0);     // this CTA's chunks
    const int64_t e0 = sp.head + (int64_t)s0 * E::EPC;                                      // token of its first chunk
    const int scalars = (rank == 0 ? sp.head : 0) + (rank == C - 1 ? sp.tail : 0);
    // token of thread tid's scalar element, tid < scalars
    const int64_t mine_scalar = rank == 0 && tid < sp.head ? tid : p.V - sp.tail + (tid - (rank == 0 ? sp.head : 0));
    int r = i;
    bool left_out = i >= distill_live(p, b);
    const float weight = p.weight ? p.weight[row] : 1.0f;
    left_out = left_out || weight == 0.0f;
    if (!left_out && p.path) r = i == 0 ? 0 : p.path[(int64_t)b * p.path_cols + i - 1];
    left_out = left_out || r < 0 || r >= p.R;
    const bool same = kGrad && ((uintptr_t)in & 15u) == ((uintptr_t)out & 15u);
    // gradient 0 of a row that is left out
    auto write_zeros = [&]() {
        if constexpr (kGrad) {
            if (tid < scalars) store_element<DT>(out, mine_scalar, 0.0f);
            if (same) {
                uint4* o4 = reinterpret_cast<uint4*>(out + e0 * E::ES);
                for (int k = tid; k < nc; k += kDistillThreads) o4[k] = make_uint4(0u, 0u, 0u, 0u);
            } else {
                for (int k = tid; k < nc * E::EPC; k += kDistillThreads) store_element<DT>(out, e0 + k, 0.0f);
            }
        }
        if (kLoss && rank == 0 && tid == 0) {
            if (p.loss) p.loss[row] = 0.0f;
            if (p.stats) reinterpret_cast<float4*>(p.stats)[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    };
    if (left_out) {                                                  // the same for every CTA of the cluster
        write_zeros();
        return;
    }
    if (kLoss && C > 1) cluster_arrive();                                     // waited for before the first access to another CTA's memory

    // ---- copies under way, then the list ----
    const int n_tiles = (nc + kDistillTile - 1) / kDistillTile;
    const int drop = p.drop < 0 ? -1 : min(p.drop, n_tiles - 1);
    constexpr int stages = kRing ? kDistillRing : kDistillMaxTiles;
    auto stage = [](int t) { return kRing ? t % kDistillRing : t; };
    auto parity = [](int t) { return kRing ? (unsigned)(t / kDistillRing) & 1u : 0u; };
    auto issue = [&](int t) {
        if (t == drop) return;                                       // test hook: this copy is never made
        const int c0 = t * kDistillTile, s = stage(t);
        const unsigned bytes = (unsigned)min(kDistillTile, nc - c0) * 16u;
        *(volatile int*)&sh.sent[s] = t;
        mbar_arrive_expect_tx(&sh.full[s], bytes);
        bulk_load((void*)(seg + s * kDistillTile), in + e0 * E::ES + (int64_t)c0 * 16, bytes, &sh.full[s]);
    };
    // a warp is done with tile t: the last one sends for the tile that takes its place
    auto release = [&](int t) {
        if constexpr (kRing) {
            __syncwarp();
            const int s = t % kDistillRing;
            if (lane == 0 && atomicAdd(&sh.released[s], 1u) == kDistillThreads / 32 - 1) {
                atomicExch(&sh.released[s], 0u);
                if (t + kDistillRing < n_tiles) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    issue(t + kDistillRing);
                }
            }
        }
    };
    auto landed = [&](int t) {
        return __all_sync(kFullMask, mbar_wait_limited(&sh.full[stage(t)], parity(t), tile_wait_limit(t, drop))) != 0;
    };
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&sh.full[s], 1);
        for (int s = 0; s < stages; ++s) sh.sent[s] = -1;
        for (int s = 0; s < kDistillRing; ++s) sh.released[s] = 0;
        sh.timeout = 0;
        sh.twice = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int t = 0; t < stages && t < n_tiles; ++t) issue(t);
    }
    const int groups = (nc + 31) / 32;
    for (int k = tid; k < groups + 2; k += kDistillThreads) first_of[k] = -1;
    int tok = -1;
    if (tid < p.K) {
        const int64_t at = ((int64_t)b * p.R + r) * p.K + tid;
        tok = p.token[at];
        if (tok < 0 || tok >= p.V) tok = -1;
        sh.token[tid] = tok;
        sh.value[tid] = p.value[at];
        sh.logit[tid] = kLoss && tok >= 0 ? E::load(in, tok) : 0.0f;
    }
    __syncthreads();
    if (tok >= 0) {
        bool once = true;
        for (int k = 0; k < tid; ++k) once = once && sh.token[k] != tok;
        sh.once[tid] = once;
        if (!once) sh.twice = 1;
        // where in this CTA's segment the token lies
        int group = -1, e = 0, c = 0;
        if (tok >= e0 && tok < e0 + (int64_t)nc * E::EPC) {
            c = (int)((tok - e0) / E::EPC);
            e = (int)((tok - e0) % E::EPC);
            group = c / 32;
        } else if (rank == 0 && tok < sp.head) { c = tok; group = groups; }
        else if (rank == C - 1 && tok >= p.V - sp.tail) { c = (int)(tok - (p.V - sp.tail)) + (rank == 0 ? sp.head : 0); group = groups + 1; }
        sh.chunk[tid] = c;
        sh.elem[tid] = (uint8_t)e;
        if (group >= 0) {
            if (!kLoss) sh.logit[tid] = E::load(in, tok);
            sh.next[tid] = (int16_t)atomicExch(&first_of[group], tid);
        }
    }
    __syncthreads();

    // ---- the target's probabilities (warp 0; the others go on to the tiles) ----
    double p_rest = 0.0, entropy = 0.0, mass = 0.0;                  // warp 0, all lanes: entropy = sum p log p of the entries
    if (warp == 0) {
        double top = -INFINITY;
        bool any = false;
        if (!p.rest) {
            for (int k = lane; k < p.K; k += 32)
                if (sh.token[k] >= 0) {
                    top = fmax(top, sh.value[k]);                    // (NaN shows in the sum)
                    any = any || !(sh.value[k] == -INFINITY);
                }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmax(top, __shfl_xor_sync(kFullMask, top, o));
        } else {
            top = p.lse ? p.lse[(int64_t)b * p.R + r] / p.inv_t : 0.0;
        }
        double sum = 0.0;
        for (int k = lane; k < p.K; k += 32) {
            double q = 0.0;
            if (sh.token[k] >= 0) {
                q = exp((sh.value[k] - top) * p.inv_t);
                if (p.rest) any = true;
            }
            sh.prob[k] = q;
            sum += q;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
        any = __any_sync(kFullMask, any);
        const double scale = p.rest ? 1.0 : 1.0 / sum, log_sum = p.rest ? 0.0 : log(sum);
        if (p.rest) p_rest = sum < 1.0 ? 1.0 - sum : (sum == sum ? 0.0 : sum);
        for (int k = lane; k < p.K; k += 32) {
            const double q = sh.prob[k] * scale;
            sh.prob[k] = q;
            if (q > 0.0) entropy += q * ((sh.value[k] - top) * p.inv_t - log_sum);
            else if (!(q == 0.0)) entropy = q;
            mass += q;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            entropy += __shfl_xor_sync(kFullMask, entropy, o);
            mass += __shfl_xor_sync(kFullMask, mass, o);
        }
        if (lane == 0) sh.left_out = any ? 0 : 1;
    }

    // bits of the elements of chunk c that are listed
    auto listed = [&](int first, int c) {
        uint32_t bits = 0;
        for (int k = first; k >= 0; k = sh.next[k])
            if (sh.chunk[k] == c) bits |= 1u << sh.elem[k];
        return bits;
    };
    bool timeout = false;
    float m_rest = 0.0f, m_all = 0.0f;
    double z_rest = 0.0, z_all = 0.0;
    if constexpr (kLoss) {
        // ---- sum over the tokens that are not listed ----
        DistillSum s{-INFINITY, kDistillLowest, 0.0};
        const uint64_t c2 = pack2(p.c, p.c);
        if (tid < scalars) {
            float x = E::load(in, mine_scalar);
            const int at = mine_scalar < sp.head ? groups : groups + 1;
            if (listed(first_of[at], tid)) x = -INFINITY;
            distill_raise(s, x, p.c);
            s.acc += (double)ex2_approx(fmaf(x, p.c, -s.ref));
            if (!(x == x)) s.m = -INFINITY;
        }
        for (int t = 0; t < n_tiles; ++t) {
            if (!landed(t)) { timeout = true; break; }
            const uint4* tile = seg + stage(t) * kDistillTile;
            const int c0 = t * kDistillTile + tid;
            constexpr uint32_t ninf = E::ES == 2 ? 0xff80ff80u : 0xff800000u;
            uint4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = c0 + u * kDistillThreads;
                w[u] = make_uint4(ninf, ninf, ninf, ninf);
                if (c < nc) {
                    w[u] = tile[u * kDistillThreads + tid];
                    const int first = first_of[c / 32];
                    if (first >= 0) blank<DT>(w[u], listed(first, c));
                }
            }
            release(t);
            const float m = E::max4(w[0], w[1], w[2], w[3]);
            if (m > s.m) distill_raise(s, m, p.c);
            const uint64_t nref2 = pack2(-s.ref, -s.ref);
            const uint64_t sum2 = add2(add2(chunk_terms<DT>(w[0], c2, nref2), chunk_terms<DT>(w[1], c2, nref2)),
                                       add2(chunk_terms<DT>(w[2], c2, nref2), chunk_terms<DT>(w[3], c2, nref2)));
            float a0, a1;
            unpack2(sum2, a0, a1);
            s.acc += (double)(a0 + a1);
        }
        // ---- threads, warps, CTAs ----
        distill_join(s);
        if (lane == 0) { sh.warp_max[warp] = s.m; sh.warp_ref[warp] = s.ref; sh.warp_sum[warp] = s.acc; }
        if (timeout) sh.timeout = 1;
        __syncthreads();
        timeout = sh.timeout != 0;
        if (warp == 0) {
            const bool in_use = lane < kDistillThreads / 32;
            s = DistillSum{in_use ? sh.warp_max[lane] : -INFINITY, in_use ? sh.warp_ref[lane] : kDistillLowest, in_use ? sh.warp_sum[lane] : 0.0};
            distill_join(s);
            if (timeout) s.acc = __longlong_as_double(0x7ff8000000000000ll);
        }
        if (C > 1) {
            cluster_wait();
            if (warp == 0 && lane < (int)C) {
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_address(&sh.peer_max[rank], lane)), "f"(s.m) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_address(&sh.peer_ref[rank], lane)), "f"(s.ref) : "memory");
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(peer_address(&sh.peer_sum[rank], lane)), "d"(s.acc) : "memory");
            }
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            if (warp == 0) {
                const bool in_use = lane < (int)C;
                s = DistillSum{in_use ? sh.peer_max[lane] : -INFINITY, in_use ? sh.peer_ref[lane] : kDistillLowest, in_use ? sh.peer_sum[lane] : 0.0};
                distill_join(s);
            }
        }
        if (warp == 0) {
            m_rest = s.m >= kDistillLowest ? s.m : -INFINITY;
            z_rest = m_rest > -INFINITY ? s.acc * kEx2BiasFix * exp2((double)s.ref - (double)m_rest * (double)p.c) : (s.acc == s.acc ? 0.0 : s.acc);
            m_all = m_rest;
            bool bad = !(s.acc == s.acc);
            for (int k = lane; k < p.K; k += 32)
                if (sh.token[k] >= 0) {
                    const float x = sh.logit[k];
                    if (!(x == x)) bad = true;
                    if (x >= kDistillLowest) m_all = fmaxf(m_all, x);
                }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(kFullMask, m_all, o));
            double z = 0.0;
            for (int k = lane; k < p.K; k += 32)
                if (sh.token[k] >= 0 && sh.once[k] && sh.logit[k] >= kDistillLowest) z += exp(((double)sh.logit[k] - (double)m_all) * p.inv_t);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(kFullMask, z, o);
            if (m_rest > -INFINITY) z += z_rest * exp(((double)m_rest - (double)m_all) * p.inv_t);
            z_all = __any_sync(kFullMask, bad) ? __longlong_as_double(0x7ff8000000000000ll) : z;
        }
    } else if (warp == 0) {
        const float4 st = reinterpret_cast<const float4*>(p.stats)[row];
        m_all = st.x; z_all = (double)st.y; m_rest = st.z; z_rest = (double)st.w;
    }

    // ---- loss and the gradient's factors (warp 0) ----
    if (warp == 0) {
        const double nan = __longlong_as_double(0x7ff8000000000000ll);
        if (!(m_all > -INFINITY)) z_all = nan;                       // a row without a finite logit
        const bool empty = !(m_rest > -INFINITY);                    // no token is left beside the list
        const double log_z = log(z_all), total = mass + p_rest;
        const double w = (p.grad_loss ? (double)p.grad_loss[row] : 1.0) * (double)weight * p.inv_t;
        double cross = 0.0;                                          // sum p log q
        for (int k = lane; k < p.K; k += 32) {
            if (sh.token[k] < 0) continue;
            const double x = sh.logit[k] < kDistillLowest ? -INFINITY : (double)sh.logit[k];
            const double log_q = (x - (double)m_all) * p.inv_t - log_z;
            if (sh.prob[k] != 0.0) cross += sh.prob[k] * log_q;
            double mine = sh.prob[k];
            if (sh.twice)
                for (int n = k + 1; n < p.K; ++n)
                    if (sh.token[n] == sh.token[k]) mine += sh.prob[n];
            if (kGrad) sh.g[k] = (float)(w * (total * exp(log_q) - mine));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) cross += __shfl_xor_sync(kFullMask, cross, o);
        if (kLoss && rank == 0 && lane == 0) {
            double loss = entropy - cross;
            if (p_rest != 0.0) {
                if (empty) loss = p_rest <= kRestRounding ? loss + 0.0 * z_all : loss + p_rest * (double)INFINITY;
                else loss += p_rest * (log(p_rest) - (((double)m_rest - (double)m_all) * p.inv_t + log(z_rest) - log_z));
            }
            const bool out_of_it = sh.left_out != 0;
            if (p.loss) p.loss[row] = out_of_it ? 0.0f : (float)((double)weight * loss);
            if (p.stats) reinterpret_cast<float4*>(p.stats)[row] =
                out_of_it ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(z_all == z_all ? m_all : (float)nan, (float)z_all, m_rest, (float)z_rest);
        }
        if (kGrad && lane == 0) {
            // an exponential below is exp((s - m_rest) / T) * 2^(m_rest c - ref)
            const float ref = empty ? 0.0f : ceilf(m_rest * p.c);
            double f = empty ? 0.0 * z_all : total * exp(((double)m_rest - (double)m_all) * p.inv_t) / z_all - (p_rest != 0.0 ? p_rest / z_rest : 0.0);
            if (!empty) f *= exp2((double)ref - (double)m_rest * (double)p.c);
            sh.ref = ref;
            sh.factor = w * f;
        }
    }
    if constexpr (kGrad) {
        __syncthreads();
        if (sh.left_out) write_zeros();
        else {
            // ---- the gradient ----
            const float nref = -sh.ref;
            float factor = (float)sh.factor;
            if (timeout) factor = __int_as_float(0x7fc00000);
            if (tid < scalars) {
                const int at = mine_scalar < sp.head ? groups : groups + 1;
                float g = factor * ex2_approx(fmaf(E::load(in, mine_scalar), p.c, nref));
                for (int k = first_of[at]; k >= 0; k = sh.next[k])
                    if (sh.chunk[k] == tid && sh.once[k]) g = sh.g[k];
                store_element<DT>(out, mine_scalar, g);
            }
            const uint64_t c2 = pack2(p.c, p.c), nref2 = pack2(nref, nref);
            uint4* o4 = reinterpret_cast<uint4*>(out + e0 * E::ES);
            for (int t = 0; t < n_tiles; ++t) {
                if (!kLoss && !timeout && !landed(t)) timeout = true;
                if (!kLoss && timeout) factor = __int_as_float(0x7fc00000);
                const uint4* tile = seg + stage(t) * kDistillTile;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = t * kDistillTile + u * kDistillThreads + tid;
                    if (c >= nc) break;
                    float f[E::EPC];
                    E::unpack(tile[u * kDistillThreads + tid], f);
#pragma unroll
                    for (int q = 0; q < E::EPC; q += 2) {
                        float t0, t1;
                        unpack2(fma2(pack2(f[q], f[q + 1]), c2, nref2), t0, t1);
                        f[q] = factor * ex2_approx(t0);
                        f[q + 1] = factor * ex2_approx(t1);
                    }
                    const int first = first_of[c / 32];
                    if (first >= 0)
                        for (int k = first; k >= 0; k = sh.next[k])
                            if (sh.chunk[k] == c && sh.once[k]) {
#pragma unroll
                                for (int q = 0; q < E::EPC; ++q)
                                    if (q == sh.elem[k]) f[q] = sh.g[k];
                            }
                    if (same) o4[c] = pack_chunk<DT>(f);
                    else {
#pragma unroll
                        for (int q = 0; q < E::EPC; ++q) store_element<DT>(out, e0 + (int64_t)c * E::EPC + q, f[q]);
                    }
                }
                if (!timeout) release(t);
            }
        }
    }
    // No CTA leaves with a copy of its own in flight.  All tiles have been waited for, but where a wait ran out or the list left the
    // row out before its first tile: then the last tile sent for in each stage is, once no warp can send for another.
    if constexpr (!kLoss) {
        if (timeout) sh.timeout = 1;
        __syncthreads();
    }
    if (tid == 0 && (sh.timeout || (!kLoss && sh.left_out))) {
        for (int s = 0; s < stages; ++s)
            if (sh.sent[s] >= 0) mbar_wait_bounded(&sh.full[s], parity(sh.sent[s]));
        if (sh.timeout && p.status) atomicOr(&p.status[b], CADD_STATUS_INTERNAL_TIMEOUT);
    }
}

// Status of one request, where it is asked for.
__global__ void __launch_bounds__(kDistillThreads) distill_status_kernel(DistillParams p) {
    __shared__ int bits;
    const int b = blockIdx.x, tid = threadIdx.x;
    if (tid == 0) bits = 0;
    __syncthreads();
    int st = 0;
    if (p.path ? p.path_len[b] < 0 || p.path_len[b] > min(p.L - 1, p.path_cols) : p.n_rows && (p.n_rows[b] < 0 || p.n_rows[b] > p.L)) st |= CADD_STATUS_BAD_LENGTH;
    const int live = distill_live(p, b);
    for (int64_t n = tid; n < (int64_t)live * p.K; n += kDistillThreads) {
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
