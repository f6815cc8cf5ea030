// Penalties, biases and grammar masks on the logits of a tree's rows (cadd_adjust_args has the definition).
//
// A CTA takes a tile of consecutive tokens (8 KB of logits) of some rows of one request.  It first gathers what its tokens have
// in common over the rows: how often each stands in the history (a table in shared memory), the sum of its biases, and a list of
// the tokens with either, in order.  A history is as long as many tiles, so the CTAs of a cluster, consecutive tiles of the
// same rows, share it: each reads a part and counts into the tables of all (distributed shared memory).  Then a warp takes a row's
// piece of the tile at a time:
//   into another array: the piece comes to shared memory by a bulk copy, the tokens that penalties or biases concern are replaced there,
//     what the mask hides is set, and a bulk copy takes it to its place; the copy of the warp's first piece is under way meanwhile;
//   in place: the same on memory itself, where only what changes is written (and read).
// Tokens of a row's own path are computed before the list's and written after them, from the input's value and their own count.
#pragma once
#include "common.cuh"
#include "tile_ring.cuh"

namespace cadd {

constexpr int kAdjustThreads = 256;
constexpr int kAdjustWarps = kAdjustThreads / 32;
constexpr int kAdjustTileBytes = 8192;         // of a row: what a warp's buffer holds
constexpr int kAdjustRows = 32;                // rows a CTA takes at most
constexpr int kAdjustMaxC = 8;                 // CTAs that share a history
constexpr int kMaxPath = 65;                   // nodes of a path: the deepest tree there is, and its root
constexpr uint32_t kInPrompt = 1u, kHasBias = 2u, kOnce = 4u;      // a token's word in the table: two flags, then n_out of the history

struct AdjustParams {
    const char* in;
    char* out;
    int64_t V, in_b, in_row, out_b, out_row;
    int batch, R, tiles, groups, rows_per_cta, part_shift, C;      // pieces of a row's tile: 1 << part_shift
    int n_bias, history_cols, n_allowed, words;
    bool in_place, penalised;
    int drop;                                                       // test hook: 1: no warp's first copy is ever made
    const int32_t *n_nodes, *token_ids, *parent_idx, *history, *history_len, *prompt_len, *bias_token, *allowed_row;
    int64_t history_stride;
    const float *repetition, *presence, *frequency, *bias;
    const uint32_t* allowed;
    int32_t* status;
};

template <int DT> constexpr int kAdjustTile = kAdjustTileBytes / Elem<DT>::ES;   // tokens

// Behind this, as far as the call needs them (see adjust_layout): the warps' buffers, the table, the list, the sums of biases.
struct AdjustShared {
    alignas(8) uint64_t full[kAdjustWarps];    // a warp's piece has landed
    int32_t mask_row[kAdjustRows];             // row of `allowed` of each of the CTA's rows, -1: none
    int path_n[kAdjustRows];
    uint16_t path[kAdjustRows][kMaxPath];      // tokens of each row's path that lie in the tile
    int list_from[kAdjustWarps + 1];           // the list's entries of each eighth of the tile
    int twice;                                 // some token has two biases
};
constexpr int kAdjustBuffer = kAdjustTileBytes + 16;                // of one warp: the piece keeps its distance from a 16-byte boundary
struct AdjustLayout { int buffers, table, list, bias, bytes; };
__host__ __device__ inline AdjustLayout adjust_layout(int tile, bool in_place, bool sparse, bool biased) {
    AdjustLayout l;
    l.buffers = (int)((sizeof(AdjustShared) + 127) & ~(size_t)127);
    l.table = l.buffers + (in_place ? 0 : kAdjustWarps * kAdjustBuffer);
    l.list = l.table + (sparse ? tile * 4 : 0);
    l.bias = l.list + (sparse ? tile * 2 : 0);
    l.bytes = l.bias + (biased ? tile * 4 : 0);
    return l;
}

__device__ __forceinline__ int adjust_live(const AdjustParams& p, int b) {
    int n = p.n_nodes ? p.n_nodes[b] : p.R - 1;
    return n < -1 ? 0 : (n > p.R - 1 ? p.R : n + 1);
}
__device__ __forceinline__ int adjust_history(const AdjustParams& p, int b, int* prompt) {
    int n = p.history_len ? p.history_len[b] : p.history_cols;
    n = n < 0 ? 0 : (n > p.history_cols ? p.history_cols : n);
    int q = p.prompt_len ? p.prompt_len[b] : 0;
    *prompt = q < 0 ? 0 : (q > n ? n : q);
    return n;
}
// Row of `allowed` for a row of the request, or NULL.
__device__ __forceinline__ const uint32_t* adjust_mask(const AdjustParams& p, int b, int j) {
    if (!p.allowed) return nullptr;
    const int m = p.allowed_row[(int64_t)b * p.R + j];
    return m < 0 || m >= p.n_allowed ? nullptr : p.allowed + (int64_t)m * p.words;
}

// -Inf in the elements of a chunk whose bit is clear.
template <int DT>
__device__ __forceinline__ void hide(uint4& w, uint32_t bits) {
    uint32_t* x = &w.x;
    if constexpr (DT == CADD_DTYPE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t keep = ((bits >> (2 * i)) & 1u ? 0x0000ffffu : 0u) | ((bits >> (2 * i + 1)) & 1u ? 0xffff0000u : 0u);
            x[i] = (x[i] & keep) | (0xff80ff80u & ~keep);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (bits >> i) & 1u ? x[i] : 0xff800000u;
    }
}
template <int DT> struct Raw;                  // an element's bits
template <> struct Raw<CADD_DTYPE_BF16> {
    using T = uint16_t;
    static constexpr T ninf = 0xff80u, nan = 0x7fc0u;
    static __device__ __forceinline__ T round(double x) { return __bfloat16_as_ushort(__double2bfloat16(x)); }
};
template <> struct Raw<CADD_DTYPE_FP32> {
    using T = uint32_t;
    static constexpr T ninf = 0xff800000u, nan = 0x7fc00000u;
    static __device__ __forceinline__ T round(double x) { return __float_as_uint((float)x); }
};

// What penalties make of a logit: n_out = times, seen: n_all > 0.
struct Penalty {
    double rep, inv, pres, freq;
};
__device__ __forceinline__ double penalised(const Penalty& q, double x, uint32_t times, bool seen) {
    if (seen) x *= x > 0.0 ? q.inv : q.rep;    // (x / rep to 2^-52, long before the rounding to fp32 or bf16)
    if (times > 0u) x -= q.freq * (double)times + q.pres;
    return x;
}

// What a mask hides of n elements at x, whose first is token v (a multiple of 32): x lies in shared memory, or is memory itself.  A warp.
template <int DT, bool kShared>
__device__ __forceinline__ void mask_piece(char* x, int n, const uint32_t* mask, int words, int64_t v, const uint32_t (&first)[kAdjustTileBytes / Elem<DT>::ES / 1024]) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    constexpr int kRegs = kAdjustTileBytes / E::ES / 1024;          // words of the mask a lane holds: 4 or 2
    constexpr int kPer = 32 / E::EPC;                               // chunks a word covers: 4 or 8
    const int lane = threadIdx.x & 31;
    const int mis = (int)(((uintptr_t)x & 15u) / E::ES);
    const int head = min(n, mis ? E::EPC - mis : 0), nc = (n - head) / E::EPC, tail = n - head - nc * E::EPC;
    // the head's and tail's elements, and the bits of 32 elements each from the head on
    if (lane < head + tail) {
        const int i = lane < head ? lane : n - tail + (lane - head);
        if (!((mask[(v + i) >> 5] >> (i & 31)) & 1u)) ((T*)x)[i] = Raw<DT>::ninf;
    }
    uint32_t word[kRegs];
    const int w0 = (int)(v >> 5);
#pragma unroll
    for (int k = 0; k < kRegs; ++k) {
        word[k] = first[k];
        if (head) {
            uint32_t up = __shfl_down_sync(kFullMask, first[k], 1);
            const uint32_t wrap = k + 1 < kRegs ? __shfl_sync(kFullMask, first[k + 1 < kRegs ? k + 1 : k], 0) : 0u;
            if (lane == 31) up = wrap;
            const int at = w0 + 32 * k + lane + 1;
            if (lane == 31 && k + 1 == kRegs && at < words && 32 * (32 * k + lane + 1) < n) up = mask[at];
            word[k] = __funnelshift_r(first[k], up, head);
        }
    }
    uint4* x4 = (uint4*)(x + head * E::ES);
    constexpr uint32_t kAll = (1u << E::EPC) - 1u;
    constexpr uint32_t ninf2 = E::ES == 2 ? 0xff80ff80u : 0xff800000u;
    constexpr int kStep = 4;                                        // chunks of a lane under way
#pragma unroll
    for (int i0 = 0; i0 < kAdjustTileBytes / 512; i0 += kStep) {
        if (32 * i0 >= nc) break;
        uint4 w[kStep];
        uint32_t bits[kStep];
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
            constexpr int kWordsPerStep = 32 / kPer;                // 8 or 4
            const int at = (i0 + u) * kWordsPerStep;
            const uint32_t mine = __shfl_sync(kFullMask, word[at / 32], at % 32 + lane / kPer);
            const int c = 32 * (i0 + u) + lane;
            bits[u] = c < nc ? (mine >> ((lane % kPer) * E::EPC)) & kAll : kAll;
            w[u] = make_uint4(ninf2, ninf2, ninf2, ninf2);
            if (bits[u] != kAll && bits[u] != 0u) w[u] = x4[c];
        }
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
            const int c = 32 * (i0 + u) + lane;
            if (bits[u] != kAll) {
                hide<DT>(w[u], bits[u]);
                x4[c] = w[u];
            }
        }
    }
}

__device__ __forceinline__ void adjust_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int DT, bool kInPlace>
__global__ void __launch_bounds__(kAdjustThreads, kInPlace ? 4 : 2) adjust_kernel(AdjustParams p) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    constexpr int kTile = kAdjustTile<DT>;
    extern __shared__ __align__(128) unsigned char adjust_smem_raw[];
    AdjustShared& sh = *reinterpret_cast<AdjustShared*>(adjust_smem_raw);
    const bool sparse = p.penalised || p.n_bias > 0;
    const AdjustLayout lay = adjust_layout(kTile, kInPlace, sparse, p.n_bias > 0);
    uint32_t* table = reinterpret_cast<uint32_t*>(adjust_smem_raw + lay.table);
    uint16_t* list = reinterpret_cast<uint16_t*>(adjust_smem_raw + lay.list);
    float* bias_of = reinterpret_cast<float*>(adjust_smem_raw + lay.bias);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned padded = (unsigned)((p.tiles + p.C - 1) / p.C * p.C);
    const unsigned bg = blockIdx.x / padded;
    const int tile = (int)(blockIdx.x - bg * padded);
    const int b = (int)(bg / (unsigned)p.groups), g = (int)(bg - (unsigned)b * (unsigned)p.groups);
    const int live = adjust_live(p, b);
    const int j0 = g * p.rows_per_cta, j1 = min(live, j0 + p.rows_per_cta);
    if (j0 >= j1) return;                                           // the same for every CTA of a cluster
    const int64_t v0 = (int64_t)tile * kTile;
    const int n = (int)max((int64_t)0, min((int64_t)kTile, p.V - v0));     // 0: a CTA that only helps with the history
    const int parts = 1 << p.part_shift, piece = kTile >> p.part_shift;
    const int units = (j1 - j0) << p.part_shift;                   // a row's pieces one after the other

    struct Unit { char *src, *dst; int row, e0, n; };
    auto unit_at = [&](int k) {
        Unit u;
        u.row = k >> p.part_shift;
        u.e0 = (k & (parts - 1)) * piece;
        u.n = min(piece, n - u.e0);
        const int64_t j = j0 + u.row;
        u.src = const_cast<char*>(p.in) + ((int64_t)b * p.in_b + j * p.in_row + v0 + u.e0) * E::ES;
        u.dst = p.out + ((int64_t)b * p.out_b + j * p.out_row + v0 + u.e0) * E::ES;
        return u;
    };
    unsigned char* buffer = adjust_smem_raw + lay.buffers + warp * kAdjustBuffer;
    // a piece's way into the warp's buffer: whole 16-byte chunks by one copy, the elements before and behind them by the lanes
    bool dropped = p.drop != 0;
    auto fetch = [&](const Unit& u) {
        const int mis = (int)((uintptr_t)u.src & 15u);
        const int head = min(u.n, mis ? E::EPC - mis / E::ES : 0), nc = (u.n - head) / E::EPC, tail = u.n - head - nc * E::EPC;
        if (lane == 0 && nc > 0 && !dropped) {
            mbar_arrive_expect_tx(&sh.full[warp], (unsigned)nc * 16u);
            bulk_load(buffer + (mis ? 16 : 0), u.src + head * E::ES, (unsigned)nc * 16u, &sh.full[warp]);
        }
        if (lane < head + tail) {
            const int i = lane < head ? lane : u.n - tail + (lane - head);
            ((T*)(buffer + mis))[i] = ((const T*)u.src)[i];
        }
        return nc > 0;
    };
    bool coming = false;
    unsigned phase = 0;
    if constexpr (!kInPlace) {
        if (lane == 0) {
            mbar_init(&sh.full[warp], 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        if (warp < units) {
            const Unit u = unit_at(warp);
            if (u.n > 0) coming = fetch(u);
        }
    }

    // ---- what the rows have in common ----
    if (tid == 0) sh.twice = 0;
    if (tid < j1 - j0) {
        sh.path_n[tid] = 0;
        int m = -1;
        if (p.allowed) m = p.allowed_row[(int64_t)b * p.R + j0 + tid];
        sh.mask_row[tid] = m < p.n_allowed ? m : -1;
    }
    if (sparse) {
        uint4* t4 = reinterpret_cast<uint4*>(table);
        for (int i = tid; i < kTile / 4; i += kAdjustThreads) t4[i] = make_uint4(0u, 0u, 0u, 0u);
        if (p.C > 1) adjust_cluster_sync();
        else __syncthreads();
        if (p.n_bias > 0) {
            const int32_t* at = p.bias_token + (int64_t)b * p.n_bias;
            const float* val = p.bias + (int64_t)b * p.n_bias;
            for (int i = tid; i < p.n_bias; i += kAdjustThreads) {
                const int64_t t = (int64_t)at[i] - v0;
                if (t < 0 || t >= n) continue;
                if (atomicOr(&table[t], kHasBias) & kHasBias) sh.twice = 1;
                bias_of[t] = val[i];
            }
            __syncthreads();
            if (sh.twice)                                           // a token's first entry adds up all of them, in their order
                for (int i = tid; i < p.n_bias; i += kAdjustThreads) {
                    const int64_t t = (int64_t)at[i] - v0;
                    if (t < 0 || t >= n) continue;
                    bool once = true;
                    for (int k = 0; k < i && once; ++k) once = at[k] != at[i];
                    if (!once) continue;
                    double s = 0.0;
                    for (int k = i; k < p.n_bias; ++k)
                        if (at[k] == at[i]) s += (double)val[k];
                    bias_of[t] = (float)s;
                }
        }
        if (p.penalised && p.history) {
            int prompt;
            const int len = adjust_history(p, b, &prompt);
            const int32_t* h = p.history + (int64_t)b * p.history_stride;
            const unsigned rank = (unsigned)tile % (unsigned)p.C;
            const int64_t base = v0 - (int64_t)rank * kTile;        // first token of the cluster's tiles
            const int step = p.C * kAdjustThreads;
            auto count = [&](int i, int tok) {
                const int64_t t64 = (int64_t)tok - base;
                if (t64 < 0 || t64 >= (int64_t)p.C * kTile || tok >= p.V) return;
                const uint32_t t = (uint32_t)t64;
                if (p.C == 1) {
                    if (i < prompt) atomicOr(&table[t], kInPrompt);
                    else atomicAdd(&table[t], kOnce);
                } else {
                    uint32_t a;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(&table[t % kTile])), "r"(t / kTile));
                    if (i < prompt) asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(a), "r"(kInPrompt) : "memory");
                    else asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(a), "r"(kOnce) : "memory");
                }
            };
            for (int i0 = (int)rank * kAdjustThreads + tid; i0 < len; i0 += 4 * step) {
                int tok[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) tok[u] = (int64_t)i0 + (int64_t)u * step < len ? h[i0 + (int64_t)u * step] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) count(i0 + u * step, tok[u]);
            }
        }
        if (p.penalised && p.token_ids && tid < j1 - j0) {          // one thread a row: up the path
            const int32_t* tok = p.token_ids + (int64_t)b * p.R;
            const int32_t* par = p.parent_idx + (int64_t)b * p.R;
            int at = j0 + tid, k = 0;
            for (int step = 0; step < kMaxPath; ++step) {
                const int64_t t = (int64_t)tok[at] - v0;
                if (t >= 0 && t < n) sh.path[tid][k++] = (uint16_t)t;
                const int up = par[at];
                if (up < 0 || up >= at) break;
                at = up;
            }
            sh.path_n[tid] = k;
        }
        if (p.C > 1) adjust_cluster_sync();                         // no CTA counts into another's table from here on
        else __syncthreads();
        // the list: every thread has kTile / kAdjustThreads consecutive tokens, a warp an eighth of the tile
        constexpr int kEach = kTile / kAdjustThreads;               // 16 or 8
        uint32_t have = 0;
#pragma unroll
        for (int k = 0; k < kEach; k += 4) {
            const uint4 w = t4[(tid * kEach + k) / 4];
            have |= (w.x ? 1u : 0u) << k | (w.y ? 2u : 0u) << k | (w.z ? 4u : 0u) << k | (w.w ? 8u : 0u) << k;
        }
        int at = __popc(have), sum = at;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFullMask, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) sh.list_from[warp + 1] = sum;
        __syncthreads();
        int before = 0;
        for (int k = 0; k < warp; ++k) before += sh.list_from[k + 1];
        __syncthreads();
        if (lane == 31) sh.list_from[warp + 1] = before + sum;
        if (tid == 0) sh.list_from[0] = 0;
        at = before + sum - at;
        while (have) {
            list[at++] = (uint16_t)(tid * kEach + __ffs(have) - 1);
            have &= have - 1;
        }
    }
    __syncthreads();
    // ---- the rows ----
    Penalty q;
    q.rep = p.repetition ? (double)p.repetition[b] : 1.0;
    q.inv = 1.0 / q.rep;
    q.pres = p.presence ? (double)p.presence[b] : 0.0;
    q.freq = p.frequency ? (double)p.frequency[b] : 0.0;
    for (int k = warp; k < units; k += kAdjustWarps) {
        const Unit u = unit_at(k);
        if (u.n <= 0) continue;
        constexpr int kRegs = kTile / 1024;
        const int m = sh.mask_row[u.row];
        const uint32_t* mask = m < 0 ? nullptr : p.allowed + (int64_t)m * p.words;
        const int64_t v = v0 + u.e0;
        uint32_t word[kRegs];
        if (mask) {
#pragma unroll
            for (int i = 0; i < kRegs; ++i) {
                const int at = 32 * i + lane;
                word[i] = 32 * at < u.n ? mask[(v >> 5) + at] : 0u;
            }
        }
        char* x = u.src;
        if constexpr (!kInPlace) {
            x = (char*)buffer + ((uintptr_t)u.src & 15u);
            if (coming) {
                if (!__all_sync(kFullMask, mbar_wait_limited(&sh.full[warp], phase, dropped ? kTestSpinLimit : kSpinLimit))) {
                    // a copy that does not come: NaN in the warp's pieces from here on, and the copy is waited for once more before leaving
                    for (int o = k; o < units; o += kAdjustWarps) {
                        const Unit lost = unit_at(o);
                        for (int i = lane; i < lost.n; i += 32) ((T*)lost.dst)[i] = Raw<DT>::nan;
                    }
                    if (lane == 0) {
                        if (!dropped) mbar_wait_bounded(&sh.full[warp], phase);
                        if (p.status) atomicOr(&p.status[b], CADD_STATUS_INTERNAL_TIMEOUT);
                    }
                    break;
                }
                phase ^= 1u;
            }
            __syncwarp();
        }
        if (sparse) {
            const int np = sh.path_n[u.row];
            const uint16_t* path = sh.path[u.row];
            T own[3];
            constexpr int kOwn = (kMaxPath + 31) / 32;
#pragma unroll
            for (int s = 0; s < kOwn; ++s) {
                const int i = s * 32 + lane;
                if (i < np) {
                    const int t = path[i], at = t - u.e0;
                    if (at >= 0 && at < u.n) {
                        const uint32_t word = table[t];
                        uint32_t times = word / kOnce;
                        for (int o = 0; o < np; ++o) times += path[o] == t;
                        own[s] = Raw<DT>::round(penalised(q, (double)E::load(x, at), times, true) + (word & kHasBias ? (double)bias_of[t] : 0.0));
                    }
                }
            }
            __syncwarp();
            // entries of the list in [e0, e0 + piece): pieces are whole eighths
            const int from = sh.list_from[(u.e0 * kAdjustWarps) / kTile], to = sh.list_from[((u.e0 + piece) * kAdjustWarps) / kTile];
            for (int i = from + lane; i < to; i += 32) {
                const int t = list[i], at = t - u.e0;
                const uint32_t word = table[t], times = word / kOnce;
                double y = penalised(q, (double)E::load(x, at), times, times > 0u || (word & kInPrompt));
                if (word & kHasBias) y += (double)bias_of[t];
                ((T*)x)[at] = Raw<DT>::round(y);
            }
            __syncwarp();
#pragma unroll
            for (int s = 0; s < kOwn; ++s) {
                const int i = s * 32 + lane;
                if (i < np) {
                    const int at = path[i] - u.e0;
                    if (at >= 0 && at < u.n) ((T*)x)[at] = own[s];
                }
            }
            __syncwarp();
        }
        if (mask) mask_piece<DT, !kInPlace>(x, u.n, mask, p.words, v, word);
        if constexpr (!kInPlace) {
            const int mis = (int)((uintptr_t)u.src & 15u);
            if (mis == (int)((uintptr_t)u.dst & 15u)) {
                const int head = min(u.n, mis ? E::EPC - mis / E::ES : 0), nc = (u.n - head) / E::EPC, tail = u.n - head - nc * E::EPC;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0 && nc > 0) {
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                                 ::"l"(u.dst + head * E::ES), "r"(smem_u32(buffer + (mis ? 16 : 0))), "r"((unsigned)nc * 16u) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
                if (lane < head + tail) {
                    const int i = lane < head ? lane : u.n - tail + (lane - head);
                    ((T*)u.dst)[i] = ((const T*)x)[i];
                }
            } else {                                                // rows that start differently: element by element
                __syncwarp();
                for (int i = lane; i < u.n; i += 32) ((T*)u.dst)[i] = ((const T*)x)[i];
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
            coming = false;
            if (k + kAdjustWarps < units) {
                const Unit next = unit_at(k + kAdjustWarps);
                if (next.n > 0) coming = fetch(next);
            }
        }
    }
}

// Status of one request, where it is asked for: lengths, paths and masks of its live rows.
__global__ void __launch_bounds__(kAdjustThreads) adjust_status_kernel(AdjustParams p) {
    __shared__ int bits;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) bits = 0;
    __syncthreads();
    int st = 0;
    if (tid == 0) {
        const int nn = p.n_nodes ? p.n_nodes[b] : p.R - 1;
        if (nn < -1 || nn > p.R - 1) st |= CADD_STATUS_BAD_N_NODES;
        if (p.history) {
            const int hl = p.history_len ? p.history_len[b] : p.history_cols, pl = p.prompt_len ? p.prompt_len[b] : 0;
            int prompt;
            if (adjust_history(p, b, &prompt) != hl || prompt != pl) st |= CADD_STATUS_BAD_LENGTH;
        }
    }
    const int live = adjust_live(p, b);
    if (p.token_ids && p.penalised) {
        const int32_t* par = p.parent_idx + (int64_t)b * p.R;
        for (int j = tid; j < live; j += kAdjustThreads) {
            int at = j;
            for (int step = 0; at > 0; ++step) {
                const int up = par[at];
                if (up < 0) break;
                if (up >= at || step == kMaxPath - 1) { st |= CADD_STATUS_BAD_PATH; break; }
                at = up;
            }
        }
    }
    if (p.allowed) {
        for (int j = tid >> 5; j < live; j += kAdjustThreads / 32) {
            const int m = p.allowed_row[(int64_t)b * p.R + j];
            if (m < -1 || m >= p.n_allowed) st |= CADD_STATUS_BAD_MASK;
            const uint32_t* mask = adjust_mask(p, b, j);
            if (!mask) continue;
            bool any = false;
            for (int w0 = 0; w0 < p.words && !any; w0 += 32) {
                uint32_t w = w0 + lane < p.words ? mask[w0 + lane] : 0u;
                if (w0 + lane == p.words - 1 && (p.V & 31)) w &= (1u << (p.V & 31)) - 1u;
                any = __any_sync(kFullMask, w != 0u);
            }
            if (!any) st |= CADD_STATUS_NOTHING_ALLOWED;
        }
    }
    if (st) atomicOr(&bits, st);
    __syncthreads();
    if (tid == 0) p.status[b] = bits;
}

}  // namespace cadd
