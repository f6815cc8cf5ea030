// Penalties, biases and grammar masks on the logits of a tree's rows (cadd_adjust_args has the definition).
//
// A CTA takes kAdjustTile consecutive tokens of some rows of one request.  It first gathers what its tokens have in common
// over the rows: how often each stands in the history (a table in shared memory), the sum of its biases, and a list of the
// tokens with either.  Then it streams the rows: copies them and applies the masks (in place: writes only what a mask hides).
// Last, for every row, a warp goes over the lists and over the row's own path and writes the tokens that penalties or biases
// concern, from the input's value, in 64 bits.  Hidden tokens are not touched again, so the order does not matter in place.
#pragma once
#include "common.cuh"

namespace cadd {

constexpr int kAdjustThreads = 256;
constexpr int kAdjustTile = 4096;              // tokens a CTA takes of each of its rows
constexpr int kAdjustRows = 32;                // rows a CTA takes at most
constexpr int kMaxPath = 65;                   // nodes of a path: the deepest tree there is, and its root
constexpr uint32_t kInPrompt = 1u, kHasBias = 2u, kOnce = 4u;      // a token's word in the table: two flags, then n_out of the history

struct AdjustParams {
    const char* in;
    char* out;
    int64_t V, in_b, in_row, out_b, out_row;
    int batch, R, tiles, groups, rows_per_cta;
    int n_bias, history_cols, n_allowed, words;
    bool in_place, penalised;
    const int32_t *n_nodes, *token_ids, *parent_idx, *history, *history_len, *prompt_len, *bias_token, *allowed_row;
    int64_t history_stride;
    const float *repetition, *presence, *frequency, *bias;
    const uint32_t* allowed;
    int32_t* status;
};

// Shared memory behind this: float bias_sum[cap], uint16_t bias_at[cap], cap = adjust_bias_cap().
struct AdjustShared {
    uint32_t table[kAdjustTile];
    uint16_t listed[kAdjustTile];              // tokens with a history and no bias
    uint16_t path[kAdjustRows][kMaxPath];      // tokens of each row's path that lie in the tile
    int path_n[kAdjustRows];
    int n_listed, n_biased;
};
__host__ __device__ inline int adjust_bias_cap(int n_bias) { return n_bias < kAdjustTile ? n_bias : kAdjustTile; }
inline size_t adjust_smem_bytes(int n_bias) { return sizeof(AdjustShared) + (size_t)adjust_bias_cap(n_bias) * 6 + 16; }

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
// Mask bits of the tokens v .. v+n-1 (n <= 8), lowest first.
__device__ __forceinline__ uint32_t mask_bits_at(const uint32_t* mask, int words, int64_t v, int n) {
    const int w = (int)(v >> 5), s = (int)(v & 31);
    const uint32_t lo = mask[w], hi = s + n > 32 && w + 1 < words ? mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, s) & ((1u << n) - 1u);
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
template <int DT> __device__ __forceinline__ void store_rounded(char* row, int64_t i, double x) {
    if constexpr (DT == CADD_DTYPE_BF16) ((__nv_bfloat16*)row)[i] = __double2bfloat16(x);
    else ((float*)row)[i] = (float)x;
}
template <int DT> __device__ __forceinline__ void store_hidden(char* row, int64_t i) {
    if constexpr (DT == CADD_DTYPE_BF16) ((uint16_t*)row)[i] = 0xff80u;
    else ((uint32_t*)row)[i] = 0xff800000u;
}

// Copy of n elements from src to dst with the mask applied (mask: bits from token v0 on, or NULL).
template <int DT>
__device__ __forceinline__ void stream_row(const AdjustParams& p, const char* src, char* dst, int n, const uint32_t* mask, int64_t v0) {
    using E = Elem<DT>;
    const int tid = threadIdx.x;
    if (p.in_place && !mask) return;
    const int mis = (int)(((uintptr_t)src & 15u) / E::ES);
    if (((uintptr_t)src & 15u) != ((uintptr_t)dst & 15u)) {              // rows that start differently: element by element
        for (int i = tid; i < n; i += kAdjustThreads) {
            const bool keep = !mask || mask_bits_at(mask, p.words, v0 + i, 1);
            if (!keep) store_hidden<DT>(dst, i);
            else if constexpr (DT == CADD_DTYPE_BF16) ((uint16_t*)dst)[i] = ((const uint16_t*)src)[i];
            else ((uint32_t*)dst)[i] = ((const uint32_t*)src)[i];
        }
        return;
    }
    const int head = min(n, mis ? E::EPC - mis : 0), nc = (n - head) / E::EPC, tail = n - head - nc * E::EPC;
    if (tid < head + tail) {
        const int i = tid < head ? tid : n - tail + (tid - head);
        const bool keep = !mask || mask_bits_at(mask, p.words, v0 + i, 1);
        if (!keep) store_hidden<DT>(dst, i);
        else if (!p.in_place) {
            if constexpr (DT == CADD_DTYPE_BF16) ((uint16_t*)dst)[i] = ((const uint16_t*)src)[i];
            else ((uint32_t*)dst)[i] = ((const uint32_t*)src)[i];
        }
    }
    const uint4* s4 = (const uint4*)(src + head * E::ES);
    uint4* d4 = (uint4*)(dst + head * E::ES);
    constexpr uint32_t kAll = (1u << E::EPC) - 1u;
    const uint32_t ninf = E::ES == 2 ? 0xff80ff80u : 0xff800000u;
    for (int c0 = tid; c0 < nc; c0 += 4 * kAdjustThreads) {
        uint4 w[4];
        uint32_t bits[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int c = c0 + u * kAdjustThreads;
            bits[u] = kAll;
            if (c < nc && mask) bits[u] = mask_bits_at(mask, p.words, v0 + head + (int64_t)c * E::EPC, E::EPC);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int c = c0 + u * kAdjustThreads;
            w[u] = make_uint4(ninf, ninf, ninf, ninf);
            if (c < nc && bits[u] != 0u && !(p.in_place && bits[u] == kAll)) w[u] = s4[c];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int c = c0 + u * kAdjustThreads;
            if (bits[u] != kAll) hide<DT>(w[u], bits[u]);
            if (c < nc && !(p.in_place && bits[u] == kAll)) d4[c] = w[u];
        }
    }
}

template <int DT>
__global__ void __launch_bounds__(kAdjustThreads) adjust_kernel(AdjustParams p) {
    using E = Elem<DT>;
    extern __shared__ __align__(16) unsigned char adjust_smem_raw[];
    AdjustShared& sh = *reinterpret_cast<AdjustShared*>(adjust_smem_raw);
    const int cap = adjust_bias_cap(p.n_bias);
    float* bias_sum = reinterpret_cast<float*>(adjust_smem_raw + ((sizeof(AdjustShared) + 15) & ~(size_t)15));
    uint16_t* bias_at = reinterpret_cast<uint16_t*>(bias_sum + cap);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tile = (int)(blockIdx.x % (unsigned)p.tiles);
    const int bg = (int)(blockIdx.x / (unsigned)p.tiles);
    const int b = bg / p.groups, g = bg - b * p.groups;
    const int live = adjust_live(p, b);
    const int j0 = g * p.rows_per_cta, j1 = min(live, j0 + p.rows_per_cta);
    if (j0 >= j1) return;
    const int64_t v0 = (int64_t)tile * kAdjustTile;
    const int n = (int)min((int64_t)kAdjustTile, p.V - v0);
    const bool sparse = p.penalised || p.n_bias > 0;

    if (sparse) {
        // ---- what the rows have in common ----
        uint4* t4 = reinterpret_cast<uint4*>(sh.table);
        for (int i = tid; i < kAdjustTile / 4; i += kAdjustThreads) t4[i] = make_uint4(0u, 0u, 0u, 0u);
        if (tid == 0) { sh.n_listed = 0; sh.n_biased = 0; }
        if (tid < kAdjustRows) sh.path_n[tid] = 0;
        __syncthreads();
        for (int i = tid; i < p.n_bias; i += kAdjustThreads) {                // a token's first entry adds up all of them, in order
            const int32_t* at = p.bias_token + (int64_t)b * p.n_bias;
            const float* val = p.bias + (int64_t)b * p.n_bias;
            const int64_t t = (int64_t)at[i] - v0;
            if (t < 0 || t >= n) continue;
            bool first = true;
            for (int k = 0; k < i && first; ++k) first = at[k] != at[i];
            if (!first) continue;
            double s = 0.0;
            for (int k = i; k < p.n_bias; ++k)
                if (at[k] == at[i]) s += (double)val[k];
            const int e = atomicAdd(&sh.n_biased, 1);                        // at most one entry per token of the tile: within cap
            bias_at[e] = (uint16_t)t;
            bias_sum[e] = (float)s;
            sh.table[t] = kHasBias;
        }
        __syncthreads();
        if (p.penalised && p.history) {
            int prompt;
            const int len = adjust_history(p, b, &prompt);
            const int32_t* h = p.history + (int64_t)b * p.history_stride;
            for (int i = tid; i < len; i += kAdjustThreads) {
                const int64_t t = (int64_t)h[i] - v0;
                if (t < 0 || t >= n) continue;
                const uint32_t old = i < prompt ? atomicOr(&sh.table[t], kInPrompt) : atomicAdd(&sh.table[t], kOnce);
                if (old == 0u) sh.listed[atomicAdd(&sh.n_listed, 1)] = (uint16_t)t;
            }
        }
        if (p.penalised && p.token_ids && tid < j1 - j0) {                    // one thread a row: up the path
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
    }
    // ---- the rows ----
    for (int j = j0; j < j1; ++j) {
        const char* src = p.in + ((int64_t)b * p.in_b + (int64_t)j * p.in_row + v0) * E::ES;
        char* dst = p.out + ((int64_t)b * p.out_b + (int64_t)j * p.out_row + v0) * E::ES;
        stream_row<DT>(p, src, dst, n, adjust_mask(p, b, j), v0);
    }
    if (!sparse) return;
    __syncthreads();
    // ---- tokens that penalties and biases concern ----
    const double rep = p.repetition ? (double)p.repetition[b] : 1.0;
    const double pres = p.presence ? (double)p.presence[b] : 0.0, freq = p.frequency ? (double)p.frequency[b] : 0.0;
    const int n_biased = sh.n_biased, n_all = n_biased + sh.n_listed;
    for (int j = j0 + warp; j < j1; j += kAdjustThreads / 32) {
        const char* src = p.in + ((int64_t)b * p.in_b + (int64_t)j * p.in_row + v0) * E::ES;
        char* dst = p.out + ((int64_t)b * p.out_b + (int64_t)j * p.out_row + v0) * E::ES;
        const uint32_t* mask = adjust_mask(p, b, j);
        const uint16_t* path = sh.path[j - j0];
        const int np = sh.path_n[j - j0];
        for (int i = lane; i < n_all + np; i += 32) {
            int t;
            double bias = 0.0;
            bool mine = true;
            if (i < n_biased) { t = bias_at[i]; bias = (double)bias_sum[i]; }
            else if (i < n_all) t = sh.listed[i - n_biased];
            else {                                                           // of the path: what neither list has, once
                t = path[i - n_all];
                mine = sh.table[t] == 0u;
                for (int k = 0; k < i - n_all; ++k) mine = mine && path[k] != t;
            }
            if (!mine || (mask && !mask_bits_at(mask, p.words, v0 + t, 1))) continue;
            const uint32_t word = sh.table[t];
            uint32_t times = word / kOnce;
            for (int k = 0; k < np; ++k) times += path[k] == t;
            double x = (double)E::load(src, t);
            if (times > 0u || (word & kInPrompt)) x = x > 0.0 ? x / rep : x * rep;
            if (times > 0u) x = x - freq * (double)times - pres;
            store_rounded<DT>(dst, t, x + bias);
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
