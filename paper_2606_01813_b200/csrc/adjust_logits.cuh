// Penalties, biases and grammar masks on the logits of a tree's rows (cadd_adjust_args has the definition).
//
// adjust_rows_kernel, into another array or in place.  A CTA takes a tile of consecutive tokens (8 KB of logits) of some rows of one request.  It
// first gathers what its tokens have in common over the rows: how often each stands in the history (a table in shared memory; every
// CTA reads the whole history, which stays in L2), the sum of its biases, and from that a list of the tokens with either, in order.  Then
// a warp takes a row's piece of the tile at a time: it comes to shared memory by a bulk copy, the tokens that penalties or biases
// concern are replaced there, what the mask hides is set, and a bulk copy takes it to its place.  Tokens of a row's own path are
// computed before the list's and written after them, from the input's value and their own count.
//
// With few rows a table for every tile is not worth its while: then adjust_stream_kernel copies and masks, and adjust_tokens_kernel
// replaces single tokens in memory afterwards, a CTA for all tokens of a request (a hash table in shared memory).  Its launch is under way
// while the kernel before it still runs, no more: a CTA wants an SM's whole register file and up to 200 KB of shared memory, and begins where the copying
// CTAs have left.  In place the former writes (and reads) only what masks change: masks alone are its, too (six CTAs an SM, for which it spills 56 bytes).
//
// What bounds it.  32 trees of up to 65 rows of 151936, bf16, histories of 4000 (779 MB): 141 us, 5.5 TB/s; issue 64 % (logic 55 %: masks), DRAM 64 % of
// nominal.  8 trees of up to 257 rows of 32001 in fp32, histories of 32768 (382 MB): 108 us, 3.5 TB/s; half of all tokens are replaced, in 64 bits, and
// that takes the issue slots (68 %).  A grammar of 1 % in place (399 MB, nearly all of it writes): 116 us, where writes alone take 103.  One
// token for 64 requests, histories of 8192 (41 MB): 19.6 us, most of it in hash tables and gathers of single logits (issue 37 %, DRAM 8 %
// in that kernel); for one request 6.1 us, launches and chains of loads.
#pragma once
#include "common.cuh"
#include "tile_ring.cuh"

namespace cadd {

constexpr int kAdjustThreads = 256;
constexpr int kAdjustWarps = kAdjustThreads / 32;
constexpr int kAdjustTileBytes = 8192;         // of a row: the tokens whose tables a CTA of adjust_rows_kernel has; a piece of adjust_stream_kernel
constexpr int kAdjustPieceBytes = 4096;        // of a row: a piece of adjust_rows_kernel
constexpr int kAdjustRows = 24;                // rows a CTA takes at most (trees of 65 rows 147 us with 36, 144 with 24, 146 with 20; of 257 rows 127, 114, 116)
constexpr int kAdjustBatch = 8;                // tokens of the history that a thread has under way
constexpr int kMaxPath = 65;                   // nodes of a path: the deepest tree there is, and its root
constexpr uint32_t kInPrompt = 1u, kHasBias = 2u, kOnce = 4u;      // a token's word in the table: two flags, then n_out of the history

struct AdjustParams {
    const char* in;
    char* out;
    int64_t V, in_b, in_row, out_b, out_row;
    int batch, R, tiles, groups, rows_per_cta, part_shift;         // pieces of a row's tile: 1 << part_shift
    int S, slots, slot_shift;                                       // adjust_tokens_kernel: CTAs that share a request's tokens (token t: CTA t % S); 1 << (32 - slot_shift) slots
    int n_bias, history_cols, n_allowed, words;
    bool penalised;
    bool followed;                                                  // adjust_tokens_kernel comes next
    int drop;                                                       // test hook: 1: no copy is ever made
    const int32_t *n_nodes, *token_ids, *parent_idx, *history, *history_len, *prompt_len, *bias_token, *allowed_row;
    int64_t history_stride;
    const float *repetition, *presence, *frequency, *bias;
    const uint32_t* allowed;
    int32_t* status;
};

template <int DT> constexpr int kAdjustTile = kAdjustTileBytes / Elem<DT>::ES;   // tokens

// Tokens of a tile that the history or biases concern, in order; what list_from and the like index.  An entry without a bias is one
// word: place | kListPrompt | n_out << kListShift; one with a bias has the same word and the sum of its biases.
constexpr uint32_t kListPlace = 4095u, kListPrompt = 4096u;
constexpr int kListShift = 13;
constexpr int kListMost = (1 << (32 - kListShift)) - 1;             // uses that a word has room for
// Behind this (see adjust_layout): the table and the sums of biases by place, and then, in their stead, the warps' buffers; the two lists.
struct AdjustShared {
    alignas(8) uint64_t full[kAdjustWarps];    // a warp's piece has landed
    int path_n[kAdjustRows];
    uint16_t path[kAdjustRows][kMaxPath];      // tokens of each row's path that lie in the tile
    int from[2][kAdjustWarps + 1];             // the entries, without and with a bias, of each eighth of the tile
    int twice;                                 // some token has two biases
};
template <int kBytes> constexpr int kAdjustBuffer = kBytes + 16;    // of one warp: the piece keeps its distance from a 16-byte boundary
struct AdjustLayout { int table, bias, buffers, plain, biased, sums, bytes; };
__host__ __device__ inline AdjustLayout adjust_layout(int tile, int n_bias) {
    AdjustLayout l;
    const int most = n_bias < tile ? n_bias : tile, tables = tile * (n_bias > 0 ? 8 : 4), buffers = kAdjustWarps * (kAdjustPieceBytes + 16);
    l.table = l.buffers = (int)((sizeof(AdjustShared) + 127) & ~(size_t)127);
    l.bias = l.table + tile * 4;
    l.plain = l.table + (tables > buffers ? tables : buffers);
    l.biased = l.plain + tile * 4;
    l.sums = l.biased + most * 4;
    l.bytes = l.sums + most * 4;
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
        for (int i = 0; i < 4; i += 2) {
            // four bits to the top bits of four bytes (the shifted copies share no position), and each byte's top bit over a half word
            const uint32_t tops = ((bits >> (2 * i)) & 15u) * 0x10204080u;
            uint32_t lo, hi;
            asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(lo) : "r"(tops));
            asm("prmt.b32 %0, %1, 0, 0xbbaa;" : "=r"(hi) : "r"(tops));
            x[i] = (x[i] & lo) | (0xff80ff80u & ~lo);
            x[i + 1] = (x[i + 1] & hi) | (0xff80ff80u & ~hi);
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
__device__ __forceinline__ double penalised(const Penalty& q, float logit, uint32_t times, bool seen) {
    double x = (double)logit;
    if (seen) x *= logit > 0.0f ? q.inv : q.rep;      // (x / rep to 2^-52, long before the rounding to fp32 or bf16)
    // (times as a double: the low word of 2^52's, less 2^52; four times the rate of a conversion)
    if (times > 0u) x -= q.freq * (__hiloint2double(0x43300000, (int)times) - 0x1p52) + q.pres;
    return x;
}

// Words of a mask that a lane holds for a piece of so many bytes: 4, 2 or 1.
template <int DT, int kBytes> constexpr int kMaskRegs = kBytes / Elem<DT>::ES / 1024;
// What a mask hides of n elements at x, whose first is token v (a multiple of 32): x lies in shared memory, or is memory itself.  A warp.
template <int DT, int kBytes>
__device__ __forceinline__ void mask_piece(char* x, int n, const uint32_t* mask, int words, int64_t v, const uint32_t (&first)[kMaskRegs<DT, kBytes>]) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    constexpr int kRegs = kMaskRegs<DT, kBytes>;
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
    for (int i0 = 0; i0 < kBytes / 512; i0 += kStep) {
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

__device__ __forceinline__ void count_use(uint32_t* word, bool in_prompt) {
    if (in_prompt) atomicOr(word, kInPrompt);
    else atomicAdd(word, kOnce);
}
// Sums of the biases of the tokens that have a place here (place(token) >= 0), marked in the table, which holds nothing else yet.  A sum of several
// is taken in 64 bits and kept in 32, as the biases come.
template <int kThreadsHere, typename Place>
__device__ __forceinline__ void gather_biases(const AdjustParams& p, int b, uint32_t* table, float* bias_of, int* twice, Place place) {
    const int32_t* at = p.bias_token + (int64_t)b * p.n_bias;
    const float* val = p.bias + (int64_t)b * p.n_bias;
    for (int i = threadIdx.x; i < p.n_bias; i += kThreadsHere) {
        const int t = place(at[i]);
        if (t < 0) continue;
        if (atomicOr(&table[t], kHasBias) & kHasBias) *twice = 1;
        bias_of[t] = val[i];
    }
    __syncthreads();
    if (!*twice) return;
    // Some token is listed more than once.  Its word becomes the place of its first entry (counted from behind, from bit 2 on) and a top bit;
    // a warp adds up its entries: lane l the l-th of every 32, and then the lanes' sums, so the order is always the same.
    constexpr uint32_t kMore = 0x80000000u;
    const uint32_t lane = threadIdx.x & 31u;
#pragma unroll 1
    for (int i = threadIdx.x; i < p.n_bias; i += kThreadsHere) {
        const int t = place(at[i]);
        if (t >= 0) atomicMax(&table[t], (uint32_t)(p.n_bias - i) << 2 | kHasBias);
    }
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < p.n_bias; i += kThreadsHere) {
        const int t = place(at[i]);
        if (t >= 0 && (table[t] & ~kMore) >> 2 != (uint32_t)(p.n_bias - i)) atomicOr(&table[t], kMore);
    }
    __syncthreads();
#pragma unroll 1
    for (int i0 = (int)(threadIdx.x - lane); i0 < p.n_bias; i0 += kThreadsHere) {
        const int i = i0 + (int)lane, tok = i < p.n_bias ? at[i] : -1, t = i < p.n_bias ? place(tok) : -1;
        unsigned firsts = __ballot_sync(kFullMask, t >= 0 && table[t] == ((uint32_t)(p.n_bias - i) << 2 | kHasBias | kMore));
        while (firsts) {
            const int from = __ffs(firsts) - 1, want = __shfl_sync(kFullMask, tok, from), to = __shfl_sync(kFullMask, t, from);
            firsts &= firsts - 1u;
            double s = 0.0;
#pragma unroll 4
            for (int k = i0 + (int)lane; k < p.n_bias; k += 32)
                if (at[k] == want) s += (double)val[k];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFullMask, s, o);
            if (lane == 0) bias_of[to] = (float)s;
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < p.n_bias; i += kThreadsHere) {
        const int t = place(at[i]);
        if (t >= 0) table[t] = kHasBias;
    }
    __syncthreads();
}
// Rows 0 .. n-1 of a request's tree brought to shared memory (n tokens, then n parents), where there is room: a path is a chain of
// loads, each of them a round trip to memory otherwise.
template <int kThreadsHere>
__device__ __forceinline__ void stage_tree(const AdjustParams& p, int b, int n, int32_t* stage, int room) {
    if (2 * n > room) return;
    const int32_t* tok = p.token_ids + (int64_t)b * p.R;
    const int32_t* par = p.parent_idx + (int64_t)b * p.R;
    for (int i = threadIdx.x; i < n; i += kThreadsHere) {
        stage[i] = tok[i];
        stage[n + i] = par[i];
    }
}
// Places of the tokens on row j's path (j < n), the row's own first; returns how many.  One thread.
template <typename Place>
__device__ __forceinline__ int gather_path(const AdjustParams& p, int b, int j, int n, const int32_t* stage, int room, uint16_t* path, Place place) {
    const bool staged = room > 0 && 2 * n <= room;
    const int32_t* tok = staged ? stage : p.token_ids + (int64_t)b * p.R;
    const int32_t* par = staged ? stage + n : p.parent_idx + (int64_t)b * p.R;
    int k = 0;
    for (int step = 0; step < kMaxPath; ++step) {
        const int t = place(tok[j]), up = par[j];
        if (t >= 0) path[k++] = (uint16_t)t;
        if (up < 0 || up >= j) break;
        j = up;
    }
    return k;
}
__device__ __forceinline__ uint32_t four(const uint4& w, int j) { return j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w; }
// The lists from the table (whole CTA; warp w has the w-th eighth of the places); from[0], from[1]: the entries without and with a bias
// of each eighth.
template <int kPlaces>
__device__ __forceinline__ void gather_lists(const uint32_t* table, const float* bias_of, uint32_t* plain, uint32_t* biased, float* sums, int (*from)[kAdjustWarps + 1]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kEighth = kPlaces / kAdjustWarps, kSteps = kEighth / 128;
    // entries among a lane's four places: without a bias, and with one (from bit 16 on; at most 4096 in all: no carry)
    auto kinds = [](const uint4& w) {
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) n += four(w, j) == 0u ? 0u : (four(w, j) & kHasBias ? 0x10000u : 1u);
        return n;
    };
    const uint4* mine = reinterpret_cast<const uint4*>(table) + warp * (kEighth / 4) + lane;
    uint32_t all = 0;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) all += kinds(mine[k * 32]);
    all = __reduce_add_sync(kFullMask, all);
    if (lane == 0) { from[0][warp + 1] = (int)(all & 0xffffu); from[1][warp + 1] = (int)(all >> 16); }
    __syncthreads();
    uint32_t at = 0, upto = 0;
#pragma unroll
    for (int k = 0; k < kAdjustWarps; ++k) {
        const uint32_t c = (uint32_t)from[0][k + 1] | (uint32_t)from[1][k + 1] << 16;
        upto += k <= warp ? c : 0u;
        at += k < warp ? c : 0u;
    }
    __syncthreads();                                                // (everybody has read the counts)
    if (lane == 0) {
        from[0][warp + 1] = (int)(upto & 0xffffu);
        from[1][warp + 1] = (int)(upto >> 16);
        if (warp == 0) from[0][0] = from[1][0] = 0;
    }
#pragma unroll 1
    for (int k = 0; k < kSteps; ++k) {                              // (rolled: code that runs once has to be fetched once)
        const uint4 w = mine[k * 32];
        const uint32_t n4 = kinds(w);
        if (!__any_sync(kFullMask, n4 != 0u)) continue;
        uint32_t to = n4;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(kFullMask, to, o);
            if (lane >= o) to += up;
        }
        const uint32_t total = __shfl_sync(kFullMask, to, 31);
        to += at - n4;
        at += total;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = four(w, j);
            if (x == 0u) continue;
            const int place = warp * kEighth + k * 128 + lane * 4 + j;
            const uint32_t word = (uint32_t)place | (x & kInPrompt ? kListPrompt : 0u) | (x / kOnce) << kListShift;
            if (x & kHasBias) {
                biased[to >> 16] = word;
                sums[to >> 16] = bias_of[place];
                to += 0x10000u;
            } else {
                plain[to++ & 0xffffu] = word;
            }
        }
    }
}
// Where an ordered list of words has a place between from and to, or -1.
__device__ __forceinline__ int find_place(const uint32_t* list, int from, int to, int place) {
    while (from < to) {
        const int mid = (from + to) / 2, here = (int)(list[mid] & kListPlace);
        if (here == place) return mid;
        if (here < place) from = mid + 1;
        else to = mid;
    }
    return -1;
}
// What a CTA asks memory for first, all at once: each of these would cost a round trip where it is needed.
template <int kThreadsHere>
struct AdjustFirst {
    float rep, pres, freq;
    int live, len, prompt;
    int tok[kAdjustBatch];                     // the thread's first tokens of the history (-1 behind its room)
    __device__ __forceinline__ AdjustFirst(const AdjustParams& p, int b) {
        const int32_t* h = p.history + (int64_t)b * p.history_stride;
        const bool history = p.penalised && p.history;
        rep = p.repetition ? p.repetition[b] : 1.0f;
        pres = p.presence ? p.presence[b] : 0.0f;
        freq = p.frequency ? p.frequency[b] : 0.0f;
        len = prompt = 0;
        if (history) len = adjust_history(p, b, &prompt);
#pragma unroll
        for (int u = 0; u < kAdjustBatch; ++u) {
            const int at = (int)threadIdx.x + u * kThreadsHere;
            tok[u] = history && at < p.history_cols ? h[at] : -1;
        }
        live = adjust_live(p, b);
    }
    __device__ __forceinline__ Penalty penalty() const { return Penalty{(double)rep, 1.0 / (double)rep, (double)pres, (double)freq}; }
    // count(i, token) for all of the thread's part of the history; more is asked for while a batch is counted
    template <typename Count>
    __device__ __forceinline__ void for_history(const AdjustParams& p, int b, Count count) {
        const int32_t* h = p.history + (int64_t)b * p.history_stride;
#pragma unroll 1
        for (int at = threadIdx.x; at < len; at += kAdjustBatch * kThreadsHere) {
            int now[kAdjustBatch];
#pragma unroll
            for (int u = 0; u < kAdjustBatch; ++u) {
                const int next = at + (kAdjustBatch + u) * kThreadsHere;
                now[u] = tok[u];
                tok[u] = next < len ? h[next] : -1;
            }
#pragma unroll
            for (int u = 0; u < kAdjustBatch; ++u)
                if (at + u * kThreadsHere < len) count(at + u * kThreadsHere, now[u]);
        }
    }
};
// A piece of a row that a warp takes at a time: n elements from token v on (a multiple of 32).
struct AdjustPiece {
    char *src, *dst;
    int64_t v;
    int n;
};
// Its way into the warp's buffer: whole 16-byte chunks by one copy, the elements before and behind them by the lanes.  The piece keeps its
// distance from a 16-byte boundary there.  False: no copy is under way.
template <int DT>
__device__ __forceinline__ bool fetch_piece(const AdjustPiece& u, unsigned char* buffer, uint64_t* full, bool dropped) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    const int lane = threadIdx.x & 31, mis = (int)((uintptr_t)u.src & 15u);
    const int head = min(u.n, mis ? E::EPC - mis / E::ES : 0), nc = (u.n - head) / E::EPC, tail = u.n - head - nc * E::EPC;
    if (lane == 0 && nc > 0 && !dropped) {
        mbar_arrive_expect_tx(full, (unsigned)nc * 16u);
        bulk_load(buffer + (mis ? 16 : 0), u.src + head * E::ES, (unsigned)nc * 16u, full);
    }
    if (lane < head + tail) {
        const int i = lane < head ? lane : u.n - tail + (lane - head);
        ((T*)(buffer + mis))[i] = ((const T*)u.src)[i];
    }
    return nc > 0;
}
// And out again; the buffer is free when it returns.
template <int DT>
__device__ __forceinline__ void deliver_piece(const AdjustPiece& u, unsigned char* buffer) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    const int lane = threadIdx.x & 31, mis = (int)((uintptr_t)u.src & 15u);
    const T* x = (const T*)(buffer + mis);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (mis == (int)((uintptr_t)u.dst & 15u)) {
        const int head = min(u.n, mis ? E::EPC - mis / E::ES : 0), nc = (u.n - head) / E::EPC, tail = u.n - head - nc * E::EPC;
        if (lane == 0 && nc > 0) {
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                         ::"l"(u.dst + head * E::ES), "r"(smem_u32(buffer + (mis ? 16 : 0))), "r"((unsigned)nc * 16u) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        if (lane < head + tail) {
            const int i = lane < head ? lane : u.n - tail + (lane - head);
            ((T*)u.dst)[i] = x[i];
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    } else {                                                        // rows that start differently: element by element
        for (int i = lane; i < u.n; i += 32) ((T*)u.dst)[i] = x[i];
    }
    __syncwarp();
}
// A copy that does not come: NaN in the piece, and the request is flagged.
template <int DT>
__device__ __forceinline__ void lose_piece(const AdjustParams& p, const AdjustPiece& u, int b) {
    using T = typename Raw<DT>::T;
    const int lane = threadIdx.x & 31;
    for (int i = lane; i < u.n; i += 32) ((T*)u.dst)[i] = Raw<DT>::nan;
    if (lane == 0 && p.status) atomicOr(&p.status[b], CADD_STATUS_INTERNAL_TIMEOUT);
}
// The words of a mask that a lane needs of a piece.
template <int N>
__device__ __forceinline__ void mask_words(const uint32_t* mask, const AdjustPiece& u, uint32_t (&word)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = 32 * i + (int)(threadIdx.x & 31);
        word[i] = 32 * at < u.n ? mask[(u.v >> 5) + at] : 0u;
    }
}

// Logits without penalties and biases, or before them: copied (kCopy) and masked.  A warp takes pieces of 8 KB, all of them dealt out to the CTAs
// first, then to their warps, so that few pieces have SMs to themselves.
template <int DT, bool kCopy>
__global__ void __launch_bounds__(kAdjustThreads, kCopy ? 3 : 6) adjust_stream_kernel(AdjustParams p) {
    using E = Elem<DT>;
    constexpr int kTile = kAdjustTile<DT>;
    extern __shared__ __align__(128) unsigned char adjust_smem_raw[];
    __shared__ alignas(8) uint64_t full[kAdjustWarps];
    if (p.followed) grid_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned char* buffer = adjust_smem_raw + warp * kAdjustBuffer<kAdjustTileBytes>;
    unsigned phase = 0;
    bool lost = false;                                              // a copy did not come: this piece and all that the warp would have taken after it
    if constexpr (kCopy) {
        if (lane == 0) {
            mbar_init(&full[warp], 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }
    const int64_t units = (int64_t)p.batch * p.R * p.tiles;
    for (int64_t k = blockIdx.x + (int64_t)warp * gridDim.x; k < units; k += (int64_t)gridDim.x * kAdjustWarps) {
        const int64_t row = k / p.tiles;
        const int b = (int)(row / p.R), j = (int)(row - (int64_t)b * p.R);
        if (j >= adjust_live(p, b)) continue;
        AdjustPiece u;
        u.v = (k - row * p.tiles) * kTile;
        u.n = (int)min((int64_t)kTile, p.V - u.v);
        u.src = const_cast<char*>(p.in) + ((int64_t)b * p.in_b + (int64_t)j * p.in_row + u.v) * E::ES;
        u.dst = p.out + ((int64_t)b * p.out_b + (int64_t)j * p.out_row + u.v) * E::ES;
        bool coming = false;
        if constexpr (kCopy) {
            if (lost) {
                lose_piece<DT>(p, u, b);
                continue;
            }
            coming = fetch_piece<DT>(u, buffer, &full[warp], p.drop != 0);
        }
        const uint32_t* mask = adjust_mask(p, b, j);
        uint32_t word[kMaskRegs<DT, kAdjustTileBytes>];
        if (mask) mask_words(mask, u, word);
        if constexpr (kCopy) {
            if (coming && !__all_sync(kFullMask, mbar_wait_limited(&full[warp], phase, p.drop ? kTestSpinLimit : kSpinLimit))) {
                lose_piece<DT>(p, u, b);
                lost = true;
                continue;
            }
            if (coming) phase ^= 1u;
            __syncwarp();
            if (mask) mask_piece<DT, kAdjustTileBytes>((char*)buffer + ((uintptr_t)u.src & 15u), u.n, mask, p.words, u.v, word);
            deliver_piece<DT>(u, buffer);
        } else if (mask) mask_piece<DT, kAdjustTileBytes>(u.dst, u.n, mask, p.words, u.v, word);
    }
    if constexpr (kCopy)
        if (lost && !p.drop && lane == 0) mbar_wait_bounded(&full[warp], phase);      // not to leave with a copy in flight
}

template <int DT>
__global__ void __launch_bounds__(kAdjustThreads, 4) adjust_rows_kernel(AdjustParams p) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    constexpr int kTile = kAdjustTile<DT>;
    extern __shared__ __align__(128) unsigned char adjust_smem_raw[];
    AdjustShared& sh = *reinterpret_cast<AdjustShared*>(adjust_smem_raw);
    const AdjustLayout lay = adjust_layout(kTile, p.n_bias);
    uint32_t* table = reinterpret_cast<uint32_t*>(adjust_smem_raw + lay.table);
    float* bias_of = reinterpret_cast<float*>(adjust_smem_raw + lay.bias);
    uint32_t* plain = reinterpret_cast<uint32_t*>(adjust_smem_raw + lay.plain);
    uint32_t* biased = reinterpret_cast<uint32_t*>(adjust_smem_raw + lay.biased);
    float* sums = reinterpret_cast<float*>(adjust_smem_raw + lay.sums);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned bg = blockIdx.x / (unsigned)p.tiles;
    const int tile = (int)(blockIdx.x - bg * (unsigned)p.tiles);
    const int b = (int)(bg / (unsigned)p.groups), g = (int)(bg - (unsigned)b * (unsigned)p.groups);
    AdjustFirst<kAdjustThreads> first(p, b);
    const int j0 = g * p.rows_per_cta, j1 = min(first.live, j0 + p.rows_per_cta);
    if (j0 >= j1) return;
    const int64_t v0 = (int64_t)tile * kTile;
    const int n = (int)min((int64_t)kTile, p.V - v0);
    const int parts = 1 << p.part_shift, piece = kTile >> p.part_shift;
    const int units = (j1 - j0) << p.part_shift;                   // a row's pieces one after the other

    auto piece_at = [&](int k) {
        const int e0 = (k & (parts - 1)) * piece;
        const int64_t j = j0 + (k >> p.part_shift);
        AdjustPiece u;
        u.v = v0 + e0;
        u.n = min(piece, n - e0);
        u.src = const_cast<char*>(p.in) + ((int64_t)b * p.in_b + j * p.in_row + u.v) * E::ES;
        u.dst = p.out + ((int64_t)b * p.out_b + j * p.out_row + u.v) * E::ES;
        return u;
    };
    unsigned char* buffer = adjust_smem_raw + lay.buffers + warp * kAdjustBuffer<kAdjustPieceBytes>;
    bool coming = false;
    unsigned phase = 0;
    if (lane == 0) {
        mbar_init(&sh.full[warp], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    const uint32_t* mask = nullptr;                                 // of the piece under way, and its words
    uint32_t word[kMaskRegs<DT, kAdjustPieceBytes>];
    auto fetch = [&](int k) {
        const AdjustPiece u = piece_at(k);
        if (u.n <= 0) return;
        coming = fetch_piece<DT>(u, buffer, &sh.full[warp], p.drop != 0);
        mask = adjust_mask(p, b, j0 + (k >> p.part_shift));
        if (mask) mask_words(mask, u, word);
    };

    // ---- what the rows have in common ----
    if (tid == 0) sh.twice = 0;
    if (tid < j1 - j0) sh.path_n[tid] = 0;
    uint4* t4 = reinterpret_cast<uint4*>(table);
    for (int i = tid; i < kTile / 4; i += kAdjustThreads) t4[i] = make_uint4(0u, 0u, 0u, 0u);
    const bool paths = p.penalised && p.token_ids;
    int32_t* stage = reinterpret_cast<int32_t*>(plain);             // (the list comes later)
    if (paths) stage_tree<kAdjustThreads>(p, b, j1, stage, kTile);
    __syncthreads();
    // (a token's place in the tile, or -1)
    auto place = [&](int tok) { return tok >= v0 && tok < v0 + n ? (int)(tok - v0) : -1; };
    if (p.n_bias > 0) gather_biases<kAdjustThreads>(p, b, table, bias_of, &sh.twice, place);
    first.for_history(p, b, [&](int i, int tok) {
        const int t = place(tok);
        if (t >= 0) count_use(&table[t], i < first.prompt);
    });
    if (paths && tid < j1 - j0) sh.path_n[tid] = gather_path(p, b, j0 + tid, j1, stage, kTile, sh.path[tid], place);
    __syncthreads();
    gather_lists<kTile>(table, bias_of, plain, biased, sums, sh.from);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // the tables' place becomes the buffers
    __syncthreads();
    // ---- the rows ----
    if (warp < units) fetch(warp);
    const Penalty q = first.penalty();
    for (int k = warp; k < units; k += kAdjustWarps) {
        const AdjustPiece u = piece_at(k);
        if (u.n <= 0) break;                                        // (a warp's pieces are all the same part of the tile)
        const int row = k >> p.part_shift, e0 = (int)(u.v - v0);
        char* x = (char*)buffer + ((uintptr_t)u.src & 15u);
        if (coming && !__all_sync(kFullMask, mbar_wait_limited(&sh.full[warp], phase, p.drop ? kTestSpinLimit : kSpinLimit))) {
            for (int o = k; o < units; o += kAdjustWarps) lose_piece<DT>(p, piece_at(o), b);
            if (lane == 0 && !p.drop) mbar_wait_bounded(&sh.full[warp], phase);      // not to leave with a copy in flight
            break;
        }
        if (coming) phase ^= 1u;
        __syncwarp();
        const int np = sh.path_n[row];
        const uint16_t* path = sh.path[row];
        constexpr int kOwn = (kMaxPath + 31) / 32;
        T own[kOwn];
#pragma unroll
        for (int s = 0; s < kOwn; ++s) {
            const int i = s * 32 + lane;
            if (i < np && path[i] >= e0 && path[i] < e0 + u.n) {
                const int t = path[i], eighth = t / (kTile / kAdjustWarps);
                const int a = find_place(plain, sh.from[0][eighth], sh.from[0][eighth + 1], t), c = find_place(biased, sh.from[1][eighth], sh.from[1][eighth + 1], t);
                uint32_t times = a >= 0 ? plain[a] >> kListShift : (c >= 0 ? biased[c] >> kListShift : 0u);
                for (int o = 0; o < np; ++o) times += path[o] == t;
                own[s] = Raw<DT>::round(penalised(q, E::load(x, t - e0), times, true) + (c >= 0 ? (double)sums[c] : 0.0));
            }
        }
        __syncwarp();
        // the lists' entries in [e0, e0 + piece): pieces are whole eighths
        const int part0 = e0 / (kTile / kAdjustWarps), part1 = part0 + (kAdjustWarps >> p.part_shift);
        for (int i = sh.from[0][part0] + lane, to = sh.from[0][part1]; i < to; i += 32) {
            const uint32_t e = plain[i];
            const int at = (int)(e & kListPlace) - e0;
            ((T*)x)[at] = Raw<DT>::round(penalised(q, E::load(x, at), e >> kListShift, true));
        }
        for (int i = sh.from[1][part0] + lane, to = sh.from[1][part1]; i < to; i += 32) {
            const uint32_t e = biased[i], times = e >> kListShift;
            const int at = (int)(e & kListPlace) - e0;
            ((T*)x)[at] = Raw<DT>::round(penalised(q, E::load(x, at), times, times > 0u || (e & kListPrompt)) + (double)sums[i]);
        }
        __syncwarp();
#pragma unroll
        for (int s = 0; s < kOwn; ++s) {
            const int i = s * 32 + lane;
            if (i < np && path[i] >= e0 && path[i] < e0 + u.n) ((T*)x)[path[i] - e0] = own[s];
        }
        __syncwarp();
        if (mask) mask_piece<DT, kAdjustPieceBytes>(x, u.n, mask, p.words, u.v, word);
        deliver_piece<DT>(u, buffer);
        coming = false;
        if (k + kAdjustWarps < units) fetch(k + kAdjustWarps);
    }
}

constexpr int kTokensThreads = 1024;
constexpr int kTokensSlots = 16384;            // of the hash table at most
constexpr int kTokensMost = 12288;             // tokens in it at most
constexpr int32_t kNoToken = -1;
// Behind this, for every slot: token, word, and the sum of its biases (where there are biases).
struct AdjustTokensShared {
    int path_n[kAdjustRows];
    uint16_t path[kAdjustRows][kMaxPath];      // slots of each row's path
    int twice;
};
constexpr int kTokensTable = (sizeof(AdjustTokensShared) + 15) & ~15;
inline size_t adjust_tokens_smem(int slots, bool biased) { return kTokensTable + (size_t)slots * (biased ? 12 : 8); }

// Single tokens of rows that have been copied and masked.  Every token that the history, biases or paths of the CTA's rows hold (and
// that is this CTA's among the S) gets a slot; there are more slots than such tokens, so a search ends.
template <int DT>
__global__ void __launch_bounds__(kTokensThreads) adjust_tokens_kernel(AdjustParams p) {
    using E = Elem<DT>;
    using T = typename Raw<DT>::T;
    extern __shared__ __align__(128) unsigned char adjust_smem_raw[];
    AdjustTokensShared& sh = *reinterpret_cast<AdjustTokensShared*>(adjust_smem_raw);
    int32_t* token = reinterpret_cast<int32_t*>(adjust_smem_raw + kTokensTable);
    uint32_t* table = reinterpret_cast<uint32_t*>(token + p.slots);
    float* bias_of = reinterpret_cast<float*>(table + p.slots);
    const int tid = threadIdx.x;
    const unsigned S = (unsigned)p.S, bg = blockIdx.x / S, s = blockIdx.x - bg * S;
    const int b = (int)(bg / (unsigned)p.groups), g = (int)(bg - (unsigned)b * (unsigned)p.groups);
    AdjustFirst<kTokensThreads> first(p, b);
    const int j0 = g * p.rows_per_cta, j1 = min(first.live, j0 + p.rows_per_cta);
    if (j0 >= j1) {
        grid_dependency_wait();                                     // (what comes after this kernel comes after the one before it, too)
        return;
    }
    if (tid == 0) sh.twice = 0;
    if (tid < j1 - j0) sh.path_n[tid] = 0;
    for (int i = tid; i < p.slots / 4; i += kTokensThreads) {
        reinterpret_cast<int4*>(token)[i] = make_int4(kNoToken, kNoToken, kNoToken, kNoToken);
        reinterpret_cast<uint4*>(table)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
    auto place = [&](int tok) {
        if (tok < 0 || tok >= p.V) return -1;
        if (S > 1 && (unsigned)tok % S != s) return -1;
        for (int slot = (int)(((unsigned)tok * 2654435769u) >> p.slot_shift);; slot = (slot + 1) & (p.slots - 1)) {
            const int32_t had = atomicCAS(&token[slot], kNoToken, tok);
            if (had == kNoToken || had == tok) return slot;
        }
    };
    if (p.n_bias > 0) gather_biases<kTokensThreads>(p, b, table, bias_of, &sh.twice, place);
    first.for_history(p, b, [&](int i, int tok) {
        const int t = place(tok);
        if (t >= 0) count_use(&table[t], i < first.prompt);
    });
    if (p.penalised && p.token_ids && tid < j1 - j0) sh.path_n[tid] = gather_path(p, b, j0 + tid, 0x7fffffff, nullptr, 0, sh.path[tid], place);
    __syncthreads();
    const Penalty q = first.penalty();
    grid_dependency_wait();                                         // the rows have been copied and masked
    for (int j = j0; j < j1; ++j) {
        const char* x = p.in + ((int64_t)b * p.in_b + (int64_t)j * p.in_row) * E::ES;
        T* y = (T*)(p.out + ((int64_t)b * p.out_b + (int64_t)j * p.out_row) * E::ES);
        const uint32_t* mask = adjust_mask(p, b, j);
        const int np = sh.path_n[j - j0];
        const uint16_t* path = sh.path[j - j0];
        // the path's tokens first, from the values as they are (in place, too); they are written when all others are
        T own{};
        int mine = -1;
        if (tid < np) {
            const int t = path[tid];
            mine = token[t];
            if (mask && !((mask[mine >> 5] >> (mine & 31)) & 1u)) mine = -1;
            else {
                uint32_t times = table[t] / kOnce;
                for (int o = 0; o < np; ++o) times += path[o] == t;
                const double z = penalised(q, E::load(x, mine), times, true);
                own = Raw<DT>::round(table[t] & kHasBias ? z + (double)bias_of[t] : z);
            }
        }
        __syncthreads();
        constexpr int kStep = 4;                                    // slots of a thread under way
#pragma unroll 1
        for (int i0 = tid; i0 < p.slots; i0 += kStep * kTokensThreads) {
            uint32_t word[kStep];
            int v[kStep];
            float old[kStep];
#pragma unroll
            for (int o = 0; o < kStep; ++o) {
                const int i = i0 + o * kTokensThreads;
                word[o] = i < p.slots ? table[i] : 0u;
                v[o] = word[o] ? token[i] : 0;
                old[o] = word[o] ? E::load(x, v[o]) : 0.0f;
                if (mask && word[o] && !((mask[v[o] >> 5] >> (v[o] & 31)) & 1u)) word[o] = 0u;
            }
#pragma unroll
            for (int o = 0; o < kStep; ++o) {
                if (word[o] == 0u) continue;
                const uint32_t times = word[o] / kOnce;
                const double z = penalised(q, old[o], times, times > 0u || (word[o] & kInPrompt));
                y[v[o]] = Raw<DT>::round(word[o] & kHasBias ? z + (double)bias_of[i0 + o * kTokensThreads] : z);
            }
        }
        __syncthreads();
        if (mine >= 0) y[mine] = own;
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
