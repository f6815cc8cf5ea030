// Host side of the cache and tree-attention calls of the C ABI (cadd.h): argument checks, grids, launches.  No allocation,
// no synchronisation, no state kept between calls.
#include <cuda_runtime.h>
#include <stdint.h>

#include "cadd.h"
#include "cache.cuh"
#include "tree_attention.cuh"
#include "cache_evict.cuh"
#include "attn_tiles.cuh"
#include "attn_few.cuh"
#include "launch.cuh"

namespace cadd {

static inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

static int check_cache_shape(const cadd_cache* c) {
    if (c->struct_size != sizeof(cadd_cache)) return CADD_ERR_STRUCT_SIZE;
    if (c->format != CADD_CACHE_BF16 && c->format != CADD_CACHE_FP4) return CADD_ERR_DTYPE;
    if (c->batch < 1 || c->batch > (1 << 20) || c->heads < 1 || c->heads > 4096 || (c->head_dim != 64 && c->head_dim != 128)) return CADD_ERR_SHAPE;
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return CADD_ERR_SHAPE;
    if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size >= ((int64_t)1 << 30)) return CADD_ERR_SHAPE;
    if ((int64_t)c->batch * c->heads > ((int64_t)1 << 24)) return CADD_ERR_SHAPE;
    if (c->format == CADD_CACHE_BF16 ? (c->k_exp != 0 || c->v_exp != 0) : (c->k_exp < -16 || c->k_exp > 16 || c->v_exp < -16 || c->v_exp > 16))
        return CADD_ERR_SHAPE;
    return CADD_OK;
}
static int check_cache(const cadd_cache* c) {
    int rc = check_cache_shape(c);
    if (rc != CADD_OK) return rc;
    if (c->n_pages < 1 || c->n_pages >= ((int64_t)1 << 31) || c->stride_page < 1 || c->stride_head < 1 || c->stride_slot < 1) return CADD_ERR_SHAPE;
    if (c->stride_page >= ((int64_t)1 << 40) || c->stride_head >= ((int64_t)1 << 40) || c->stride_slot >= ((int64_t)1 << 40)) return CADD_ERR_SHAPE;
    if (!c->k || !c->v || !c->block_table || !c->length) return CADD_ERR_NULL;
    if (c->format == CADD_CACHE_FP4 && (!c->k_scale || !c->v_scale)) return CADD_ERR_NULL;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->block_table, 4) || !aligned(c->length, 4)) return CADD_ERR_ALIGN;
    if (c->format == CADD_CACHE_FP4 && (!aligned(c->k_scale, 8) || !aligned(c->v_scale, 8))) return CADD_ERR_ALIGN;
    return CADD_OK;
}
static CacheView view_of(const cadd_cache* c) {
    CacheView v;
    v.k = (unsigned char*)c->k; v.v = (unsigned char*)c->v;
    v.ks = (unsigned char*)c->k_scale; v.vs = (unsigned char*)c->v_scale;
    v.block_table = c->block_table; v.length = c->length;
    v.stride_page = c->stride_page; v.stride_head = c->stride_head; v.stride_slot = c->stride_slot;
    v.n_pages = c->n_pages;
    v.batch = c->batch; v.heads = c->heads; v.head_dim = c->head_dim; v.max_pages = c->max_pages;
    v.page_shift = 0;
    while ((1 << v.page_shift) < c->page_size) ++v.page_shift;
    v.fp4 = c->format == CADD_CACHE_FP4;
    v.k_exp = c->k_exp; v.v_exp = c->v_exp;
    v.row_bytes = v.fp4 ? c->head_dim / 2 : c->head_dim * 2;
    return v;
}
// Strides of a dense bf16 operand [batch, rows, heads, head_dim] in elements: 16-byte steps, no negative ones.
static int check_strides(int64_t b, int64_t row, int64_t head) {
    if (b < 0 || row < 0 || head < 0 || b >= ((int64_t)1 << 50) || row >= ((int64_t)1 << 40) || head >= ((int64_t)1 << 40)) return CADD_ERR_SHAPE;
    return (b % 8 || row % 8 || head % 8) ? CADD_ERR_ALIGN : CADD_OK;
}
// The same of an output: along an axis longer than one, rows must not lie in one another.
static int check_out_strides(int64_t b, int64_t row, int64_t head, const cadd_cache* c, int64_t rows, int64_t heads) {
    const int rc = check_strides(b, row, head);
    if (rc != CADD_OK) return rc;
    return (c->batch > 1 && b < c->head_dim) || (rows > 1 && row < c->head_dim) || (heads > 1 && head < c->head_dim) ? CADD_ERR_SHAPE : CADD_OK;
}
// Beyond these the scores' factors, scale * 2^(what the 4-bit form leaves), leave fp32's range, and a masked score times 0 is NaN.
static bool scale_in_range(float scale) { return scale >= 0x1p-64f && scale <= 0x1p64f; }
static int launched() {
    return cudaGetLastError() == cudaSuccess ? CADD_OK : CADD_ERR_LAUNCH;
}
// Grids that only have to be large enough go by a B200's SMs without asking the device, which small calls would feel.
constexpr int kSms = 148;
static int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return kSms;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return kSms;
    return n;
}
// CTAs for one of `groups` equal pieces of work of up to `items` thread items each: enough to fill the device a few times over.
static int ctas_for(int64_t groups, int64_t items, int threads) {
    int64_t need = (items + threads - 1) / threads, most = (kSms * 32 + groups - 1) / groups;
    if (need < 1) need = 1;
    return (int)(need < most ? need : most);
}

constexpr int kMaxGrid = 512;                             // ranges at most (two CTAs on each SM are fewer)
constexpr size_t kItemsBytes = ((size_t)kMaxGrid * (sizeof(int4) + sizeof(int)) + 255) & ~(size_t)255;

// Units that a call can have at most: what its tables and row capacity have room for.
static int64_t most_units(const AttnParams& p, int bm) {
    const int64_t blocks = ((int64_t)p.R * p.group + bm - 1) / bm;
    const int64_t keys = (((int64_t)p.c.max_pages << p.c.page_shift) + kUnit - 1) / kUnit + (p.R + kUnit - 1) / kUnit;
    return (int64_t)p.c.batch * p.c.heads * blocks * keys;
}

// Attention kernel on up to `ctas` ranges, then the join.
template <int BM, int D, bool FP4>
static int launch_attention(void (*kernel)(AttnWork), AttnWork& w, int64_t ctas, int threads, size_t smem, cudaStream_t st) {
    if (cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        cudaGetLastError();
        return CADD_ERR_LAUNCH;
    }
    if (ctas > kMaxGrid) ctas = kMaxGrid;
    // where every unit can have a CTA of its own, items need not be weighed against one another
    w.p.item_cost = 0;
    int64_t grid = most_units(w.p, BM);
    if (grid > ctas) {
        grid = ctas;
        w.p.item_cost = kItemCost;
    }
    kernel<<<(unsigned)grid, threads, smem, st>>>(w);
    if (cudaGetLastError() != cudaSuccess) return CADD_ERR_LAUNCH;
    const dim3 join((unsigned)grid, BM / kJoinRows);
    if (launch_dependent(true, attn_join_kernel<BM, D, FP4>, join, dim3(kJoinRows * D / 8), 0, st, w, (int)grid) != cudaSuccess) {
        cudaGetLastError();
        return CADD_ERR_LAUNCH;
    }
    return CADD_OK;
}
// Up to 16 rows of a head (as many as the call has room for: live rows are not known here) over a 4-bit cache go to the kernel that
// walks the cache with registers, all else to the one with tensor memory.  Measured on a B200, 4 query heads to each of 8 key
// heads, this kernel / that one: 64 tokens over up to 8191 places 211 / 227 us, 16 over up to 32k 180 / 215, one over 32k 37 / 42,
// 8 trees of 4 rows over up to 16k 68 / 80; scores so far apart that every step is in bf16, 16 over up to 32k, 197 / 216.
template <int D, bool FP4>
static int launch_tree_attention(AttnWork& w, bool tiled, cudaStream_t st) {
    if constexpr (FP4) {
        if (!tiled && (int64_t)w.p.R * w.p.group <= kFewRows)
            return launch_attention<kFewRows, D, true>(attn_few_kernel<D>, w, 2 * (int64_t)sm_count(), kFewThreads, sizeof(FewShared<D>), st);
    }
    return launch_attention<kTileBM, D, FP4>(attn_tiles_kernel<D, FP4>, w, 2 * (int64_t)sm_count(), kTileThreads, tile_smem_bytes<D>(), st);
}

template <int D, bool FP4>
static int launch_weights(WeightsParams& p, int64_t cap, cudaStream_t st) {
    // Keys of a CTA: 2048 (32 requests of up to 32k tokens, measured while totals were not yet fetched ahead: 236 us; 1024: 255,
    // 4096: 248, 8192: 325), less where that would leave the device short of CTAs, 128 (32 a warp) at least.
    const int64_t bh = (int64_t)p.c.batch * p.c.heads, enough = 6 * kSms;
    p.keys_per_cta = 2048;
    while (p.keys_per_cta > 128 && bh * ((cap + p.keys_per_cta - 1) / p.keys_per_cta) < enough) p.keys_per_cta >>= 1;
    const int64_t per_head = (cap + p.keys_per_cta - 1) / p.keys_per_cta;
    if (bh * per_head >= ((int64_t)1 << 31)) return CADD_ERR_SHAPE;
    p.ctas_per_head = (int)per_head;
    if (cudaFuncSetAttribute(weights_kernel<D, FP4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(WeightsShared<D>)) != cudaSuccess) {
        cudaGetLastError();
        return CADD_ERR_LAUNCH;
    }
    weights_kernel<D, FP4><<<(unsigned)(bh * per_head), kWThreads, sizeof(WeightsShared<D>), st>>>(p);
    return launched();
}

}  // namespace cadd

using namespace cadd;

extern "C" {

int cadd_cache_append(const cadd_append_args* a, void* cuda_stream) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_append_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_cache(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->R < 1 || a->R > (1 << 24) || (a->path && (a->L < 1 || a->L > 65536))) return CADD_ERR_SHAPE;
    if (!a->k || !a->v || !a->new_length || (a->path && !a->path_len)) return CADD_ERR_NULL;
    rc = check_strides(a->stride_b, a->stride_row, a->stride_head);
    if (rc != CADD_OK) return rc;
    if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->n_rows, 4) || !aligned(a->path, 4) || !aligned(a->path_len, 4) ||
        !aligned(a->new_length, 4) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    AppendParams p;
    p.c = view_of(&a->cache);
    p.k = (const unsigned char*)a->k; p.v = (const unsigned char*)a->v;
    p.stride_b = a->stride_b; p.stride_row = a->stride_row; p.stride_head = a->stride_head;
    p.rows = RowList{a->n_rows, a->path, a->path_len, a->R, a->L};
    const bool in_place = a->new_length == a->cache.length;
    p.new_length = in_place ? nullptr : a->new_length;
    p.status = a->status;
    p.ctas_per_request = ctas_for(p.c.batch, (int64_t)(a->path ? a->L + 1 : a->R) * p.c.heads * (p.c.head_dim / 16), kCopyThreads);
    const unsigned grid = (unsigned)p.c.batch * (unsigned)p.ctas_per_request;
    if (p.c.fp4) cache_append_kernel<true><<<grid, kCopyThreads, 0, st>>>(p);
    else cache_append_kernel<false><<<grid, kCopyThreads, 0, st>>>(p);
    rc = launched();
    if (rc != CADD_OK || !in_place) return rc;
    cache_advance_kernel<<<(unsigned)(p.c.batch + 127) / 128, 128, 0, st>>>(p.c, p.rows, a->new_length);
    return launched();
}

int cadd_cache_read(const cadd_read_args* a, void* cuda_stream) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_read_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_cache(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->n_max < 1 || a->n_max > (1 << 30)) return CADD_ERR_SHAPE;
    if (!a->k || !a->v) return CADD_ERR_NULL;
    rc = check_out_strides(a->stride_b, a->stride_row, a->stride_head, &a->cache, a->n_max, a->cache.heads);
    if (rc != CADD_OK) return rc;
    if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->start, 4) || !aligned(a->count, 4) || !aligned(a->status, 4)) return CADD_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    ReadParams p;
    p.c = view_of(&a->cache);
    p.k = (unsigned char*)a->k; p.v = (unsigned char*)a->v;
    p.stride_b = a->stride_b; p.stride_row = a->stride_row; p.stride_head = a->stride_head;
    p.start = a->start; p.count = a->count; p.n_max = a->n_max; p.status = a->status;
    const int64_t cap = (int64_t)a->cache.max_pages * a->cache.page_size;
    p.ctas_per_request = ctas_for(p.c.batch, (a->n_max < cap ? a->n_max : cap) * p.c.heads * (p.c.head_dim / 16), kCopyThreads);
    const unsigned grid = (unsigned)p.c.batch * (unsigned)p.ctas_per_request;
    if (p.c.fp4) cache_read_kernel<true><<<grid, kCopyThreads, 0, st>>>(p);
    else cache_read_kernel<false><<<grid, kCopyThreads, 0, st>>>(p);
    return launched();
}

// ---------------- tree attention ----------------

static int check_attention_shape(const cadd_attention_args* a) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_attention_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_cache_shape(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->R < 1 || a->R > 65536 || a->heads_q < 1 || a->heads_q > 65536 || a->heads_q % a->cache.heads) return CADD_ERR_SHAPE;
    if ((int64_t)a->R * (a->heads_q / a->cache.heads) > ((int64_t)1 << 24)) return CADD_ERR_SHAPE;
    if ((int64_t)a->cache.batch * a->R * a->heads_q >= ((int64_t)1 << 33)) return CADD_ERR_SHAPE;
    return CADD_OK;
}

int cadd_tree_attention_workspace_bytes(const cadd_attention_args* a, size_t* out) {
    int rc = check_attention_shape(a);
    if (rc != CADD_OK) return rc;
    if (!out) return CADD_ERR_NULL;
    // two records per range of the grid with the larger records
    const size_t rec = (size_t)kTileBM * (a->cache.head_dim + 2) * 4;
    *out = kItemsBytes + (size_t)kMaxGrid * 2 * rec;
    return CADD_OK;
}

int cadd_tree_attention(const cadd_attention_args* a, void* cuda_stream) {
    int rc = check_attention_shape(a);
    if (rc != CADD_OK) return rc;
    rc = check_cache(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->window < 0 || a->n_sinks < 0 || a->n_sinks > (1 << 30) || !scale_in_range(a->scale)) return CADD_ERR_SHAPE;
    if (!a->q || !a->k || !a->v || !a->out) return CADD_ERR_NULL;
    if (a->mask_bits && a->window && !a->depth) return CADD_ERR_NULL;
    if ((rc = check_strides(a->q_stride_b, a->q_stride_row, a->q_stride_head)) != CADD_OK ||
        (rc = check_strides(a->kv_stride_b, a->kv_stride_row, a->kv_stride_head)) != CADD_OK ||
        (rc = check_out_strides(a->out_stride_b, a->out_stride_row, a->out_stride_head, &a->cache, a->R, a->heads_q)) != CADD_OK)
        return rc;
    if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->out, 16) || !aligned(a->n_nodes, 4) ||
        !aligned(a->mask_bits, 4) || !aligned(a->depth, 4) || !aligned(a->lse, 4) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    size_t need = 0;
    cadd_tree_attention_workspace_bytes(a, &need);
    if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < need) return CADD_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    AttnParams p;
    p.c = view_of(&a->cache);
    p.q = (const unsigned char*)a->q; p.k = (const unsigned char*)a->k; p.v = (const unsigned char*)a->v; p.out = (unsigned char*)a->out;
    p.qs_b = a->q_stride_b; p.qs_row = a->q_stride_row; p.qs_head = a->q_stride_head;
    p.kvs_b = a->kv_stride_b; p.kvs_row = a->kv_stride_row; p.kvs_head = a->kv_stride_head;
    p.os_b = a->out_stride_b; p.os_row = a->out_stride_row; p.os_head = a->out_stride_head;
    p.n_nodes = a->n_nodes; p.depth = a->depth; p.mask_bits = a->mask_bits; p.lse = a->lse; p.status = a->status;
    p.R = a->R; p.heads_q = a->heads_q; p.group = a->heads_q / a->cache.heads; p.window = a->window; p.n_sinks = a->n_sinks;
    p.mask_words = (a->R + 31) / 32;
    p.scale_log2 = (float)((double)a->scale * 1.4426950408889634);
    p.test_drop = (a->flags & CADD_FLAG_TEST_DROP_TILE) ? 1 : 0;
    p.wait_limit = p.test_drop ? kTileTestWaitLimit : kTileWaitLimit;
    AttnWork w;
    w.p = p;
    w.items = (int4*)a->workspace;
    w.odd = (int*)(w.items + kMaxGrid);
    w.records = (float*)((unsigned char*)a->workspace + kItemsBytes);
    const bool tiled = (a->flags & (CADD_ATTENTION_TILED_PATH | CADD_FLAG_TEST_DROP_TILE)) != 0;
    if (p.c.head_dim == 128) return p.c.fp4 ? launch_tree_attention<128, true>(w, tiled, st) : launch_tree_attention<128, false>(w, tiled, st);
    return p.c.fp4 ? launch_tree_attention<64, true>(w, tiled, st) : launch_tree_attention<64, false>(w, tiled, st);
}

// ---------------- accumulated weights, eviction ----------------

int cadd_cache_weights(const cadd_weights_args* a, void* cuda_stream) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_weights_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_cache(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->R < 1 || a->R > 65536 || (a->path && (a->L < 1 || a->L > 65536)) || a->heads_q < 1 || a->heads_q > 65536 || a->heads_q % a->cache.heads)
        return CADD_ERR_SHAPE;
    if (((int64_t)(a->path ? a->L + 1 : a->R) * (a->heads_q / a->cache.heads)) > ((int64_t)1 << 24)) return CADD_ERR_SHAPE;
    if (a->window < 0 || a->n_sinks < 0 || a->n_sinks > (1 << 30) || !scale_in_range(a->scale)) return CADD_ERR_SHAPE;
    const int64_t cap = (int64_t)a->cache.max_pages * a->cache.page_size;
    if (a->weights_stride < cap || a->weights_stride >= ((int64_t)1 << 36)) return CADD_ERR_SHAPE;
    if (!a->q || !a->lse || !a->base_length || !a->weights || !a->weights_out || (a->path && !a->path_len)) return CADD_ERR_NULL;
    if ((rc = check_strides(a->q_stride_b, a->q_stride_row, a->q_stride_head)) != CADD_OK) return rc;
    if (!aligned(a->q, 16) || !aligned(a->lse, 4) || !aligned(a->n_rows, 4) || !aligned(a->path, 4) || !aligned(a->path_len, 4) ||
        !aligned(a->base_length, 4) || !aligned(a->weights, 4) || !aligned(a->weights_out, 4) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    WeightsParams p;
    p.c = view_of(&a->cache);
    p.q = (const unsigned char*)a->q;
    p.qs_b = a->q_stride_b; p.qs_row = a->q_stride_row; p.qs_head = a->q_stride_head;
    p.lse = a->lse;
    p.rows = RowList{a->n_rows, a->path, a->path_len, a->R, a->L};
    p.base_length = a->base_length; p.w_in = a->weights; p.w_out = a->weights_out; p.w_stride = a->weights_stride; p.status = a->status;
    p.heads_q = a->heads_q; p.group = a->heads_q / a->cache.heads; p.window = a->window; p.n_sinks = a->n_sinks;
    p.scale_log2 = (float)((double)a->scale * 1.4426950408889634);
    if (a->status) {
        weights_status_kernel<<<(unsigned)p.c.batch, 128, 0, st>>>(p);
        if ((rc = launched()) != CADD_OK) return rc;
    }
    if (p.c.head_dim == 128) return p.c.fp4 ? launch_weights<128, true>(p, cap, st) : launch_weights<128, false>(p, cap, st);
    return p.c.fp4 ? launch_weights<64, true>(p, cap, st) : launch_weights<64, false>(p, cap, st);
}

int cadd_cache_evict(const cadd_evict_args* a, void* cuda_stream) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_evict_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_cache(&a->cache);
    if (rc != CADD_OK) return rc;
    if (a->n_sinks < 0 || a->n_recent < 0 || a->budget < 1 || a->budget > (1 << 30) || a->new_max_pages < 1 ||
        (int64_t)a->new_max_pages * a->cache.page_size >= ((int64_t)1 << 30))
        return CADD_ERR_SHAPE;
    const int64_t new_cap = (int64_t)a->new_max_pages * a->cache.page_size;
    const int room = (int)(a->budget < new_cap ? a->budget : new_cap);
    if ((int64_t)a->n_sinks + a->n_recent > room) return CADD_ERR_SHAPE;
    const int64_t cap = (int64_t)a->cache.max_pages * a->cache.page_size;
    if (a->weights_stride < cap || a->weights_stride >= ((int64_t)1 << 36)) return CADD_ERR_SHAPE;
    if (a->weights_out && (a->weights_out_stride < room || a->weights_out_stride >= ((int64_t)1 << 36) || a->weights_out == a->weights)) return CADD_ERR_SHAPE;
    if (!a->weights || !a->new_block_table || !a->new_length || !a->kept) return CADD_ERR_NULL;
    if (!aligned(a->weights, 4) || !aligned(a->new_block_table, 4) || !aligned(a->new_length, 4) || !aligned(a->kept, 4) ||
        !aligned(a->weights_out, 4) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    EvictParams p;
    p.c = view_of(&a->cache);
    p.weights = a->weights; p.w_stride = a->weights_stride; p.new_table = a->new_block_table;
    const bool in_place = a->new_length == a->cache.length;
    p.new_length = in_place ? nullptr : a->new_length;
    p.kept = a->kept; p.status = a->status; p.w_out = a->weights_out; p.w_out_stride = a->weights_out_stride;
    p.budget = a->budget; p.room = room; p.n_sinks = a->n_sinks; p.n_recent = a->n_recent; p.new_max_pages = a->new_max_pages;
    const int64_t bh = (int64_t)p.c.batch * p.c.heads;
    evict_select_kernel<<<(unsigned)bh, kSelectThreads, 0, st>>>(p);
    if ((rc = launched()) != CADD_OK) return rc;
    const int ctas = ctas_for(bh, (room < cap ? room : cap) * (p.c.head_dim / (p.c.fp4 ? 32 : 16)), kCopyThreads);
    if (launch_dependent(true, p.c.fp4 ? evict_copy_kernel<true> : evict_copy_kernel<false>, dim3((unsigned)(bh * ctas)), dim3(kCopyThreads), 0, st, p, ctas) != cudaSuccess) {
        cudaGetLastError();
        return CADD_ERR_LAUNCH;
    }
    rc = CADD_OK;
    if (!in_place) return rc;
    evict_length_kernel<<<(unsigned)(p.c.batch + 127) / 128, 128, 0, st>>>(p.c, p.room, a->new_length);
    return launched();
}

}  // extern "C"
