// Host side of the calls on a round's logits (cadd.h): penalties, biases and masks; distillation.  Argument checks, grids,
// launches.  No allocation, no synchronisation, no state kept between calls.
#include <cuda_runtime.h>
#include <stdint.h>

#include "cadd.h"
#include "adjust_logits.cuh"
#include "distill.cuh"

namespace cadd {

static inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
static int launched() { return cudaGetLastError() == cudaSuccess ? CADD_OK : CADD_ERR_LAUNCH; }
// Grids that only have to be large enough go by a B200's SMs without asking the device, which small calls would feel.
constexpr int kSms = 148;

// A launch in clusters, or a plain one; with `overlap`, one that may be set up while the kernel before it still runs (see launch_dependent).
template <typename P>
static int launch_cluster(void (*kernel)(P), unsigned grid, unsigned threads, unsigned cluster, size_t smem, cudaStream_t st, const P& p, bool overlap = false) {
    if (cluster == 1 && !overlap) {
        kernel<<<grid, threads, smem, st>>>(p);
        return launched();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = overlap ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
        cudaGetLastError();
        return CADD_ERR_LAUNCH;
    }
    return CADD_OK;
}

static int check_logits(int batch, int rows, int64_t V, int dtype, const void* x, int64_t stride_b, int64_t stride_row) {
    if (batch < 1 || batch > (1 << 20) || rows < 1 || rows > 65536 || V < 1 || V >= ((int64_t)1 << 31) || (int64_t)batch * rows >= ((int64_t)1 << 28))
        return CADD_ERR_SHAPE;
    if (dtype != CADD_DTYPE_BF16 && dtype != CADD_DTYPE_FP32) return CADD_ERR_DTYPE;
    if (stride_b < 0 || stride_row < 0 || stride_b >= ((int64_t)1 << 50) || stride_row >= ((int64_t)1 << 40)) return CADD_ERR_SHAPE;
    if (!x) return CADD_ERR_NULL;
    return aligned(x, dtype == CADD_DTYPE_BF16 ? 2 : 4) ? CADD_OK : CADD_ERR_ALIGN;
}
// The same of an output: rows must not lie in one another, whichever axis is the outer one.
static int check_output(int batch, int rows, int64_t V, int dtype, const void* x, int64_t stride_b, int64_t stride_row) {
    const int rc = check_logits(batch, rows, V, dtype, x, stride_b, stride_row);
    if (rc != CADD_OK) return rc;
    const int64_t by_rows = (int64_t)(rows - 1) * stride_row + V, by_batch = (int64_t)(batch - 1) * stride_b + V;
    const bool rows_in = (rows == 1 || stride_row >= V) && (batch == 1 || stride_b >= by_rows);
    const bool batch_in = (batch == 1 || stride_b >= V) && (rows == 1 || stride_row >= by_batch);
    return rows_in || batch_in ? CADD_OK : CADD_ERR_SHAPE;
}

// ---------------- penalties, biases, masks ----------------

// Dynamic shared memory that a kernel may have.  `most` is what any call of it can want: the limit belongs to the process, and a call that set its
// own size would have another thread's larger launch refused.
template <typename K>
static int room(K kernel, size_t most) {
    if (cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) == cudaSuccess) return CADD_OK;
    cudaGetLastError();
    return CADD_ERR_LAUNCH;
}
// Rows a CTA: what they have in common is gathered once for all of them, but the device wants CTAs enough.  Few rows are cut in more pieces,
// as long as each warp has one at most.
static void group_rows(AdjustParams& p, int64_t ctas_a_group, int part_shift) {
    p.groups = (p.R + kAdjustRows - 1) / kAdjustRows;
    while (p.batch * ctas_a_group * p.groups < 4 * kSms && (p.R + p.groups - 1) / p.groups > kAdjustWarps) p.groups *= 2;
    p.rows_per_cta = (p.R + p.groups - 1) / p.groups;
    p.groups = (p.R + p.rows_per_cta - 1) / p.rows_per_cta;
    p.part_shift = part_shift;
    while (p.part_shift < 3 && (p.rows_per_cta << (p.part_shift + 1)) <= kAdjustWarps) ++p.part_shift;
}

template <int DT>
static int launch_tokens(AdjustParams& p, cudaStream_t st) {
    // Rows that share a table; CTAs that share a request's tokens, as many as find room at once (single words anywhere in a row want the
    // load units of all SMs: 64 requests of 8192 tokens 32 us with one CTA each, 20 with two); and fewer rows a CTA where there is room still.
    p.groups = (p.R + kAdjustRows - 1) / kAdjustRows;
    p.S = 1;
    while (p.S < 8 && (int64_t)p.batch * p.groups * (p.S + 1) <= kSms) ++p.S;
    while ((int64_t)p.batch * p.groups * p.S * 2 <= kSms && p.groups < p.R) p.groups *= 2;
    p.rows_per_cta = (p.R + p.groups - 1) / p.groups;
    p.groups = (p.R + p.rows_per_cta - 1) / p.rows_per_cta;
    // Tokens that a CTA can meet: those of its part of the vocabulary, and no more than the history, biases and its rows' paths have.
    int64_t most = (p.penalised && p.history ? p.history_cols : 0) + p.n_bias + (p.penalised && p.token_ids ? (int64_t)p.rows_per_cta * kMaxPath : 0);
    if (most > kTokensMost) {
        const int parts = (int)((p.V + kTokensMost - 1) / kTokensMost);
        if (p.S < parts) p.S = parts;
        most = kTokensMost;
    }
    p.slots = 1024;
    p.slot_shift = 22;
    while (p.slots < kTokensSlots && p.slots * 3 < most * 4) { p.slots *= 2; --p.slot_shift; }
    const int64_t grid = (int64_t)p.batch * p.S * p.groups;
    if (grid >= ((int64_t)1 << 31)) return CADD_ERR_SHAPE;
    const size_t smem = adjust_tokens_smem(p.slots, p.n_bias > 0);
    const int rc = room(adjust_tokens_kernel<DT>, adjust_tokens_smem(kTokensSlots, true));
    if (rc != CADD_OK) return rc;
    return launch_cluster(adjust_tokens_kernel<DT>, (unsigned)grid, kTokensThreads, 1, smem, st, p, p.followed);
}

// Whether adjust_rows_kernel takes the call (us a call on the device, tables against single tokens; 151936 tokens, bf16).  Where all its CTAs
// run at once: one launch is less than two (one token, 5.8 against 6.2; 65 rows of one request in place 13 against 28).  Otherwise from
// four rows a request on (32 requests, histories of 4000: one row 26 against 14, two 26 / 19, three 28 / 25, four 30 / 32, six 40 / 50).
// In place without masks, when it has to write all that it reads, also not where few tokens can be concerned (32 requests of 65 rows: histories
// of 100 tokens 202 against 51, of 4000 211 / 256; with masks 226 / 452).  That border lies somewhere between these two histories, of one vocabulary and
// one tree size; it leaves out that single tokens take longer with more rows.  All goes by the room for a history: its lengths are on the device.
constexpr int kFewRows = 4, kFewTokens = 40;              // one token of so many
static bool by_tables(const AdjustParams& p, bool in_place) {
    const int64_t history = p.penalised && p.history ? p.history_cols : 0;
    if (history > kListMost) return false;
    if ((int64_t)p.batch * p.tiles * ((p.R + kAdjustRows - 1) / kAdjustRows) <= 4 * kSms) return true;
    return p.R >= kFewRows && (!in_place || p.allowed || (history + p.n_bias) * kFewTokens >= p.V);
}

template <int DT>
static int launch_adjust(AdjustParams& p, bool in_place, cudaStream_t st) {
    constexpr int tile = kAdjustTile<DT>;
    p.tiles = (int)((p.V + tile - 1) / tile);
    if (p.status) {
        adjust_status_kernel<<<(unsigned)p.batch, kAdjustThreads, 0, st>>>(p);
        const int rc = launched();
        if (rc != CADD_OK) return rc;
    }
    const bool sparse = p.penalised || p.n_bias > 0;
    if (sparse && by_tables(p, in_place)) {
        group_rows(p, p.tiles, kAdjustTileBytes / kAdjustPieceBytes == 2 ? 1 : 0);
        const int64_t grid = (int64_t)p.batch * p.tiles * p.groups;
        if (grid >= ((int64_t)1 << 31)) return CADD_ERR_SHAPE;
        const size_t smem = (size_t)adjust_layout(tile, p.n_bias).bytes;
        const int rc = room(adjust_rows_kernel<DT>, (size_t)adjust_layout(tile, tile).bytes);
        if (rc != CADD_OK) return rc;
        adjust_rows_kernel<DT><<<(unsigned)grid, kAdjustThreads, smem, st>>>(p);
        return launched();
    }
    if (!in_place || p.allowed) {
        p.followed = sparse;
        const int64_t units = (int64_t)p.batch * p.R * p.tiles;
        int rc = CADD_OK;
        if (in_place) {
            const int64_t most = kSms * 6;
            adjust_stream_kernel<DT, false><<<(unsigned)(units < most ? units : most), kAdjustThreads, 0, st>>>(p);
        } else {
            const size_t smem = (size_t)kAdjustWarps * kAdjustBuffer<kAdjustTileBytes>;
            const int64_t most = kSms * 3;
            if ((rc = room(adjust_stream_kernel<DT, true>, smem)) != CADD_OK) return rc;
            adjust_stream_kernel<DT, true><<<(unsigned)(units < most ? units : most), kAdjustThreads, smem, st>>>(p);
        }
        if ((rc = launched()) != CADD_OK) return rc;
    }
    if (!sparse) return CADD_OK;
    return launch_tokens<DT>(p, st);
}

// ---------------- distillation ----------------

// Chunks of a row at most: its whole 16-byte chunks where it starts on a boundary.
static int64_t row_chunks(int dtype, int64_t V) { return V / (dtype == CADD_DTYPE_BF16 ? 8 : 4); }

constexpr size_t kDistillRoom = 227 * 1024;               // shared memory of a CTA

template <int DT, bool kLoss, bool kGrad>
static int launch_distill(DistillParams& p, cudaStream_t st) {
    const size_t smem = distill_smem_bytes(p.chunks_max, p.K, p.stages);
    const int rc = room(distill_kernel<DT, kLoss, kGrad>, kDistillRoom);
    if (rc != CADD_OK) return rc;
    return launch_cluster(distill_kernel<DT, kLoss, kGrad>, (unsigned)(p.clusters * p.C), kDistillThreads, (unsigned)p.C, smem, st, p);
}

static int distill(const cadd_distill_args* a, bool loss, cudaStream_t st) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_distill_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_logits(a->batch, a->L, a->V, a->logits_dtype, a->logits, a->stride_b, a->stride_l);
    if (rc != CADD_OK) return rc;
    if (a->K < 1 || a->K > CADD_DISTILL_MAX_K || a->R < 1 || a->R > 65536 || a->V > kDistillMaxV) return CADD_ERR_SHAPE;
    if (a->path ? a->path_cols < (a->L > 1 ? 1 : 0) || a->path_cols > 65536 : a->R < a->L) return CADD_ERR_SHAPE;
    if (!(a->temperature >= 0x1p-20 && a->temperature <= 0x1p20)) return CADD_ERR_SHAPE;
    if (!a->teacher_token || !a->teacher_logit || (a->path && !a->path_len)) return CADD_ERR_NULL;
    if (loss ? !a->loss && !a->stats && !a->grad : !a->stats || !a->grad) return CADD_ERR_NULL;
    if (a->grad) {
        if ((rc = check_output(a->batch, a->L, a->V, a->logits_dtype, a->grad, a->grad_stride_b, a->grad_stride_l)) != CADD_OK) return rc;
        if (a->grad == a->logits && ((a->batch > 1 && a->grad_stride_b != a->stride_b) || (a->L > 1 && a->grad_stride_l != a->stride_l))) return CADD_ERR_SHAPE;
    }
    if (!aligned(a->teacher_token, 4) || !aligned(a->teacher_logit, 8) || !aligned(a->teacher_lse, 8) || !aligned(a->path, 4) || !aligned(a->path_len, 4) ||
        !aligned(a->n_rows, 4) || !aligned(a->weight, 4) || !aligned(a->grad_loss, 4) || !aligned(a->loss, 4) || !aligned(a->stats, 16) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    DistillParams p;
    p.logits = (const char*)a->logits; p.grad = (char*)a->grad;
    p.V = a->V; p.in_b = a->stride_b; p.in_row = a->stride_l; p.out_b = a->grad_stride_b; p.out_row = a->grad_stride_l;
    p.L = a->L; p.R = a->R; p.K = a->K; p.path_cols = a->path_cols; p.rest = (a->flags & CADD_DISTILL_REST) ? 1 : 0;
    p.c = (float)(1.4426950408889634 / a->temperature);
    p.over_c = (float)(a->temperature / 1.4426950408889634);
    p.inv_t = 1.0 / a->temperature;
    p.token = a->teacher_token; p.path = a->path; p.path_len = a->path_len; p.n_rows = a->n_rows;
    p.value = a->teacher_logit; p.lse = a->teacher_lse; p.weight = a->weight; p.grad_loss = a->grad_loss;
    p.loss = a->loss; p.stats = a->stats; p.status = a->status;
    p.drop = (a->flags & CADD_FLAG_TEST_DROP_TILE) ? 1 : -1;
    const int64_t rows = (int64_t)a->batch * a->L, chunks = row_chunks(a->logits_dtype, a->V);
    // One CTA an SM, for whole rows; where there are fewer rows than SMs they are cut in up to four (16 rows of 151936: whole 14.2 us, in two
    // 13.8, in four 11.5, in eight 18.7: so large clusters do not all find room at once).
    int C = 1;
    while (C < kDistillMaxC && rows * (C + 1) <= kSms && (chunks + C - 1) / C > kDistillCompute) ++C;
    p.rows = (int)rows;
    p.batch = a->batch;
    p.C = C;
    p.chunks_max = (int)((chunks + C - 1) / C);
    p.clusters = (int)(kSms / C < rows ? kSms / C : rows);
    p.stages = (int)((kDistillRoom - distill_ring_at(p.chunks_max, a->K)) / (kDistillTile * 16));
    if (p.stages > kDistillMaxStages) p.stages = kDistillMaxStages;
    const int tiles = (p.chunks_max + kDistillTile - 1) / kDistillTile;
    if (p.stages > tiles && p.clusters == rows) p.stages = tiles > 0 ? tiles : 1;
    if (a->status) {
        distill_status_kernel<<<(unsigned)a->batch, kDistillStatusThreads, 0, st>>>(p);
        if ((rc = launched()) != CADD_OK) return rc;
    }
    const bool bf16 = a->logits_dtype == CADD_DTYPE_BF16;
    if (!loss) return bf16 ? launch_distill<CADD_DTYPE_BF16, false, true>(p, st) : launch_distill<CADD_DTYPE_FP32, false, true>(p, st);
    if (a->grad) return bf16 ? launch_distill<CADD_DTYPE_BF16, true, true>(p, st) : launch_distill<CADD_DTYPE_FP32, true, true>(p, st);
    return bf16 ? launch_distill<CADD_DTYPE_BF16, true, false>(p, st) : launch_distill<CADD_DTYPE_FP32, true, false>(p, st);
}

}  // namespace cadd

using namespace cadd;

extern "C" {

int cadd_adjust_logits(const cadd_adjust_args* a, void* cuda_stream) {
    if (!a) return CADD_ERR_NULL;
    if (a->struct_size != sizeof(cadd_adjust_args)) return CADD_ERR_STRUCT_SIZE;
    int rc = check_logits(a->batch, a->R, a->V, a->logits_dtype, a->logits, a->stride_b, a->stride_row);
    if (rc == CADD_OK) rc = check_output(a->batch, a->R, a->V, a->logits_dtype, a->out, a->out_stride_b, a->out_stride_row);
    if (rc != CADD_OK) return rc;
    const bool in_place = a->out == a->logits;
    if (in_place && ((a->batch > 1 && a->out_stride_b != a->stride_b) || (a->R > 1 && a->out_stride_row != a->stride_row))) return CADD_ERR_SHAPE;
    if (a->n_bias < 0 || a->n_bias > 65536) return CADD_ERR_SHAPE;
    if (a->history && (a->history_cols < 1 || a->history_cols >= (1 << 30) || a->history_stride < 0 || a->history_stride >= ((int64_t)1 << 50))) return CADD_ERR_SHAPE;
    if (a->allowed && a->n_allowed < 1) return CADD_ERR_SHAPE;
    if ((a->n_bias > 0 && (!a->bias_token || !a->bias)) || (a->token_ids && !a->parent_idx) || (a->allowed && !a->allowed_row)) return CADD_ERR_NULL;
    if (!aligned(a->n_nodes, 4) || !aligned(a->token_ids, 4) || !aligned(a->parent_idx, 4) || !aligned(a->history, 4) || !aligned(a->history_len, 4) ||
        !aligned(a->prompt_len, 4) || !aligned(a->repetition, 4) || !aligned(a->presence, 4) || !aligned(a->frequency, 4) || !aligned(a->bias_token, 4) ||
        !aligned(a->bias, 4) || !aligned(a->allowed, 4) || !aligned(a->allowed_row, 4) || !aligned(a->status, 4))
        return CADD_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    AdjustParams p;
    p.in = (const char*)a->logits; p.out = (char*)a->out;
    p.V = a->V; p.in_b = a->stride_b; p.in_row = a->stride_row; p.out_b = a->out_stride_b; p.out_row = a->out_stride_row;
    p.batch = a->batch; p.R = a->R;
    p.n_bias = a->n_bias; p.history_cols = a->history_cols; p.n_allowed = a->n_allowed; p.words = (int)((a->V + 31) / 32);
    p.followed = false;
    p.penalised = a->repetition || a->presence || a->frequency;
    p.n_nodes = a->n_nodes; p.token_ids = a->token_ids; p.parent_idx = a->parent_idx;
    p.history = a->history; p.history_len = a->history_len; p.prompt_len = a->prompt_len; p.history_stride = a->history_stride;
    p.bias_token = a->bias_token; p.bias = a->bias; p.allowed = a->allowed; p.allowed_row = a->allowed_row;
    p.repetition = a->repetition; p.presence = a->presence; p.frequency = a->frequency;
    p.status = a->status;
    p.drop = (a->flags & CADD_FLAG_TEST_DROP_TILE) ? 1 : 0;
    return a->logits_dtype == CADD_DTYPE_BF16 ? launch_adjust<CADD_DTYPE_BF16>(p, in_place, st) : launch_adjust<CADD_DTYPE_FP32>(p, in_place, st);
}

int cadd_distill_loss(const cadd_distill_args* a, void* cuda_stream) { return distill(a, true, (cudaStream_t)cuda_stream); }
int cadd_distill_grad(const cadd_distill_args* a, void* cuda_stream) { return distill(a, false, (cudaStream_t)cuda_stream); }

}  // extern "C"
