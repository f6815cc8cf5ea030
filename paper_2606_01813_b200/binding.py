"""Thin ctypes binding of the C ABI in include/cadd.h.  Argument marshalling only: every step of the
path runs in the CUDA kernels of libcadd.so.  There is no CPU fallback: if the library is missing
or the tensors are not on a CUDA device the calls raise.

PyTorch is used for device memory and streams.  The functions carry the names of the C entry
points (cadd_build_tree, cadd_verify_tree, ...)."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcadd.so")

OK = 0
ERR_NULL, ERR_STRUCT_SIZE, ERR_SHAPE, ERR_DTYPE, ERR_ALIGN, ERR_WORKSPACE, ERR_LAUNCH = -1, -2, -3, -4, -5, -6, -7
STATUS_NONFINITE_INPUT, STATUS_FEWER_THAN_K_FINITE, STATUS_CAP_HIT, STATUS_FRONTIER_EXHAUSTED = 1, 2, 4, 8
STATUS_L_EFF_CLAMPED, STATUS_COST_NONPOSITIVE, STATUS_BAD_N_NODES, STATUS_INTERNAL_TIMEOUT = 16, 32, 64, 128
STATUS_BAD_TABLE_IDX = 256
STATUS_BAD_PAGE, STATUS_BAD_LENGTH, STATUS_CACHE_FULL, STATUS_BAD_PATH = 512, 1024, 2048, 4096
STATUS_BAD_MASK, STATUS_NOTHING_ALLOWED, STATUS_BAD_TOKEN = 8192, 16384, 32768
DISTILL_REST, DISTILL_MAX_K = 1, 256
CACHE_BF16, CACHE_FP4 = 0, 1
ATTENTION_TILED_PATH = 1                          # small calls too take the kernel that large ones take
DTYPE_BF16, DTYPE_FP32 = 0, 1
COST_QUADRATIC, COST_TABLE, COST_TABLE_INTERP = 0, 1, 2
FLAG_EMIT_DENSE_MASK, FLAG_EMIT_TOPK, FLAG_FIXED_BUDGET = 1, 2, 4
FLAG_ONLY_TOPK, FLAG_ONLY_EXPAND = 8, 16          # measurement aids: one of the two build kernels alone
VERIFY_ONLY_ARGMAX, VERIFY_ONLY_WALK = 1, 2       # the same for cadd_verify_tree
FLAG_TEST_DROP_TILE = 0x80000000                  # test hook: one tile per row is never copied, its wait gives up
FLAG_REGULAR_PATH, VERIFY_REGULAR_PATH = 32, 4    # small problems too take the two-kernel path
# Tests set this to run small shapes through the regular two-kernel path as well (it only adds the two flags above).
FORCE_REGULAR_PATH = False
ROWS_LIVE, ROWS_DENSE = 0, 1

EXPORTS = ("cadd_version", "cadd_status_string", "cadd_build_workspace_bytes", "cadd_verify_workspace_bytes",
           "cadd_build_tree", "cadd_verify_tree", "cadd_build_tree_static_scratch", "cadd_build_launches", "cadd_verify_launches",
           "cadd_head_workspace_bytes", "cadd_verify_tree_fused_head", "cadd_fit_cost_tables",
           "cadd_build_head_workspace_bytes", "cadd_build_tree_fused_head", "cadd_verify_tree_sampled",
           "cadd_cache_append", "cadd_cache_read", "cadd_tree_attention_workspace_bytes", "cadd_tree_attention",
           "cadd_cache_weights", "cadd_cache_evict", "cadd_adjust_logits", "cadd_distill_loss", "cadd_distill_grad")
ERR_STATIC_SCRATCH = -8
STATIC_SCRATCH_BYTES = 8 << 20


class BuildArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32),
        ("batch", C.c_int32), ("L", C.c_int32), ("K", C.c_int32), ("B_max", C.c_int32), ("R", C.c_int32),
        ("logits_dtype", C.c_int32), ("V", C.c_int64),
        ("draft_logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_l", C.c_int64),
        ("l_eff", C.c_void_p), ("bonus_token", C.c_void_p), ("ctx_len", C.c_void_p),
        ("cost_kind", C.c_int32), ("n_tables", C.c_int32),
        ("cost_coef", C.c_void_p), ("cost_table", C.c_void_p), ("table_idx", C.c_void_p), ("t_draft", C.c_void_p),
        ("ctx_grid", C.c_void_p),
        ("n_nodes", C.c_void_p), ("token_ids", C.c_void_p), ("parent_idx", C.c_void_p), ("depth", C.c_void_p),
        ("position_ids", C.c_void_p), ("node_logprob", C.c_void_p), ("phi", C.c_void_p), ("theta", C.c_void_p),
        ("theta_curve", C.c_void_p),
        ("mask_bits", C.c_void_p), ("mask_dense", C.c_void_p), ("topk_token", C.c_void_p),
        ("topk_logprob", C.c_void_p), ("status", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class VerifyArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32),
        ("batch", C.c_int32), ("L", C.c_int32), ("R", C.c_int32),
        ("logits_dtype", C.c_int32), ("rows_mode", C.c_int32), ("reserved0", C.c_int32), ("V", C.c_int64),
        ("target_logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_row", C.c_int64),
        ("n_nodes", C.c_void_p), ("token_ids", C.c_void_p), ("parent_idx", C.c_void_p),
        ("node_argmax", C.c_void_p), ("accepted_len", C.c_void_p), ("accepted_nodes", C.c_void_p),
        ("next_bonus", C.c_void_p), ("status", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class HeadArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32),
        ("batch", C.c_int32), ("L", C.c_int32), ("R", C.c_int32), ("hidden", C.c_int32),
        ("rows_mode", C.c_int32), ("reserved0", C.c_int32), ("V", C.c_int64),
        ("hidden_states", C.c_void_p), ("stride_row", C.c_int64),
        ("weight", C.c_void_p), ("stride_w", C.c_int64),
        ("n_nodes", C.c_void_p), ("token_ids", C.c_void_p), ("parent_idx", C.c_void_p),
        ("node_argmax", C.c_void_p), ("accepted_len", C.c_void_p), ("accepted_nodes", C.c_void_p),
        ("next_bonus", C.c_void_p), ("status", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class BuildHeadArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("hidden", C.c_int32), ("reserved0", C.c_int32),
        ("hidden_states", C.c_void_p), ("stride_row", C.c_int64), ("weight", C.c_void_p), ("stride_w", C.c_int64),
        ("build", BuildArgs),
    ]


class SampleArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32),
        ("batch", C.c_int32), ("L", C.c_int32), ("R", C.c_int32),
        ("logits_dtype", C.c_int32), ("rows_mode", C.c_int32), ("reserved0", C.c_int32), ("V", C.c_int64),
        ("temperature", C.c_double),
        ("target_logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_row", C.c_int64),
        ("uniforms", C.c_void_p),
        ("n_nodes", C.c_void_p), ("token_ids", C.c_void_p), ("parent_idx", C.c_void_p),
        ("node_token", C.c_void_p), ("accepted_len", C.c_void_p), ("accepted_nodes", C.c_void_p),
        ("next_bonus", C.c_void_p), ("status", C.c_void_p),
    ]


class FitArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_tables", C.c_int32), ("N", C.c_int32),
        ("y", C.c_void_p), ("fit", C.c_void_p), ("n_breaks", C.c_void_p), ("status", C.c_void_p),
    ]


class CacheArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("format", C.c_int32), ("batch", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
        ("page_size", C.c_int32), ("max_pages", C.c_int32), ("k_exp", C.c_int32), ("v_exp", C.c_int32), ("reserved0", C.c_int32),
        ("n_pages", C.c_int64), ("stride_page", C.c_int64), ("stride_head", C.c_int64), ("stride_slot", C.c_int64),
        ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
        ("block_table", C.c_void_p), ("length", C.c_void_p),
    ]


class AppendArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("R", C.c_int32), ("L", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p), ("stride_b", C.c_int64), ("stride_row", C.c_int64), ("stride_head", C.c_int64),
        ("n_rows", C.c_void_p), ("path", C.c_void_p), ("path_len", C.c_void_p), ("new_length", C.c_void_p), ("status", C.c_void_p),
        ("cache", CacheArgs),
    ]


class ReadArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_max", C.c_int32), ("reserved0", C.c_int32),
        ("start", C.c_void_p), ("count", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
        ("stride_b", C.c_int64), ("stride_row", C.c_int64), ("stride_head", C.c_int64), ("status", C.c_void_p),
        ("cache", CacheArgs),
    ]


class AttentionArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("R", C.c_int32), ("heads_q", C.c_int32),
        ("window", C.c_int32), ("n_sinks", C.c_int32), ("scale", C.c_float), ("reserved0", C.c_int32),
        ("q", C.c_void_p), ("q_stride_b", C.c_int64), ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64),
        ("k", C.c_void_p), ("v", C.c_void_p), ("kv_stride_b", C.c_int64), ("kv_stride_row", C.c_int64), ("kv_stride_head", C.c_int64),
        ("n_nodes", C.c_void_p), ("mask_bits", C.c_void_p), ("depth", C.c_void_p),
        ("out", C.c_void_p), ("out_stride_b", C.c_int64), ("out_stride_row", C.c_int64), ("out_stride_head", C.c_int64),
        ("lse", C.c_void_p), ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("cache", CacheArgs),
    ]


class WeightsArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("R", C.c_int32), ("L", C.c_int32), ("heads_q", C.c_int32),
        ("window", C.c_int32), ("n_sinks", C.c_int32), ("scale", C.c_float),
        ("q", C.c_void_p), ("q_stride_b", C.c_int64), ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64),
        ("lse", C.c_void_p), ("n_rows", C.c_void_p), ("path", C.c_void_p), ("path_len", C.c_void_p), ("base_length", C.c_void_p),
        ("weights", C.c_void_p), ("weights_out", C.c_void_p), ("weights_stride", C.c_int64), ("status", C.c_void_p),
        ("cache", CacheArgs),
    ]


class EvictArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("budget", C.c_int32), ("n_sinks", C.c_int32), ("n_recent", C.c_int32),
        ("new_max_pages", C.c_int32), ("weights", C.c_void_p), ("weights_stride", C.c_int64), ("new_block_table", C.c_void_p),
        ("new_length", C.c_void_p), ("kept", C.c_void_p), ("weights_out", C.c_void_p), ("weights_out_stride", C.c_int64),
        ("status", C.c_void_p), ("cache", CacheArgs),
    ]


class AdjustArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("batch", C.c_int32), ("R", C.c_int32),
        ("logits_dtype", C.c_int32), ("n_bias", C.c_int32), ("V", C.c_int64),
        ("logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_row", C.c_int64),
        ("out", C.c_void_p), ("out_stride_b", C.c_int64), ("out_stride_row", C.c_int64),
        ("n_nodes", C.c_void_p), ("token_ids", C.c_void_p), ("parent_idx", C.c_void_p),
        ("history", C.c_void_p), ("history_stride", C.c_int64), ("history_cols", C.c_int32), ("n_allowed", C.c_int32),
        ("history_len", C.c_void_p), ("prompt_len", C.c_void_p),
        ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p),
        ("bias_token", C.c_void_p), ("bias", C.c_void_p), ("allowed", C.c_void_p), ("allowed_row", C.c_void_p), ("status", C.c_void_p),
    ]


class DistillArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("batch", C.c_int32), ("L", C.c_int32), ("R", C.c_int32), ("K", C.c_int32),
        ("logits_dtype", C.c_int32), ("path_cols", C.c_int32), ("V", C.c_int64), ("temperature", C.c_double),
        ("logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_l", C.c_int64),
        ("teacher_token", C.c_void_p), ("teacher_logit", C.c_void_p), ("teacher_lse", C.c_void_p),
        ("path", C.c_void_p), ("path_len", C.c_void_p), ("n_rows", C.c_void_p), ("weight", C.c_void_p), ("grad_loss", C.c_void_p),
        ("loss", C.c_void_p), ("stats", C.c_void_p), ("grad", C.c_void_p), ("grad_stride_b", C.c_int64), ("grad_stride_l", C.c_int64),
        ("status", C.c_void_p),
    ]


_lib = None


def lib() -> C.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_01813_b200.build` "
                               "(there is no CPU fallback)")
        l = C.CDLL(LIB_PATH)
        l.cadd_version.restype = C.c_int
        l.cadd_status_string.restype = C.c_char_p
        l.cadd_status_string.argtypes = [C.c_int]
        l.cadd_build_workspace_bytes.argtypes = [C.POINTER(BuildArgs), C.POINTER(C.c_size_t)]
        l.cadd_verify_workspace_bytes.argtypes = [C.POINTER(VerifyArgs), C.POINTER(C.c_size_t)]
        l.cadd_build_tree.argtypes = [C.POINTER(BuildArgs), C.c_void_p]
        l.cadd_verify_tree.argtypes = [C.POINTER(VerifyArgs), C.c_void_p]
        l.cadd_head_workspace_bytes.argtypes = [C.POINTER(HeadArgs), C.POINTER(C.c_size_t)]
        l.cadd_verify_tree_fused_head.argtypes = [C.POINTER(HeadArgs), C.c_void_p]
        l.cadd_fit_cost_tables.argtypes = [C.POINTER(FitArgs), C.c_void_p]
        l.cadd_verify_tree_sampled.argtypes = [C.POINTER(SampleArgs), C.c_void_p]
        l.cadd_build_head_workspace_bytes.argtypes = [C.POINTER(BuildHeadArgs), C.POINTER(C.c_size_t)]
        l.cadd_build_tree_fused_head.argtypes = [C.POINTER(BuildHeadArgs), C.c_void_p]
        l.cadd_build_tree_static_scratch.argtypes = [C.POINTER(BuildArgs), C.c_void_p]
        l.cadd_build_launches.argtypes = [C.POINTER(BuildArgs)]
        l.cadd_verify_launches.argtypes = [C.POINTER(VerifyArgs)]
        l.cadd_cache_append.argtypes = [C.POINTER(AppendArgs), C.c_void_p]
        l.cadd_cache_read.argtypes = [C.POINTER(ReadArgs), C.c_void_p]
        l.cadd_tree_attention_workspace_bytes.argtypes = [C.POINTER(AttentionArgs), C.POINTER(C.c_size_t)]
        l.cadd_tree_attention.argtypes = [C.POINTER(AttentionArgs), C.c_void_p]
        l.cadd_cache_weights.argtypes = [C.POINTER(WeightsArgs), C.c_void_p]
        l.cadd_cache_evict.argtypes = [C.POINTER(EvictArgs), C.c_void_p]
        l.cadd_adjust_logits.argtypes = [C.POINTER(AdjustArgs), C.c_void_p]
        l.cadd_distill_loss.argtypes = [C.POINTER(DistillArgs), C.c_void_p]
        l.cadd_distill_grad.argtypes = [C.POINTER(DistillArgs), C.c_void_p]
        _lib = l
    return _lib


class CaddError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"cadd error {code}: {lib().cadd_status_string(code).decode()}")


def cadd_version() -> int:
    return int(lib().cadd_version())


def cadd_status_string(code: int) -> str:
    return lib().cadd_status_string(code).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_FP32
    raise TypeError(f"unsupported logits dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_of(stream: Optional[torch.cuda.Stream], dev) -> torch.cuda.Stream:
    """The stream a call is enqueued on: the given one, else the current stream OF THE TENSORS' DEVICE (which need
    not be the current device).  The same object serves the C call and record_stream."""
    return torch.cuda.current_stream(dev) if stream is None else stream


def _dev(t: Optional[torch.Tensor], device, dtype) -> Optional[torch.Tensor]:
    if t is None:
        return None
    return t.to(device=device, dtype=dtype).contiguous()


@dataclass
class Tree:
    """Outputs of cadd_build_tree (device tensors)."""
    n_nodes: torch.Tensor
    token_ids: torch.Tensor
    parent_idx: torch.Tensor
    depth: torch.Tensor
    position_ids: torch.Tensor
    node_logprob: torch.Tensor
    phi: torch.Tensor
    theta: torch.Tensor
    mask_bits: torch.Tensor
    mask_dense: Optional[torch.Tensor]
    topk_token: Optional[torch.Tensor]
    topk_logprob: Optional[torch.Tensor]
    status: torch.Tensor
    theta_curve: Optional[torch.Tensor] = None


@dataclass
class Verdict:
    """Outputs of cadd_verify_tree (device tensors)."""
    node_argmax: torch.Tensor
    accepted_len: torch.Tensor
    accepted_nodes: torch.Tensor
    next_bonus: torch.Tensor
    status: torch.Tensor


def _build_args(x, K, B_max, R, flags, cost_kind) -> BuildArgs:
    a = BuildArgs()
    a.struct_size = C.sizeof(BuildArgs)
    a.flags = flags
    a.batch, a.L, a.V = x.shape
    a.K, a.B_max, a.R = K, B_max, R
    a.logits_dtype = _dtype_code(x)
    a.cost_kind = cost_kind
    return a


def _marshal_build(a: BuildArgs, dev, batch, L, K, R, flags, theta_curve, out, l_eff, bonus_token, ctx_len, cost_coef,
                   cost_table, table_idx, t_draft, ctx_grid):
    """Fills the per-request inputs and the output pointers of a BuildArgs; returns (out, tensors to keep alive)."""
    keep = [_dev(l_eff, dev, torch.int32), _dev(bonus_token, dev, torch.int32), _dev(ctx_len, dev, torch.int32),
            _dev(cost_coef, dev, torch.float64), _dev(cost_table, dev, torch.float64),
            _dev(table_idx, dev, torch.int32), _dev(t_draft, dev, torch.float64), _dev(ctx_grid, dev, torch.int32)]
    a.l_eff, a.bonus_token, a.ctx_len = _ptr(keep[0]), _ptr(keep[1]), _ptr(keep[2])
    a.cost_coef, a.cost_table, a.table_idx, a.t_draft = _ptr(keep[3]), _ptr(keep[4]), _ptr(keep[5]), _ptr(keep[6])
    a.ctx_grid = _ptr(keep[7])
    a.n_tables = 0 if keep[4] is None else keep[4].shape[0]
    if out is None:
        W = (R + 31) // 32
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
        f64 = lambda *s: torch.empty(*s, dtype=torch.float64, device=dev)
        out = Tree(n_nodes=i32(batch), token_ids=i32(batch, R), parent_idx=i32(batch, R), depth=i32(batch, R),
                   position_ids=i32(batch, R), node_logprob=f64(batch, R), phi=f64(batch), theta=f64(batch),
                   mask_bits=i32(batch, R, W),
                   mask_dense=torch.empty(batch, R, R, dtype=torch.uint8, device=dev) if flags & FLAG_EMIT_DENSE_MASK else None,
                   topk_token=i32(batch, L, K) if flags & FLAG_EMIT_TOPK else None,
                   topk_logprob=f64(batch, L, K) if flags & FLAG_EMIT_TOPK else None,
                   status=i32(batch), theta_curve=f64(batch, R) if theta_curve else None)
    a.n_nodes, a.token_ids, a.parent_idx, a.depth = _ptr(out.n_nodes), _ptr(out.token_ids), _ptr(out.parent_idx), _ptr(out.depth)
    a.position_ids, a.node_logprob, a.phi, a.theta = _ptr(out.position_ids), _ptr(out.node_logprob), _ptr(out.phi), _ptr(out.theta)
    a.theta_curve = _ptr(out.theta_curve)
    a.mask_bits, a.mask_dense = _ptr(out.mask_bits), _ptr(out.mask_dense)
    a.topk_token, a.topk_logprob, a.status = _ptr(out.topk_token), _ptr(out.topk_logprob), _ptr(out.status)
    return out, keep


def cadd_build_workspace_bytes(batch: int, L: int, V: int, K: int, B_max: int, R: int, dtype: torch.dtype) -> int:
    a = BuildArgs()
    a.struct_size = C.sizeof(BuildArgs)
    a.batch, a.L, a.V, a.K, a.B_max, a.R = batch, L, V, K, B_max, R
    a.logits_dtype = DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_FP32
    out = C.c_size_t()
    rc = lib().cadd_build_workspace_bytes(C.byref(a), C.byref(out))
    if rc != OK:
        raise CaddError(rc)
    return int(out.value)


def cadd_round_launches(batch: int, L: int, V: int, K: int, B_max: int, R: int, dtype: torch.dtype, rows_mode: int = ROWS_LIVE) -> int:
    """Kernels one round (cadd_build_tree + cadd_verify_tree) enqueues for this shape: 4, or 2 for small problems."""
    a = BuildArgs()
    a.struct_size = C.sizeof(BuildArgs)
    a.batch, a.L, a.V, a.K, a.B_max, a.R = batch, L, V, K, B_max, R
    a.logits_dtype = DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_FP32
    v = VerifyArgs()
    v.struct_size = C.sizeof(VerifyArgs)
    v.batch, v.L, v.R, v.V = batch, L, R, V
    v.logits_dtype, v.rows_mode = a.logits_dtype, rows_mode
    nb, nv = lib().cadd_build_launches(C.byref(a)), lib().cadd_verify_launches(C.byref(v))
    if nb < 0 or nv < 0:
        raise CaddError(min(nb, nv))
    return int(nb + nv)


def cadd_build_tree(draft_logits: torch.Tensor, K: int, B_max: int, R: Optional[int] = None, *,
                    l_eff=None, bonus_token=None, ctx_len=None,
                    cost_kind: int = COST_QUADRATIC, cost_coef=None, cost_table=None, table_idx=None,
                    t_draft=None, ctx_grid=None, theta_curve: bool = False, flags: int = 0, out: Optional[Tree] = None,
                    workspace: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> Tree:
    """Build the draft trees of a batch (Eq. 1, Algorithm 1, Section 3.3) on the current CUDA stream.

    draft_logits: CUDA tensor [batch, L, V], bf16 or fp32, vocabulary axis contiguous.
    Small per-request inputs (l_eff, cost model, ...) are moved to the device if they are not there.
    `out` / `workspace` let a caller reuse buffers across rounds (no allocation inside the call then).
    """
    x = draft_logits
    if not x.is_cuda:
        raise ValueError("draft_logits must be a CUDA tensor (there is no CPU path)")
    if x.dim() != 3 or x.stride(2) != 1:
        raise ValueError("draft_logits must be [batch, L, V] with a contiguous vocabulary axis")
    dev = x.device
    batch, L, V = x.shape
    R = B_max + 1 if R is None else R
    a = _build_args(x, K, B_max, R, flags | (FLAG_REGULAR_PATH if FORCE_REGULAR_PATH else 0), cost_kind)
    a.draft_logits = x.data_ptr()
    a.stride_b, a.stride_l = x.stride(0), x.stride(1)
    out, keep = _marshal_build(a, dev, batch, L, K, R, flags, theta_curve, out, l_eff, bonus_token, ctx_len, cost_coef,
                               cost_table, table_idx, t_draft, ctx_grid)
    if workspace is None:
        nbytes = cadd_build_workspace_bytes(batch, L, V, K, B_max, R, x.dtype)
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_build_tree(C.byref(a), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    # the call is asynchronous: keep temporaries alive until the stream has consumed them
    for t in keep + [workspace]:
        if t is not None:
            t.record_stream(st)
    return out


def cadd_verify_tree(target_logits: torch.Tensor, L: int, n_nodes: torch.Tensor, token_ids: torch.Tensor,
                     parent_idx: torch.Tensor, rows_mode: int = ROWS_LIVE, *, out: Optional[Verdict] = None,
                     flags: int = 0, stream: Optional[torch.cuda.Stream] = None) -> Verdict:
    """Greedy tree verification (Sections 3.1, 3.3): per-node argmax of target_logits [batch, R, V]
    and the walk along the longest accepted path, on the current CUDA stream."""
    y = target_logits
    if not y.is_cuda:
        raise ValueError("target_logits must be a CUDA tensor (there is no CPU path)")
    if y.dim() != 3 or y.stride(2) != 1:
        raise ValueError("target_logits must be [batch, R, V] with a contiguous vocabulary axis")
    dev = y.device
    batch, R, V = y.shape
    for t in (n_nodes, token_ids, parent_idx):
        if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
            raise ValueError("tree arrays must be contiguous int32 CUDA tensors")
    a = VerifyArgs()
    a.struct_size = C.sizeof(VerifyArgs)
    a.flags = flags | (VERIFY_REGULAR_PATH if FORCE_REGULAR_PATH else 0)
    a.batch, a.L, a.R, a.V = batch, L, R, V
    a.logits_dtype = _dtype_code(y)
    a.rows_mode = rows_mode
    a.target_logits = y.data_ptr()
    a.stride_b, a.stride_row = y.stride(0), y.stride(1)
    a.n_nodes, a.token_ids, a.parent_idx = n_nodes.data_ptr(), token_ids.data_ptr(), parent_idx.data_ptr()
    if out is None:
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
        out = Verdict(node_argmax=i32(batch, R), accepted_len=i32(batch), accepted_nodes=i32(batch, L),
                      next_bonus=i32(batch), status=i32(batch))
    a.node_argmax, a.accepted_len, a.accepted_nodes = _ptr(out.node_argmax), _ptr(out.accepted_len), _ptr(out.accepted_nodes)
    a.next_bonus, a.status = _ptr(out.next_bonus), _ptr(out.status)
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_verify_tree(C.byref(a), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    return out


def cadd_head_workspace_bytes(batch: int, R: int, hidden: int, V: int, L: int = 1, rows_mode: int = ROWS_LIVE) -> int:
    """Scratch bytes of cadd_verify_tree_fused_head; LIVE mode (the default here) needs room for a packed copy of the
    live hidden states and is therefore the larger of the two."""
    a = HeadArgs()
    a.struct_size = C.sizeof(HeadArgs)
    a.batch, a.L, a.R, a.hidden, a.V = batch, L, R, hidden, V
    a.rows_mode = rows_mode
    n = C.c_size_t(0)
    rc = lib().cadd_head_workspace_bytes(C.byref(a), C.byref(n))
    if rc != OK:
        raise CaddError(rc)
    return int(n.value)


def cadd_verify_tree_fused_head(hidden_states: torch.Tensor, weight: torch.Tensor, L: int, n_nodes: torch.Tensor,
                                token_ids: torch.Tensor, parent_idx: torch.Tensor, rows_mode: int = ROWS_LIVE, *,
                                out: Optional[Verdict] = None, workspace: Optional[torch.Tensor] = None,
                                stream: Optional[torch.cuda.Stream] = None) -> Verdict:
    """Greedy tree verification from the target's last hidden states [batch, R, hidden] and its output-projection
    weight [V, hidden] (both bf16): the logits h . W^T are formed on the tensor cores and reduced to the per-node
    argmax without being written to memory (Section 3.1), then the accepted path is walked (Section 3.3)."""
    h, w = hidden_states, weight
    if not (h.is_cuda and w.is_cuda):
        raise ValueError("hidden_states and weight must be CUDA tensors (there is no CPU path)")
    if h.dtype != torch.bfloat16 or w.dtype != torch.bfloat16:
        raise ValueError("hidden_states and weight must be bfloat16")
    if h.dim() != 3 or h.stride(2) != 1 or h.stride(0) != h.shape[1] * h.stride(1):
        raise ValueError("hidden_states must be [batch, R, hidden] with contiguous rows of equal stride")
    if w.dim() != 2 or w.stride(1) != 1 or w.shape[1] != h.shape[2]:
        raise ValueError("weight must be [V, hidden] with a contiguous hidden axis")
    dev = h.device
    batch, R, hidden = h.shape
    V = w.shape[0]
    for t in (n_nodes, token_ids, parent_idx):
        if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
            raise ValueError("tree arrays must be contiguous int32 CUDA tensors")
    a = HeadArgs()
    a.struct_size = C.sizeof(HeadArgs)
    a.batch, a.L, a.R, a.hidden, a.V = batch, L, R, hidden, V
    a.rows_mode = rows_mode
    a.hidden_states, a.stride_row = h.data_ptr(), h.stride(1)
    a.weight, a.stride_w = w.data_ptr(), w.stride(0)
    a.n_nodes, a.token_ids, a.parent_idx = n_nodes.data_ptr(), token_ids.data_ptr(), parent_idx.data_ptr()
    if out is None:
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
        out = Verdict(node_argmax=i32(batch, R), accepted_len=i32(batch), accepted_nodes=i32(batch, L),
                      next_bonus=i32(batch), status=i32(batch))
    a.node_argmax, a.accepted_len, a.accepted_nodes = _ptr(out.node_argmax), _ptr(out.accepted_len), _ptr(out.accepted_nodes)
    a.next_bonus, a.status = _ptr(out.next_bonus), _ptr(out.status)
    if workspace is None:
        workspace = torch.empty(cadd_head_workspace_bytes(batch, R, hidden, V, L, rows_mode), dtype=torch.uint8, device=dev)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_verify_tree_fused_head(C.byref(a), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    workspace.record_stream(st)
    return out


def _build_head_args(batch, L, V, hidden, K, B_max, R, flags, cost_kind) -> BuildHeadArgs:
    h = BuildHeadArgs()
    h.struct_size = C.sizeof(BuildHeadArgs)
    h.hidden = hidden
    a = h.build
    a.struct_size = C.sizeof(BuildArgs)
    a.flags = flags
    a.batch, a.L, a.V = batch, L, V
    a.K, a.B_max, a.R = K, B_max, R
    a.logits_dtype = DTYPE_FP32
    a.cost_kind = cost_kind
    return h


def cadd_build_head_workspace_bytes(batch: int, L: int, V: int, hidden: int, K: int, B_max: int, R: int) -> int:
    h = _build_head_args(batch, L, V, hidden, K, B_max, R, 0, COST_QUADRATIC)
    n = C.c_size_t(0)
    rc = lib().cadd_build_head_workspace_bytes(C.byref(h), C.byref(n))
    if rc != OK:
        raise CaddError(rc)
    return int(n.value)


def cadd_build_tree_fused_head(hidden_states: torch.Tensor, weight: torch.Tensor, K: int, B_max: int, R: Optional[int] = None, *,
                               l_eff=None, bonus_token=None, ctx_len=None,
                               cost_kind: int = COST_QUADRATIC, cost_coef=None, cost_table=None, table_idx=None,
                               t_draft=None, ctx_grid=None, theta_curve: bool = False, flags: int = 0,
                               out: Optional[Tree] = None, workspace: Optional[torch.Tensor] = None,
                               stream: Optional[torch.cuda.Stream] = None) -> Tree:
    """cadd_build_tree from the drafter's last hidden states [batch, L, hidden] and its output-projection weight
    [V, hidden] (both bf16): the draft logits are formed on the tensor cores and consumed by the softmax statistics
    and the top-K selection without being written to memory (Eq. 1, Algorithm 1)."""
    hs, w = hidden_states, weight
    if not (hs.is_cuda and w.is_cuda):
        raise ValueError("hidden_states and weight must be CUDA tensors (there is no CPU path)")
    if hs.dtype != torch.bfloat16 or w.dtype != torch.bfloat16:
        raise ValueError("hidden_states and weight must be bfloat16")
    if hs.dim() != 3 or hs.stride(2) != 1 or hs.stride(0) != hs.shape[1] * hs.stride(1):
        raise ValueError("hidden_states must be [batch, L, hidden] with contiguous rows of equal stride")
    if w.dim() != 2 or w.stride(1) != 1 or w.shape[1] != hs.shape[2]:
        raise ValueError("weight must be [V, hidden] with a contiguous hidden axis")
    dev = hs.device
    batch, L, hidden = hs.shape
    V = w.shape[0]
    R = B_max + 1 if R is None else R
    h = _build_head_args(batch, L, V, hidden, K, B_max, R, flags, cost_kind)
    h.hidden_states, h.stride_row = hs.data_ptr(), hs.stride(1)
    h.weight, h.stride_w = w.data_ptr(), w.stride(0)
    out, keep = _marshal_build(h.build, dev, batch, L, K, R, flags, theta_curve, out, l_eff, bonus_token, ctx_len, cost_coef,
                               cost_table, table_idx, t_draft, ctx_grid)
    if workspace is None:
        workspace = torch.empty(cadd_build_head_workspace_bytes(batch, L, V, hidden, K, B_max, R), dtype=torch.uint8, device=dev)
    h.build.workspace, h.build.workspace_bytes = workspace.data_ptr(), workspace.numel()
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_build_tree_fused_head(C.byref(h), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    for t in keep + [workspace]:
        if t is not None:
            t.record_stream(st)
    return out


def cadd_verify_tree_sampled(target_logits: torch.Tensor, uniforms: torch.Tensor, L: int, n_nodes: torch.Tensor,
                             token_ids: torch.Tensor, parent_idx: torch.Tensor, rows_mode: int = ROWS_LIVE, *,
                             temperature: float = 1.0, out: Optional[Verdict] = None, flags: int = 0,
                             stream: Optional[torch.cuda.Stream] = None) -> Verdict:
    """Tree verification under sampling: one token is drawn per node from softmax(target_logits / temperature) by the
    inverse CDF at uniforms[b, j]; the walk follows the child that carries the drawn token.  Verdict.node_argmax holds
    the drawn tokens."""
    y = target_logits
    if not (y.is_cuda and uniforms.is_cuda):
        raise ValueError("target_logits and uniforms must be CUDA tensors (there is no CPU path)")
    if y.dim() != 3 or y.stride(2) != 1:
        raise ValueError("target_logits must be [batch, R, V] with a contiguous vocabulary axis")
    dev = y.device
    batch, R, V = y.shape
    if uniforms.dtype != torch.float64 or tuple(uniforms.shape) != (batch, R) or not uniforms.is_contiguous():
        raise ValueError("uniforms must be a contiguous float64 tensor [batch, R]")
    for t in (n_nodes, token_ids, parent_idx):
        if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
            raise ValueError("tree arrays must be contiguous int32 CUDA tensors")
    a = SampleArgs()
    a.struct_size = C.sizeof(SampleArgs)
    a.flags = flags
    a.batch, a.L, a.R, a.V = batch, L, R, V
    a.logits_dtype = _dtype_code(y)
    a.rows_mode = rows_mode
    a.temperature = float(temperature)
    a.target_logits = y.data_ptr()
    a.stride_b, a.stride_row = y.stride(0), y.stride(1)
    a.uniforms = uniforms.data_ptr()
    a.n_nodes, a.token_ids, a.parent_idx = n_nodes.data_ptr(), token_ids.data_ptr(), parent_idx.data_ptr()
    if out is None:
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
        out = Verdict(node_argmax=i32(batch, R), accepted_len=i32(batch), accepted_nodes=i32(batch, L),
                      next_bonus=i32(batch), status=i32(batch))
    a.node_token, a.accepted_len, a.accepted_nodes = _ptr(out.node_argmax), _ptr(out.accepted_len), _ptr(out.accepted_nodes)
    a.next_bonus, a.status = _ptr(out.next_bonus), _ptr(out.status)
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_verify_tree_sampled(C.byref(a), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    return out


def cadd_fit_cost_tables(y: torch.Tensor, *, stream: Optional[torch.cuda.Stream] = None):
    """Offline cost fitting (Eq. 12): the convex, non-decreasing least-squares fit of every row of y [n_tables, N]
    (fp64, CUDA).  Returns (fit [n_tables, N] fp64, n_breaks [n_tables] int32, status [n_tables] int32)."""
    if not y.is_cuda:
        raise ValueError("y must be a CUDA tensor (there is no CPU path)")
    if y.dtype != torch.float64 or y.dim() != 2 or not y.is_contiguous():
        raise ValueError("y must be a contiguous float64 tensor [n_tables, N]")
    a = FitArgs()
    a.struct_size = C.sizeof(FitArgs)
    a.n_tables, a.N = y.shape
    fit = torch.empty_like(y)
    nb = torch.empty(y.shape[0], dtype=torch.int32, device=y.device)
    st = torch.empty(y.shape[0], dtype=torch.int32, device=y.device)
    a.y, a.fit, a.n_breaks, a.status = y.data_ptr(), fit.data_ptr(), nb.data_ptr(), st.data_ptr()
    with torch.cuda.device(y.device):
        rc = lib().cadd_fit_cost_tables(C.byref(a), _stream_of(stream, y.device).cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    return fit, nb, st


def cadd_build_tree_static_scratch(draft_logits: torch.Tensor, K: int, B_max: int, R: Optional[int] = None, *,
                                   l_eff=None, bonus_token=None, ctx_len=None,
                                   cost_kind: int = COST_QUADRATIC, cost_coef=None, cost_table=None,
                                   table_idx=None, t_draft=None, ctx_grid=None, flags: int = 0, out: Tree = None,
                                   stream: Optional[torch.cuda.Stream] = None) -> Tree:
    """cadd_build_tree without a workspace argument: the library uses its built-in scratch array.

    For callers that may not allocate device memory (for instance code running inside a host
    application that owns the memory pool): pass every input on the device already and a preallocated
    `out`; the call then allocates nothing.  (If `out` is omitted it is allocated here with torch, which
    is a convenience for tests.)  Shapes whose scratch need exceeds STATIC_SCRATCH_BYTES raise CaddError
    with code ERR_STATIC_SCRATCH.  Calls on one device share the scratch: do not let two of them overlap
    on the GPU.  The first call per device performs a one-time address look-up and belongs outside any
    stream capture."""
    x = draft_logits
    if not x.is_cuda:
        raise ValueError("draft_logits must be a CUDA tensor (there is no CPU path)")
    if x.dim() != 3 or x.stride(2) != 1:
        raise ValueError("draft_logits must be [batch, L, V] with a contiguous vocabulary axis")
    dev = x.device
    batch, L, V = x.shape
    R = B_max + 1 if R is None else R
    a = _build_args(x, K, B_max, R, flags, cost_kind)
    a.draft_logits = x.data_ptr()
    a.stride_b, a.stride_l = x.stride(0), x.stride(1)
    keep = [_dev(l_eff, dev, torch.int32), _dev(bonus_token, dev, torch.int32), _dev(ctx_len, dev, torch.int32),
            _dev(cost_coef, dev, torch.float64), _dev(cost_table, dev, torch.float64),
            _dev(table_idx, dev, torch.int32), _dev(t_draft, dev, torch.float64), _dev(ctx_grid, dev, torch.int32)]
    a.l_eff, a.bonus_token, a.ctx_len = _ptr(keep[0]), _ptr(keep[1]), _ptr(keep[2])
    a.cost_coef, a.cost_table, a.table_idx, a.t_draft = _ptr(keep[3]), _ptr(keep[4]), _ptr(keep[5]), _ptr(keep[6])
    a.ctx_grid = _ptr(keep[7])
    a.n_tables = 0 if keep[4] is None else keep[4].shape[0]
    if out is None:
        W = (R + 31) // 32
        i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
        f64 = lambda *s: torch.empty(*s, dtype=torch.float64, device=dev)
        out = Tree(n_nodes=i32(batch), token_ids=i32(batch, R), parent_idx=i32(batch, R), depth=i32(batch, R),
                   position_ids=i32(batch, R), node_logprob=f64(batch, R), phi=f64(batch), theta=f64(batch),
                   mask_bits=i32(batch, R, W),
                   mask_dense=torch.empty(batch, R, R, dtype=torch.uint8, device=dev) if flags & FLAG_EMIT_DENSE_MASK else None,
                   topk_token=i32(batch, L, K) if flags & FLAG_EMIT_TOPK else None,
                   topk_logprob=f64(batch, L, K) if flags & FLAG_EMIT_TOPK else None,
                   status=i32(batch))
    a.n_nodes, a.token_ids, a.parent_idx, a.depth = _ptr(out.n_nodes), _ptr(out.token_ids), _ptr(out.parent_idx), _ptr(out.depth)
    a.position_ids, a.node_logprob, a.phi, a.theta = _ptr(out.position_ids), _ptr(out.node_logprob), _ptr(out.phi), _ptr(out.theta)
    a.mask_bits, a.mask_dense = _ptr(out.mask_bits), _ptr(out.mask_dense)
    a.topk_token, a.topk_logprob, a.status = _ptr(out.topk_token), _ptr(out.topk_logprob), _ptr(out.status)
    st = _stream_of(stream, dev)
    with torch.cuda.device(dev):
        rc = lib().cadd_build_tree_static_scratch(C.byref(a), st.cuda_stream)
    if rc != OK:
        raise CaddError(rc)
    for t in keep:
        if t is not None:
            t.record_stream(st)
    return out


# ---- the paged key/value cache and the tree attention over it ----

def _need(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _need_i32(t: Optional[torch.Tensor], shape, dev, name: str) -> Optional[int]:
    """Pointer of an int32 input of the given shape on the call's device (None passes)."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.device != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on {dev}")
    return t.data_ptr()


def _need_rows(t: torch.Tensor, shape, dev, name: str):
    """Pointer and (batch, row, head) strides of a bf16 operand [batch, rows, heads, head_dim]."""
    if t.dtype != torch.bfloat16 or t.device != dev or t.shape != shape:
        raise ValueError(f"{name} must be a bfloat16 tensor {list(shape)} on {dev}")
    sb, sr, sh, se = t.stride()
    if se != 1:
        raise ValueError(f"{name} must have a contiguous last axis")
    # an axis of length one may carry any stride; it is never stepped along
    return t.data_ptr(), sb if shape[0] > 1 else 0, sr if shape[1] > 1 else 0, sh if shape[2] > 1 else 0


def _enqueue(fn, args, dev, stream) -> None:
    """The call, on the given stream or the current one of the tensors' device, with that device current."""
    raw = torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == dev.index:
        rc = fn(C.byref(args), raw)
    else:
        with torch.cuda.device(dev):
            rc = fn(C.byref(args), raw)
    if rc != OK:
        raise CaddError(rc)


class KvCache:
    """A paged key/value cache (cadd_cache): the pools and a batch's view of them.

    k, v: CUDA tensors [n_pages, heads, page_size, head_dim] in bf16, or in 4 bits as uint8 codes [..., head_dim / 2] with
    k_scale, v_scale uint8 (e4m3) [..., head_dim / 16].  A token's row must be contiguous; the other axes may be strided
    alike in all pools (permuted views fit).  block_table [batch, max_pages] and length [batch] are int32 on the same device.
    In the 4-bit form k_exp and v_exp are the powers of two that rows are multiplied by before they are stored.

    The object describes these tensors and is fixed; their contents may change.  For other tensors make another one."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, block_table: torch.Tensor, length: torch.Tensor,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, k_exp: int = 0, v_exp: int = 0):
        dev, dtype, shape, strides = k.device, k.dtype, k.shape, k.stride()
        if dev.type != "cuda":
            raise ValueError("the cache must be on a CUDA device (there is no CPU path)")
        fp4 = dtype == torch.uint8
        if not fp4 and dtype != torch.bfloat16:
            raise TypeError(f"unsupported cache dtype {dtype}")
        if len(shape) != 4 or v.shape != shape or v.dtype != dtype or v.device != dev or v.stride() != strides:
            raise ValueError("k and v must be alike, [n_pages, heads, page_size, ...]")
        pages, heads, page_size, n = shape
        rows = self._rows(shape, strides)
        if fp4:
            if k_scale is None or v_scale is None:
                raise ValueError("a 4-bit cache needs k_scale and v_scale")
            want = (pages, heads, page_size, n // 8)
            for t in (k_scale, v_scale):
                if t.dtype != torch.uint8 or t.device != dev or t.shape != want or n % 8:
                    raise ValueError("k_scale and v_scale must be uint8 with one scale for 8 bytes of codes")
                if self._rows(want, t.stride()) != rows:
                    raise ValueError("all pools must be laid out alike")
        elif k_scale is not None or v_scale is not None:
            raise ValueError("a bf16 cache has no scales")
        if block_table.dim() != 2 or block_table.dtype != torch.int32 or block_table.device != dev or not block_table.is_contiguous():
            raise ValueError("block_table must be a contiguous int32 tensor [batch, max_pages] on the cache's device")
        batch, max_pages = block_table.shape
        args = CacheArgs(C.sizeof(CacheArgs), CACHE_FP4 if fp4 else CACHE_BF16, batch, heads, 2 * n if fp4 else n, page_size, max_pages, k_exp, v_exp, 0,
                         pages, *rows, k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if fp4 else None, v_scale.data_ptr() if fp4 else None,
                         block_table.data_ptr(), _need_i32(length, (batch,), dev, "length"))
        self.__dict__.update(k=k, v=v, block_table=block_table, length=length, k_scale=k_scale, v_scale=v_scale, k_exp=k_exp, v_exp=v_exp,
                             args=args, device=dev, batch=batch, heads=heads, head_dim=args.head_dim, capacity=max_pages * page_size)

    @staticmethod
    def _rows(shape, strides):
        """Strides of the first three axes in rows."""
        n = shape[3]
        if strides[3] != 1:
            raise ValueError("a token's row must be contiguous")
        out = []
        for i in range(3):
            if shape[i] <= 1:
                out.append(1)                     # never stepped along
            elif n and strides[i] % n == 0:
                out.append(strides[i] // n)
            else:
                raise ValueError("the pools' strides must be whole rows")
        return out

    def __setattr__(self, name, value):
        raise AttributeError("a KvCache is fixed: make another one")


@dataclass
class Attention:
    """Outputs of cadd_tree_attention (device tensors): out bf16 [batch, R, heads_q, head_dim]; lse fp32 [batch, R, heads_q]
    and status int32 [batch], which may be None (not written then)."""
    out: torch.Tensor
    lse: Optional[torch.Tensor] = None
    status: Optional[torch.Tensor] = None


@dataclass
class Evicted:
    """Outputs of cadd_cache_evict (device tensors); weights and status may be None (not written then)."""
    new_length: torch.Tensor
    kept: torch.Tensor
    weights: Optional[torch.Tensor] = None
    status: Optional[torch.Tensor] = None


def _some_column(path: Optional[torch.Tensor], B: int, dev, stream) -> Optional[torch.Tensor]:
    """A path without columns has a NULL pointer, which would mean no path: one column of no row instead, so that the root is left."""
    if path is None or path.dim() != 2 or path.shape[1] != 0 or path.shape[0] != B:
        return path
    _need_like(path, torch.int32, (B, 0), dev.index, "path")
    with torch.cuda.stream(_stream_of(stream, dev)):
        return torch.full((B, 1), -1, dtype=torch.int32, device=dev)


def _row_list(cache: KvCache, n_rows, path, path_len):
    """L and the pointers of n_rows, path and path_len, of the calls that take a path or leading rows.  (The caller keeps its
    own names bound to the tensors until the call is enqueued: a temporary would otherwise be freed, and its memory given out.)"""
    B, dev = cache.batch, cache.device
    if path is None:
        if path_len is not None:
            raise ValueError("path_len comes with path")
        return 0, _need_i32(n_rows, (B,), dev, "n_rows"), None, None
    if path_len is None or n_rows is not None:
        raise ValueError("path comes with path_len and without n_rows")
    if path.dim() != 2:
        raise ValueError("path must be [batch, L]")
    L = path.shape[1]
    return L, None, _need_i32(path, (B, L), dev, "path"), _need_i32(path_len, (B,), dev, "path_len")


def cadd_cache_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, *, n_rows=None, path=None, path_len=None,
                      new_length: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Write rows of k and v (bf16 [batch, R, heads, head_dim]) behind each request's cached tokens: rows 0..n_rows[b]-1
    (all R without n_rows), or with path / path_len (a verification's accepted_nodes / accepted_len) the root and the accepted
    path (without a column: the root alone).  Returns new_length (which may be given, cache.length itself included: the cache then goes on from there)."""
    B, dev = cache.batch, cache.device
    _need(k.dim() == 4 and k.shape[0] == B, "k must be [batch, R, heads, head_dim]")
    R = k.shape[1]
    shape = (B, R, cache.heads, cache.head_dim)
    kp, *strides = _need_rows(k, shape, dev, "k")
    vp, *vs = _need_rows(v, shape, dev, "v")
    _need(strides == vs, "k and v must have the same strides")
    path = _some_column(path, B, dev, stream)
    L, *rows = _row_list(cache, n_rows, path, path_len)
    if new_length is None:
        with torch.cuda.stream(_stream_of(stream, dev)):
            new_length = torch.empty(B, dtype=torch.int32, device=dev)
    a = AppendArgs(C.sizeof(AppendArgs), 0, R, L, kp, vp, *strides, *rows, _need_i32(new_length, (B,), dev, "new_length"),
                   _need_i32(status, (B,), dev, "status"), cache.args)
    _enqueue(lib().cadd_cache_append, a, dev, stream)
    return new_length


def cadd_cache_read(cache: KvCache, n_max: int, *, start=None, count=None, out=None, status: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None):
    """Cached rows as bf16: out = (k, v), each [batch, n_max, heads, head_dim], row i being place start[b] + i (start 0 and
    count up to the length unless given).  Rows that are not read keep what `out` held (zeros if it is made here)."""
    B, dev = cache.batch, cache.device
    shape = (B, n_max, cache.heads, cache.head_dim)
    if out is None:
        with torch.cuda.stream(_stream_of(stream, dev)):
            out = tuple(torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(2))
    kp, *strides = _need_rows(out[0], shape, dev, "out k")
    vp, *vs = _need_rows(out[1], shape, dev, "out v")
    _need(strides == vs, "both outputs must have the same strides")
    a = ReadArgs(C.sizeof(ReadArgs), 0, n_max, 0, _need_i32(start, (B,), dev, "start"), _need_i32(count, (B,), dev, "count"), kp, vp, *strides,
                 _need_i32(status, (B,), dev, "status"), cache.args)
    _enqueue(lib().cadd_cache_read, a, dev, stream)
    return out


def cadd_tree_attention_workspace_bytes(batch: int, R: int, heads_q: int, cache: KvCache) -> int:
    a = AttentionArgs()
    a.struct_size = C.sizeof(AttentionArgs)
    a.R, a.heads_q = R, heads_q
    a.cache = cache.args
    a.cache.batch = batch
    n = C.c_size_t(0)
    rc = lib().cadd_tree_attention_workspace_bytes(C.byref(a), C.byref(n))
    if rc != OK:
        raise CaddError(rc)
    return int(n.value)


def cadd_tree_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cache: KvCache, *, mask_bits=None, n_nodes=None,
                        depth=None, scale: Optional[float] = None, window: int = 0, n_sinks: int = 0, flags: int = 0,
                        out: Optional[Attention] = None, workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> Attention:
    """Attention of a tree's rows (q bf16 [batch, R, heads_q, head_dim]) over the cache and over the tree's own rows (k, v bf16
    [batch, R, heads, head_dim]) through mask_bits, n_nodes and depth as cadd_build_tree returns them (Section 3.3).
    Without mask_bits row r sees rows 0..r (a prompt chunk; one decoded token is R = 1).  window > 0: the last `window`
    places and the first n_sinks only.  scale is 1/sqrt(head_dim) unless given.  Rows above n_nodes keep what `out` held
    (zeros if it is made here, lse too)."""
    B, dev, D = cache.batch, cache.device, cache.head_dim
    _need(q.is_cuda, "q must be a CUDA tensor (there is no CPU path)")
    _need(q.dim() == 4, "q must be [batch, R, heads_q, head_dim]")
    R, hq = q.shape[1], q.shape[2]
    qshape, kvshape = (B, R, hq, D), (B, R, cache.heads, D)
    qargs = _need_rows(q, qshape, dev, "q")
    kp, *strides = _need_rows(k, kvshape, dev, "k")
    vp, *vs = _need_rows(v, kvshape, dev, "v")
    _need(strides == vs, "k and v must have the same strides")
    if out is None:
        with torch.cuda.stream(_stream_of(stream, dev)):
            out = Attention(out=torch.zeros(qshape, dtype=torch.bfloat16, device=dev), lse=torch.zeros(qshape[:3], device=dev),
                            status=torch.zeros(B, dtype=torch.int32, device=dev))
    lse = out.lse
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.device == dev and lse.shape == qshape[:3] and lse.is_contiguous(),
              "lse must be a contiguous float32 tensor [batch, R, heads_q]")
        lse = lse.data_ptr()
    if workspace is None:                         # (allocated on the call's stream, so it may be given back as soon as the call is enqueued)
        with torch.cuda.stream(_stream_of(stream, dev)):
            workspace = torch.empty(cadd_tree_attention_workspace_bytes(B, R, hq, cache), dtype=torch.uint8, device=dev)
    _need(workspace.device == dev and workspace.is_contiguous(), "workspace must be on the call's device")
    a = AttentionArgs(C.sizeof(AttentionArgs), flags, R, hq, window, n_sinks, D ** -0.5 if scale is None else scale, 0, *qargs, kp, vp, *strides,
                      _need_i32(n_nodes, (B,), dev, "n_nodes"), _need_i32(mask_bits, (B, R, (R + 31) // 32), dev, "mask_bits"),
                      _need_i32(depth, (B, R), dev, "depth"), *_need_rows(out.out, qshape, dev, "out"), lse, _need_i32(out.status, (B,), dev, "status"),
                      workspace.data_ptr(), workspace.numel() * workspace.element_size(), cache.args)
    _enqueue(lib().cadd_tree_attention, a, dev, stream)
    return out


def _need_weights(w: torch.Tensor, B: int, H: int, n: int, dev, name: str):
    if w.dim() != 3 or w.dtype != torch.float32 or w.device != dev:
        raise ValueError(f"{name} must be a float32 tensor [batch, heads, >= {n}] on {dev}")
    (wb, wh, wn), (sb, sh, sn) = w.shape, w.stride()
    if wb != B or wh != H or wn < n or sn != 1 or (B > 1 and H > 1 and sb != H * sh):
        raise ValueError(f"{name} must be [batch, heads, >= {n}] with rows of equal stride")
    return w.data_ptr(), sh if H > 1 else (sb if B > 1 else wn)


def cadd_cache_weights(q: torch.Tensor, lse: torch.Tensor, cache: KvCache, base_length: torch.Tensor, weights: torch.Tensor, *,
                       n_rows=None, path=None, path_len=None, scale: Optional[float] = None, window: int = 0, n_sinks: int = 0,
                       out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Add the attention weight that the accepted rows (rows and lse as in cadd_tree_attention, path / path_len / n_rows as in
    cadd_cache_append, the rows being in the cache by now) spent on every cached place to weights fp32 [batch, heads, capacity].
    base_length is the length before the append.  Works in place unless `out` is given, which becomes the whole new array."""
    B, dev, D = cache.batch, cache.device, cache.head_dim
    _need(q.dim() == 4, "q must be [batch, R, heads_q, head_dim]")
    R, hq = q.shape[1], q.shape[2]
    path = _some_column(path, B, dev, stream)
    L, *rows = _row_list(cache, n_rows, path, path_len)
    _need(lse.dtype == torch.float32 and lse.device == dev and lse.shape == (B, R, hq) and lse.is_contiguous(),
          "lse must be a contiguous float32 tensor [batch, R, heads_q]")
    wp, stride = _need_weights(weights, B, cache.heads, cache.capacity, dev, "weights")
    if out is None:
        out, op = weights, wp
    else:
        op, so = _need_weights(out, B, cache.heads, cache.capacity, dev, "out")
        _need(so == stride, "weights and out must have the same strides")
    a = WeightsArgs(C.sizeof(WeightsArgs), 0, R, L, hq, window, n_sinks, D ** -0.5 if scale is None else scale, *_need_rows(q, (B, R, hq, D), dev, "q"),
                    lse.data_ptr(), *rows, _need_i32(base_length, (B,), dev, "base_length"), wp, op, stride,
                    _need_i32(status, (B,), dev, "status"), cache.args)
    _enqueue(lib().cadd_cache_weights, a, dev, stream)
    return out


def cadd_cache_evict(cache: KvCache, weights: torch.Tensor, new_block_table: torch.Tensor, budget: int, *, n_sinks: int = 0,
                     n_recent: int = 0, out: Optional[Evicted] = None, stream: Optional[torch.cuda.Stream] = None) -> Evicted:
    """Keep `budget` places of every (request, head): the first n_sinks, the last n_recent and the heaviest between them by
    weights (as cadd_cache_weights keeps them).  Their rows go, in order, to the pages of new_block_table [batch, pages] in the same
    pools; the old pages are not changed.  The cache goes on as KvCache(..., block_table=new_block_table,
    length=result.new_length) with result.weights."""
    B, H, dev = cache.batch, cache.heads, cache.device
    _need(new_block_table.dim() == 2, "new_block_table must be [batch, pages]")
    pages = new_block_table.shape[1]
    wp, stride = _need_weights(weights, B, H, cache.capacity, dev, "weights")
    if out is None:
        _need(budget >= 1, "budget must be at least 1")
        with torch.cuda.stream(_stream_of(stream, dev)):
            out = Evicted(new_length=torch.empty(B, dtype=torch.int32, device=dev), kept=torch.empty(B, H, budget, dtype=torch.int32, device=dev),
                          weights=torch.zeros(B, H, pages * cache.args.page_size, device=dev), status=torch.empty(B, dtype=torch.int32, device=dev))
    op, so = (None, 0) if out.weights is None else _need_weights(out.weights, B, H, min(budget, pages * cache.args.page_size), dev, "out.weights")
    a = EvictArgs(C.sizeof(EvictArgs), 0, budget, n_sinks, n_recent, pages, wp, stride, _need_i32(new_block_table, (B, pages), dev, "new_block_table"),
                  _need_i32(out.new_length, (B,), dev, "new_length"), _need_i32(out.kept, (B, H, budget), dev, "kept"), op, so,
                  _need_i32(out.status, (B,), dev, "status"), cache.args)
    _enqueue(lib().cadd_cache_evict, a, dev, stream)
    return out


# ---- the logits of a round: penalties, biases, masks; distillation ----

def _need_logits(t: torch.Tensor, shape, dtype, index: int, name: str):
    """Pointer and (batch, row) strides of logits [batch, rows, V]."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} on cuda:{index}")
    sb, sr, sv = t.stride()
    if sv != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have a contiguous vocabulary axis")
    # an axis of length one may carry any stride; it is never stepped along
    return t.data_ptr(), sb if shape[0] > 1 else 0, sr if shape[1] > 1 else 0


def _need_like(t: Optional[torch.Tensor], dtype, shape, index: int, name: str) -> Optional[int]:
    """Pointer of a contiguous input or output of the given dtype and shape on the call's device (None passes)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on cuda:{index}")
    return t.data_ptr()


def _logits_of(t: torch.Tensor, name: str):
    """Device, its index, and dtype code of the logits of a call."""
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be a CUDA tensor (there is no CPU path)")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [batch, rows, V]")
    return t.device, index, _dtype_code(t)


def cadd_adjust_logits(logits: torch.Tensor, *, n_nodes=None, token_ids=None, parent_idx=None, history=None, history_len=None,
                       prompt_len=None, repetition=None, presence=None, frequency=None, bias_token=None, bias=None, allowed=None,
                       allowed_row=None, out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, flags: int = 0,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Penalties, biases and grammar masks on logits [batch, R, V] (bf16 or fp32), before cadd_verify_tree,
    cadd_verify_tree_sampled or cadd_build_tree: each row by its own context, the history and, with token_ids / parent_idx
    (and n_nodes) of cadd_build_tree, the row's path.  Works in place unless `out` is given; rows above n_nodes keep what `out` held.

    history int32 [batch, n] (rows may be strided) with history_len and prompt_len int32 [batch]: what stands before row 0's token
    (which counts itself where the tree was built with bonus_token); the first prompt_len tokens count for repetition alone.  repetition, presence, frequency fp32 [batch].  bias_token int32,
    bias fp32 [batch, n_bias].  allowed int32 [n_masks, ceil(V / 32)] (bit v % 32 of word v / 32), allowed_row int32 [batch, R],
    -1 for rows without a mask (of no masks at all, n_masks 0, it is not looked at).  status int32 [batch]."""
    dev, index, code = _logits_of(logits, "logits")
    B, R, V = shape = logits.shape
    lp, sb, sr = _need_logits(logits, shape, logits.dtype, index, "logits")
    if out is None or out is logits:
        out, op, ob, orow = logits, lp, sb, sr
    else:
        op, ob, orow = _need_logits(out, shape, logits.dtype, index, "out")
    hp, hs, hc = None, 0, 0
    if history is not None:
        _need(history.dim() == 2 and history.shape[0] == B and history.dtype is torch.int32 and history.get_device() == index
              and (history.shape[1] <= 1 or history.stride(1) == 1), "history must be an int32 tensor [batch, n] on the call's device with contiguous rows")
        hc = history.shape[1]
        hp, hs = (history.data_ptr(), history.stride(0) if B > 1 else 0) if hc else (None, 0)
    else:
        _need(history_len is None and prompt_len is None, "history_len and prompt_len come with history")
    if (bias_token is None) != (bias is None) or (allowed is None) != (allowed_row is None) or (token_ids is None) != (parent_idx is None):
        raise ValueError("bias comes with bias_token, allowed with allowed_row, token_ids with parent_idx")
    n_bias, n_allowed, f32, i32 = 0, 0, torch.float32, torch.int32
    if bias is not None:
        _need(bias.dim() == 2, "bias must be [batch, n_bias]")
        n_bias = bias.shape[1]
    if allowed is not None:
        _need(allowed.dim() == 2, "allowed must be [n_masks, ceil(V / 32)]")
        n_allowed = allowed.shape[0]
    a = AdjustArgs(C.sizeof(AdjustArgs), flags, B, R, code, n_bias, V, lp, sb, sr, op, ob, orow,
                   _need_like(n_nodes, i32, (B,), index, "n_nodes"), _need_like(token_ids, i32, (B, R), index, "token_ids"),
                   _need_like(parent_idx, i32, (B, R), index, "parent_idx"), hp, hs, hc, n_allowed,
                   _need_like(history_len, i32, (B,), index, "history_len"), _need_like(prompt_len, i32, (B,), index, "prompt_len"),
                   _need_like(repetition, f32, (B,), index, "repetition"), _need_like(presence, f32, (B,), index, "presence"),
                   _need_like(frequency, f32, (B,), index, "frequency"), _need_like(bias_token, i32, (B, n_bias), index, "bias_token"),
                   _need_like(bias, f32, (B, n_bias), index, "bias"), _need_like(allowed, i32, (n_allowed, (V + 31) // 32), index, "allowed"),
                   _need_like(allowed_row, i32, (B, R), index, "allowed_row"), _need_like(status, i32, (B,), index, "status"))
    _enqueue(lib().cadd_adjust_logits, a, dev, stream)
    return out


@dataclass
class Distilled:
    """Outputs of cadd_distill_loss (device tensors): loss fp32 [batch, L], stats fp32 [batch, L, 4], grad like the logits and
    status int32 [batch]; those that are None are not written."""
    loss: Optional[torch.Tensor] = None
    stats: Optional[torch.Tensor] = None
    grad: Optional[torch.Tensor] = None
    status: Optional[torch.Tensor] = None


def _distill_args(x, teacher_token, teacher_logit, teacher_lse, rest, temperature, path, path_len, n_rows, weight, grad_loss, out, flags, stream):
    dev, index, code = _logits_of(x, "draft_logits")
    B, L, V = shape = x.shape
    _need(teacher_token.dim() == 3 and teacher_token.shape[0] == B, "teacher_token must be [batch, R, K]")
    R, K = teacher_token.shape[1:]
    _need(teacher_lse is None or rest, "teacher_lse goes with rest")
    f32, f64, i32, P = torch.float32, torch.float64, torch.int32, 0
    if path is not None:
        _need(path_len is not None and n_rows is None, "path comes with path_len and without n_rows")
        _need(path.dim() == 2, "path must be [batch, columns]")
        path = _some_column(path, B, dev, stream)
        P = path.shape[1]
    else:
        _need(path_len is None, "path_len comes with path")
    gp, gb, gl = (None, 0, 0) if out.grad is None else _need_logits(out.grad, shape, x.dtype, index, "grad")
    return dev, DistillArgs(
        C.sizeof(DistillArgs), flags | (DISTILL_REST if rest else 0), B, L, R, K, code, P, V, float(temperature), *_need_logits(x, shape, x.dtype, index, "draft_logits"),
        _need_like(teacher_token, i32, (B, R, K), index, "teacher_token"), _need_like(teacher_logit, f64, (B, R, K), index, "teacher_logit"),
        _need_like(teacher_lse, f64, (B, R), index, "teacher_lse"), _need_like(path, i32, (B, P), index, "path"), _need_like(path_len, i32, (B,), index, "path_len"),
        _need_like(n_rows, i32, (B,), index, "n_rows"), _need_like(weight, f32, (B, L), index, "weight"), _need_like(grad_loss, f32, (B, L), index, "grad_loss"),
        _need_like(out.loss, f32, (B, L), index, "loss"), _need_like(out.stats, f32, (B, L, 4), index, "stats"), gp, gb, gl, _need_like(out.status, i32, (B,), index, "status"))


def cadd_distill_loss(draft_logits: torch.Tensor, teacher_token: torch.Tensor, teacher_logit: torch.Tensor, *, teacher_lse=None,
                      rest: bool = False, temperature: float = 1.0, path=None, path_len=None, n_rows=None, weight=None, grad_loss=None,
                      grad: bool = False, out: Optional[Distilled] = None, flags: int = 0,
                      stream: Optional[torch.cuda.Stream] = None) -> Distilled:
    """Distillation: the divergence of the drafter's distribution at each position of draft_logits [batch, L, V] from the
    target's top tokens, teacher_token int32 and teacher_logit fp64 [batch, R, K] (cadd_build_tree's topk_token and topk_logprob fit),
    and with `grad` (with `out`: where it has a grad, which may be draft_logits itself) the gradient of its sum in the same pass: go on with
    draft_logits.backward(result.grad).  Position i learns from row i of the lists, with path / path_len (a verification's
    accepted_nodes / accepted_len) from row 0, then from the accepted nodes, as far as they go (a path without a column: from row 0 alone).  `rest`: all tokens that are not
    listed are one more class (teacher_logit are then log-probabilities, or logits with teacher_lse fp64 [batch, R]).
    weight and grad_loss fp32 [batch, L]; n_rows int32 [batch]."""
    dev = draft_logits.device
    _need(out is None or not grad or out.grad is not None, "grad goes with out.grad, where out is given")
    if out is None:
        _need(dev.type == "cuda" and draft_logits.dim() == 3, "draft_logits must be a CUDA tensor [batch, L, V] (there is no CPU path)")
        B, L = draft_logits.shape[:2]
        with torch.cuda.stream(_stream_of(stream, dev)):
            out = Distilled(loss=torch.empty(B, L, device=dev), stats=torch.empty(B, L, 4, device=dev),
                            grad=torch.empty(draft_logits.shape, dtype=draft_logits.dtype, device=dev) if grad else None,
                            status=torch.empty(B, dtype=torch.int32, device=dev))
    dev, a = _distill_args(draft_logits, teacher_token, teacher_logit, teacher_lse, rest, temperature, path, path_len, n_rows, weight, grad_loss, out, flags, stream)
    _enqueue(lib().cadd_distill_loss, a, dev, stream)
    return out


def cadd_distill_grad(draft_logits: torch.Tensor, teacher_token: torch.Tensor, teacher_logit: torch.Tensor, stats: torch.Tensor, *,
                      teacher_lse=None, rest: bool = False, temperature: float = 1.0, path=None, path_len=None, n_rows=None, weight=None,
                      grad_loss=None, grad: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, flags: int = 0,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The gradient of cadd_distill_loss with respect to draft_logits, given the gradient grad_loss fp32 [batch, L] of its losses (1
    without) and the stats it left; the other arguments as there.  Returns grad (made here unless given; may be draft_logits)."""
    dev = draft_logits.device
    if grad is None:
        _need(dev.type == "cuda" and draft_logits.dim() == 3, "draft_logits must be a CUDA tensor [batch, L, V] (there is no CPU path)")
        with torch.cuda.stream(_stream_of(stream, dev)):
            grad = torch.empty(draft_logits.shape, dtype=draft_logits.dtype, device=dev)
    dev, a = _distill_args(draft_logits, teacher_token, teacher_logit, teacher_lse, rest, temperature, path, path_len, n_rows, weight, grad_loss,
                           Distilled(stats=stats, grad=grad, status=status), flags, stream)
    _enqueue(lib().cadd_distill_grad, a, dev, stream)
    return grad
