"""Host-side checks of the cache and tree-attention calls: what they refuse, before anything is launched.  The pointers given
here are never followed: every call is refused for another reason, and the good call itself is not made."""
import ctypes as C

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from paper_2606_01813_b200 import build as B
from cache_util import E2M1, E4M3, decode, encode

PTR = 1 << 20


@pytest.fixture(scope="module")
def lib():
    B.build()
    return G.lib()


def cache(fp4=True):
    c = G.CacheArgs()
    c.struct_size = C.sizeof(G.CacheArgs)
    c.format, c.batch, c.heads, c.head_dim, c.page_size, c.max_pages, c.n_pages = int(fp4), 2, 4, 128, 16, 10, 40
    c.stride_page, c.stride_head, c.stride_slot = 64, 16, 1
    for f in ("k", "v", "k_scale", "v_scale", "block_table", "length"):
        setattr(c, f, PTR)
    return c


def fill(a, **kw):
    a.struct_size = C.sizeof(type(a))
    a.cache = cache()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def append():
    return fill(G.AppendArgs(), R=5, L=3, k=PTR, v=PTR, stride_b=5 * 512, stride_row=512, stride_head=128, path=PTR, path_len=PTR, new_length=PTR)


def read():
    return fill(G.ReadArgs(), n_max=5, k=PTR, v=PTR, stride_b=5 * 512, stride_row=512, stride_head=128)


def attention():
    return fill(G.AttentionArgs(), R=33, heads_q=8, scale=0.1, q=PTR, k=PTR, v=PTR, out=PTR, q_stride_b=33 * 1024, q_stride_row=1024, q_stride_head=128,
                kv_stride_b=33 * 512, kv_stride_row=512, kv_stride_head=128, out_stride_b=33 * 1024, out_stride_row=1024, out_stride_head=128,
                mask_bits=PTR, depth=PTR, workspace=PTR, workspace_bytes=1 << 40)


def weights():
    return fill(G.WeightsArgs(), R=5, L=3, heads_q=8, scale=0.1, q=PTR, q_stride_b=5 * 1024, q_stride_row=1024, q_stride_head=128, lse=PTR, path=PTR,
                path_len=PTR, base_length=PTR, weights=PTR, weights_out=PTR, weights_stride=160)


def evict():
    return fill(G.EvictArgs(), budget=64, n_sinks=4, n_recent=8, new_max_pages=4, weights=PTR, weights_stride=160, new_block_table=PTR, new_length=PTR,
                kept=PTR, weights_out=PTR * 2, weights_out_stride=64)


CALLS = {"append": append, "read": read, "attention": attention, "weights": weights, "evict": evict}
NAMES = {"append": "cadd_cache_append", "read": "cadd_cache_read", "attention": "cadd_tree_attention", "weights": "cadd_cache_weights",
         "evict": "cadd_cache_evict"}

OWN = {
    "append": [(dict(R=0), G.ERR_SHAPE), (dict(L=0), G.ERR_SHAPE), (dict(k=None), G.ERR_NULL), (dict(v=None), G.ERR_NULL), (dict(path_len=None), G.ERR_NULL),
               (dict(new_length=None), G.ERR_NULL), (dict(k=PTR + 8), G.ERR_ALIGN), (dict(stride_row=508), G.ERR_ALIGN), (dict(stride_head=-128), G.ERR_SHAPE),
               (dict(status=PTR + 2), G.ERR_ALIGN)],
    "read": [(dict(n_max=0), G.ERR_SHAPE), (dict(k=None), G.ERR_NULL), (dict(v=PTR + 4), G.ERR_ALIGN), (dict(stride_b=4), G.ERR_ALIGN), (dict(start=PTR + 1), G.ERR_ALIGN)],
    "attention": [(dict(R=0), G.ERR_SHAPE), (dict(R=65537), G.ERR_SHAPE), (dict(heads_q=6), G.ERR_SHAPE), (dict(heads_q=0), G.ERR_SHAPE), (dict(window=-1), G.ERR_SHAPE),
                  (dict(n_sinks=-1), G.ERR_SHAPE), (dict(scale=0.0), G.ERR_SHAPE), (dict(scale=-1.0), G.ERR_SHAPE), (dict(scale=float("inf")), G.ERR_SHAPE),
                  (dict(scale=float("nan")), G.ERR_SHAPE), (dict(q=None), G.ERR_NULL), (dict(k=None), G.ERR_NULL), (dict(v=None), G.ERR_NULL),
                  (dict(out=None), G.ERR_NULL), (dict(window=5, depth=None), G.ERR_NULL), (dict(q=PTR + 2), G.ERR_ALIGN), (dict(out=PTR + 8), G.ERR_ALIGN),
                  (dict(q_stride_row=1020), G.ERR_ALIGN), (dict(kv_stride_head=-8), G.ERR_SHAPE), (dict(mask_bits=PTR + 1), G.ERR_ALIGN),
                  (dict(workspace=None), G.ERR_WORKSPACE), (dict(workspace=PTR + 16), G.ERR_WORKSPACE), (dict(workspace_bytes=0), G.ERR_WORKSPACE)],
    "weights": [(dict(R=0), G.ERR_SHAPE), (dict(L=0), G.ERR_SHAPE), (dict(heads_q=7), G.ERR_SHAPE), (dict(scale=0.0), G.ERR_SHAPE), (dict(window=-2), G.ERR_SHAPE),
                (dict(weights_stride=159), G.ERR_SHAPE), (dict(q=None), G.ERR_NULL), (dict(lse=None), G.ERR_NULL), (dict(base_length=None), G.ERR_NULL),
                (dict(weights=None), G.ERR_NULL), (dict(weights_out=None), G.ERR_NULL), (dict(path_len=None), G.ERR_NULL), (dict(lse=PTR + 2), G.ERR_ALIGN)],
    "evict": [(dict(budget=0), G.ERR_SHAPE), (dict(budget=11), G.ERR_SHAPE), (dict(new_max_pages=1, n_recent=13), G.ERR_SHAPE), (dict(n_sinks=-1), G.ERR_SHAPE), (dict(n_recent=-1), G.ERR_SHAPE),
              (dict(new_max_pages=0), G.ERR_SHAPE), (dict(weights_stride=100), G.ERR_SHAPE), (dict(weights_out_stride=63), G.ERR_SHAPE),
              (dict(weights_out=PTR), G.ERR_SHAPE), (dict(weights=None), G.ERR_NULL), (dict(new_block_table=None), G.ERR_NULL), (dict(new_length=None), G.ERR_NULL),
              (dict(kept=None), G.ERR_NULL), (dict(kept=PTR + 2), G.ERR_ALIGN)],
}
CACHE = [(dict(struct_size=8), G.ERR_STRUCT_SIZE), (dict(format=2), G.ERR_DTYPE), (dict(format=-1), G.ERR_DTYPE), (dict(batch=0), G.ERR_SHAPE), (dict(heads=0), G.ERR_SHAPE),
         (dict(head_dim=96), G.ERR_SHAPE), (dict(head_dim=256), G.ERR_SHAPE), (dict(page_size=0), G.ERR_SHAPE), (dict(page_size=24), G.ERR_SHAPE),
         (dict(page_size=1 << 17), G.ERR_SHAPE), (dict(max_pages=0), G.ERR_SHAPE), (dict(max_pages=1 << 26), G.ERR_SHAPE), (dict(n_pages=0), G.ERR_SHAPE),
         (dict(stride_slot=0), G.ERR_SHAPE), (dict(stride_page=-64), G.ERR_SHAPE), (dict(k_exp=17), G.ERR_SHAPE), (dict(v_exp=-17), G.ERR_SHAPE),
         (dict(format=0, k_exp=1), G.ERR_SHAPE), (dict(k=None), G.ERR_NULL), (dict(v_scale=None), G.ERR_NULL), (dict(block_table=None), G.ERR_NULL),
         (dict(length=None), G.ERR_NULL), (dict(v=PTR + 8), G.ERR_ALIGN), (dict(k_scale=PTR + 4), G.ERR_ALIGN), (dict(length=PTR + 2), G.ERR_ALIGN)]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_calls_refuse_bad_arguments(lib, name):
    fn = getattr(lib, NAMES[name])
    assert fn(None, None) == G.ERR_NULL
    a = CALLS[name]()
    a.struct_size -= 8
    assert fn(C.byref(a), None) == G.ERR_STRUCT_SIZE
    for change, code in OWN[name]:
        a = CALLS[name]()
        for k, v in change.items():
            setattr(a, k, v)
        assert fn(C.byref(a), None) == code, change
    for change, code in CACHE:
        a = CALLS[name]()
        for k, v in change.items():
            setattr(a.cache, k, v)
        if name in ("weights", "evict") and change.get("max_pages") == 1 << 26:
            a.weights_stride = 1 << 34
        assert fn(C.byref(a), None) == code, change


def test_more_rows_than_weights_count_are_refused(lib):
    a = weights()
    a.cache.heads, a.heads_q, a.L = 1, 65536, 256                          # 257 rows of 2^16 heads: above 2^24
    assert lib.cadd_cache_weights(C.byref(a), None) == G.ERR_SHAPE
    a.R, a.path, a.path_len = 65536, None, None                            # 2^32
    assert lib.cadd_cache_weights(C.byref(a), None) == G.ERR_SHAPE


def test_workspace_query_is_host_arithmetic(lib):
    a = attention()
    for f in ("q", "k", "v", "out", "workspace"):
        setattr(a, f, None)
    a.cache.k = a.cache.block_table = None
    out = C.c_size_t()
    assert lib.cadd_tree_attention_workspace_bytes(C.byref(a), C.byref(out)) == G.OK and 0 < out.value < 1 << 30
    assert lib.cadd_tree_attention_workspace_bytes(C.byref(a), None) == G.ERR_NULL
    assert lib.cadd_tree_attention_workspace_bytes(None, C.byref(out)) == G.ERR_NULL
    a.heads_q = 5
    assert lib.cadd_tree_attention_workspace_bytes(C.byref(a), C.byref(out)) == G.ERR_SHAPE


def test_binding_refuses_cpu_tensors():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        G.KvCache(k=torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), v=torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16),
                  block_table=i32(1, 4), length=i32(1))


def test_the_plain_four_bit_form():
    """The tests' own encoder: exact on the codes' grid, to nearest even in between, and never off by more than half a step."""
    assert E4M3[0x7e] == 448 and E4M3[1] == 2.0 ** -9 and E4M3[0x38] == 1.0
    grid = torch.cat([E2M1[:8], -E2M1[1:8], torch.tensor([6.0])]).double()
    codes, scales = encode(grid * 0.375)
    assert torch.equal(decode(codes, scales), grid * 0.375)
    x = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 5.01, 2.49, 0.26, 0.0, -6.0, 1.0], dtype=torch.float64)
    want = torch.tensor([6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, -1.0, 6.0, 2.0, 0.5, 0.0, -6.0, 1.0], dtype=torch.float64)
    assert torch.equal(decode(*encode(x)), want)
    g = torch.Generator().manual_seed(2)
    y = torch.randn(50, 64, generator=g, dtype=torch.float64)
    codes, scales = encode(y)
    s = E4M3[scales.long()].repeat_interleave(16, -1)
    assert bool(((decode(codes, scales) - y).abs() <= s * (1 + 6 * 2.0 ** -4)).all())


@pytest.mark.parametrize("name", ["attention", "weights"])
@pytest.mark.parametrize("scale", [1e-45, 2.0 ** -65, 2.0 ** 65, 3e38])
def test_scales_out_of_range_are_refused(lib, name, scale):
    a = CALLS[name]()
    a.scale = scale
    assert getattr(lib, NAMES[name])(C.byref(a), None) == G.ERR_SHAPE


@pytest.mark.parametrize("name,fields", [("read", ("stride_b", "stride_row", "stride_head")), ("attention", ("out_stride_b", "out_stride_row", "out_stride_head"))])
@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("stride", [0, 64])
def test_outputs_whose_rows_lie_in_one_another_are_refused(lib, name, fields, axis, stride):
    a = CALLS[name]()
    setattr(a, fields[axis], stride)
    assert getattr(lib, NAMES[name])(C.byref(a), None) == G.ERR_SHAPE
