"""Tree attention where numbers and shapes leave the ordinary: weights far below the largest, queries whose elements differ by
many powers of two, ranges of many units (buffers reused, the running maximum raised, steps of a warp one after the other), and
what rows with non-finite numbers cost."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from cache_util import Problem, check_attention, decode, encode

pytestmark = pytest.mark.gpu
DEV = "cuda"


def problem(**kw):
    d = dict(batch=2, heads=2, group=2, dim=128, page=16, fp4=False, lens=[70, 33], R=5, live=[5, 3], causal=False, seed=1)
    d.update(kw)
    return Problem(**d)


def store(p, which, b, x):
    """Rows x [n, heads, dim] in place of request b's keys (0) or values (1)."""
    if p.fp4:
        exp = (p.k_exp, p.v_exp)[which]
        codes, scales = encode(x, exp)
        p.put(which, b, 0, codes)
        p.put(which + 2, b, 0, scales)
        x = decode(codes, scales, exp)
    else:
        x = x.bfloat16().double()
        p.put(which, b, 0, x.bfloat16())
    (p.V if which else p.K)[b] = x


FLAGS = [0, G.ATTENTION_TILED_PATH]


@pytest.mark.parametrize("fp4,flags", [(False, 0), (True, 0), (True, G.ATTENTION_TILED_PATH)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gap", [8.0, 17.0, 20.0, 23.0, 40.0, 80.0])
@pytest.mark.parametrize("at", [0, 150, 299])
def test_one_key_far_above_the_rest_whose_value_is_zero(fp4, flags, dim, gap, at):
    """What a row gets is then a sum over weights of e^-gap and less, each of which is to be good to its rounding: the outputs'
    tolerance goes by the sum of their products with the values."""
    p = problem(fp4=fp4, dim=dim, lens=[300, 300], R=2, live=[2, 1], group=4, seed=int(gap))
    p.q[:] = 1.0
    p.k[:] = 0.0
    for b in range(2):
        k, v = p.K[b] * 0.125, p.V[b].clone()
        k[at], v[at] = 1.0, 0.0
        store(p, 0, b, k)
        store(p, 1, b, v)
    p.scale = gap / float(p.K[0][at, 0].sum())
    check_attention(p, p.run(G, flags=flags))


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("power", [12, 16, 20, 30, 33, 60, 100, -100])
@pytest.mark.parametrize("every", [True, False])
def test_queries_with_an_element_far_above_the_others(flags, dim, power, every):
    """Keys are zero at that element, so the scores are the other elements', which have to keep their bits."""
    p = problem(fp4=True, dim=dim, lens=[400, 90], R=3, live=[3, 3], group=4, seed=5)
    for b in range(2):
        k = p.K[b].clone()
        k[:, :, 5] = 0.0
        store(p, 0, b, k)
    p.k[..., 5] = 0.0
    rows = slice(None) if every else slice(1, 2)
    p.q[:, rows, :, 5] = 1.5 * 2.0 ** power
    if power < 0:
        p.q[:, rows] = p.q[:, rows, :, 5:6] * (1 + torch.arange(dim) % 3)
    check_attention(p, p.run(G, flags=flags))


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 40])
def test_small_and_large_scales(flags, scale):
    """Queries make up for the scale; a row of the smallest normal numbers has scores of nearly zero."""
    p = problem(fp4=True, lens=[75, 40], R=3, live=[3, 3], group=4, seed=9, scale=scale, k_exp=16, v_exp=0)
    p.q = (p.q.double() / scale * 128 ** -0.5 * 2.0 ** 16).bfloat16()
    p.q[0, 1] = 2.0 ** -126
    p.k = (p.k.double() * 2.0 ** -16).bfloat16()
    check_attention(p, p.run(G, flags=flags))


LONG = [(False, 0, 16), (False, 0, 64), (True, 0, 16), (True, 0, 64), (True, G.ATTENTION_TILED_PATH, 64)]


@pytest.mark.parametrize("fp4,flags,page", LONG)
@pytest.mark.parametrize("growing", [False, True])
def test_ranges_of_many_units(fp4, flags, page, growing):
    """Eight heads over 20000 places: 2500 units and more for some 300 ranges, so a CTA goes through eight and more of one item, and a warp
    of the few-rows kernel through several steps.  Growing: keys whose scores rise by far more than 40 powers of two along a range."""
    p = problem(batch=1, heads=8, group=2, page=page, fp4=fp4, lens=[20011], R=2, live=[2], seed=2, scale=8.0 if growing else None)
    if growing:
        store(p, 0, 0, p.K[0] * torch.linspace(0.05, 3.0, 20011, dtype=torch.float64)[:, None, None])
    got = p.run(G, flags=flags)
    check_attention(p, got)
    again = p.run(G, flags=flags)
    assert torch.equal(again.out, got.out) and torch.equal(again.lse, got.lse)


@pytest.mark.parametrize("fp4", [False, True])
def test_blocks_of_rows_over_many_units(fp4):
    """Two blocks of rows to an item, the second one partly empty, over ranges of many units; a window whose units lie apart from the sinks'."""
    p = problem(batch=1, heads=4, group=8, page=32, fp4=fp4, lens=[20011], R=20, live=[20], seed=3)
    check_attention(p, p.run(G))
    p.window, p.sinks = 15000, 70
    check_attention(p, p.run(G))


def time_of(call):
    call()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    call()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("fp4,R", [(False, 4), (True, 4), (True, 40)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_rows_with_results_that_are_not_finite_are_walked_once(fp4, R, value):
    """A value row of Inf or NaN that all rows see.  Bound: the 16 rows of a block go once through 8192 places, shared out over 8 warps,
    at no more than 1 us a key and warp (a look-up, a row and five exchanges one after the other): 16 * 8232 / 8 us."""
    p = problem(fp4=fp4, batch=1, heads=1, group=4, lens=[8192], R=R, live=[R], page=64)
    p.v[0, 0] = value
    c = p.cache(G)
    q, k, v, mask, depth = (x.to(DEV) for x in (p.q, p.k, p.v, p.mask_bits(), p.depth))
    out = G.Attention(out=torch.zeros(1, R, 4, 128, dtype=torch.bfloat16, device=DEV), lse=torch.zeros(1, R, 4, device=DEV))
    ws = torch.zeros(G.cadd_tree_attention_workspace_bytes(1, R, 4, c), dtype=torch.uint8, device=DEV)
    ms = time_of(lambda: G.cadd_tree_attention(q, k, v, c, mask_bits=mask, depth=depth, out=out, workspace=ws))
    if value == math.inf:
        assert bool((out.out == math.inf).all())
    else:
        assert bool(torch.isnan(out.out).all())
    assert bool(torch.isfinite(out.lse).all())
    assert ms <= 16 * 8232 / 8 * 1e-3, ms


@pytest.mark.parametrize("fp4,R", [(False, 4), (True, 4), (False, 50), (True, 50)])
def test_single_elements_that_are_not_finite(fp4, R):
    """In a long cache: one element of a tree row's value is Inf and another NaN; everything else is what it was without them."""
    p = problem(fp4=fp4, batch=1, heads=2, group=2, lens=[3001], R=R, live=[R], page=32)
    last = R - 1
    p.v[0, 0, 0, 17], p.v[0, last, 1, 90], p.v[0, last, 0, 0] = math.inf, math.nan, -math.inf
    got = p.run(G).out.cpu().double()
    p.v[0, 0, 0, 17] = p.v[0, last, 1, 90] = p.v[0, last, 0, 0] = 0.0
    want, _, amass, _ = p.attention(0)
    sees = p.mask[0, :, last]
    odd = torch.zeros(R, 4, 128, dtype=torch.bool)
    odd[:, :2, 17] = True
    odd[sees, 2:, 90] = True
    odd[sees, :2, 0] = True
    assert bool((got[0, :, :2, 17] == math.inf).all()) and bool(torch.isnan(got[0, sees][:, 2:, 90]).all()) and bool((got[0, sees][:, :2, 0] == -math.inf).all())
    err = (got[0] - want).abs()[~odd]
    assert bool((err <= 2.0 ** -6 * amass[~odd] + 1e-6).all())


def test_rows_lost_to_fp16_whose_results_are_not_finite():
    """Queries that the few-rows kernel cannot hold in fp16, over values of NaN that all or some of a row's elements get: lse, and the
    other elements, are still the row's."""
    p = problem(fp4=True, lens=[300, 70], R=2, live=[2, 2], group=2, heads=1)
    p.q[..., 9] = 2.0 ** -70
    wants = [p.attention(b) for b in range(2)]
    root = p.v[:, 0].clone()
    p.v[0, 0], p.v[1, 0, 0, 3] = math.nan, math.nan
    got = p.run(G)
    assert bool(torch.isnan(got.out[0]).all()) and bool(torch.isnan(got.out[1, :, :, 3]).all())
    p.v[:, 0] = root
    out = got.out.cpu()
    for b, at in ((0, slice(None)), (1, slice(3, 4))):
        out[b, ..., at] = wants[b][0][..., at].bfloat16()
    check_attention(p, G.Attention(out=out, lse=got.lse))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R,group", [(1, 4), (20, 4), (40, 7)])
def test_non_finite_rows_in_ranges_of_many_items(fp4, dim, R, group):
    """Hundreds of items of a few units each: a range goes through several whole ones and parts of others, some with elements that are not
    finite, different ones in each."""
    batch = 150
    g = torch.Generator().manual_seed(R)
    lens, live = torch.randint(0, 200, (batch,), generator=g).tolist(), torch.randint(1, R + 1, (batch,), generator=g).tolist()
    p = problem(fp4=fp4, batch=batch, heads=4, dim=dim, group=group, lens=lens, R=R, live=live, page=64)
    clean = p.run(G)
    put = {}
    for b in range(0, batch, 3):
        h, d = int(torch.randint(0, 4, (), generator=g)), int(torch.randint(0, dim, (), generator=g))
        value = (math.nan, math.inf, -math.inf)[b // 3 % 3]
        put[b] = (h, d, value)
        p.v[b, 0, h, d] = value
    got = p.run(G)
    assert torch.equal(got.lse, clean.lse)
    want = clean.out.clone()
    for b, (h, d, value) in put.items():
        want[b, :live[b], h * group:(h + 1) * group, d] = value           # the root: every row sees it
    assert torch.equal(torch.isnan(got.out), torch.isnan(want)) and torch.equal(torch.nan_to_num(got.out, nan=0.0), torch.nan_to_num(want, nan=0.0))
