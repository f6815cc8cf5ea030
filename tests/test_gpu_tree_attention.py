"""cadd_tree_attention against its definition in 64 bits: both cache forms, head layouts, lengths and pages of every kind,
trees, prompt chunks, windows, rows that see nothing, and what lies in places that nobody sees."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from cache_util import Problem, attention_tolerance, check_attention

pytestmark = pytest.mark.gpu


def problem(**kw):
    d = dict(batch=2, heads=2, group=2, dim=128, page=16, fp4=False, lens=[70, 33], R=5, live=[5, 3], causal=False, seed=1)
    d.update(kw)
    return Problem(**d)


FORMS = [(fp4, dim) for fp4 in (False, True) for dim in (64, 128)]


@pytest.mark.parametrize("fp4,dim", FORMS)
@pytest.mark.parametrize("length", [0, 1, 2, 31, 32, 33, 127, 128, 129, 255, 257, 600])
def test_one_token_at_every_kind_of_length(fp4, dim, length):
    p = problem(fp4=fp4, dim=dim, lens=[length, 5], R=1, live=[1, 1], group=4)
    got = p.run(G)
    check_attention(p, got)
    assert int(got.status.abs().max()) == 0


@pytest.mark.parametrize("fp4,dim", FORMS)
@pytest.mark.parametrize("R,group", [(2, 1), (3, 5), (4, 4), (2, 8), (16, 1), (17, 1), (5, 7), (33, 4), (32, 4), (65, 2), (129, 1), (70, 8), (300, 3)])
def test_trees_of_every_kind_of_size(fp4, dim, R, group):
    p = problem(fp4=fp4, dim=dim, R=R, live=[R, max(1, R // 2)], group=group, lens=[150, 0], seed=R)
    check_attention(p, p.run(G))


@pytest.mark.parametrize("fp4,dim", FORMS)
@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 128, 256])
@pytest.mark.parametrize("token_major", [False, True])
def test_pages_that_end_inside_tiles(fp4, dim, page, token_major):
    p = problem(fp4=fp4, dim=dim, page=page, lens=[259, 100], R=9, live=[9, 9], heads=3, group=3, token_major=token_major, seed=page)
    check_attention(p, p.run(G))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("R,group", [(1, 4), (13, 1), (40, 4), (200, 1), (260, 2)])
@pytest.mark.parametrize("length", [0, 90, 300])
def test_prompt_chunks(fp4, R, group, length):
    p = problem(fp4=fp4, R=R, live=[R, (R + 1) // 2], group=group, lens=[length, 17], causal=True, seed=R + length)
    check_attention(p, p.run(G))


@pytest.mark.parametrize("fp4,dim", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 1), (40, 0), (64, 4), (130, 129), (200, 500), (5000, 2)])
@pytest.mark.parametrize("R,causal", [(1, True), (12, False), (150, False), (150, True)])
def test_windows_and_sinks(fp4, dim, window, sinks, R, causal):
    p = problem(fp4=fp4, dim=dim, R=R, live=[R, max(1, R // 3)], lens=[420, 9], causal=causal, window=window, sinks=sinks, seed=window)
    check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [6, 80])
def test_rows_that_see_nothing_give_zero(R):
    for lens in ([0, 0], [0, 40]):
        p = problem(R=R, live=[R, R], lens=lens)
        p.mask[:, 1] = False
        p.mask[0, R - 2] = False
        check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [6, 80])
def test_masks_need_not_be_trees(R):
    p = problem(R=R, live=[R, R - 1], lens=[50, 3])
    p.mask[:] = torch.rand(p.mask.shape, generator=p.g) < 0.3
    p.mask[1, :, R - 1] = False
    check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [4, 100])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_has_no_influence(R, value):
    """Non-finite numbers in tree rows that other rows do not see, in live rows' hidden window and in rows behind the live ones."""
    p = problem(R=R, live=[R, R // 2], lens=[200, 90], window=60, sinks=2, seed=3)
    for b in range(2):
        p.k[b, p.live[b]:] = value
        p.v[b, p.live[b]:] = value
    clean = p.run(G)
    check_attention(p, clean)
    # a row nobody but itself sees, and places outside every row's window
    last = R - 1
    others = [j for j in range(R) if not bool(p.mask[0, j, last])]
    p.v[0, last] = value
    p.k[0, last] = value
    for pos in (2, 50, 100, 139):
        for pool in p.pools:
            pool[int(p.block_table[0, pos // p.page]), :, pos % p.page] = value
    dirty = p.run(G)
    assert len(others) >= R // 2
    for b, rows in ((0, others), (1, list(range(R // 2)))):
        # the same numbers go through the same steps, except that a row may be redone alone: equal up to the tolerances
        p2 = problem(R=R, live=[R, R // 2], lens=[200, 90], window=60, sinks=2, seed=3)
        want, wlse, amass, size = p2.attention(b)
        assert bool(((dirty.out[b, rows].cpu().double() - want[rows]).abs() <= 2.0 ** -6 * amass[rows] + 1e-6).all())
        assert bool(((dirty.lse[b, rows].cpu().double() - wlse[rows]).abs() <= 1e-4).all())


@pytest.mark.parametrize("R", [4, 100])
def test_what_a_row_sees_counts(R):
    p = problem(R=R, live=[R, R], lens=[200, 90])
    p.v[0, 0, 0, 7] = math.nan                                  # the root: every row sees it; head 0, element 7
    got = p.run(G)
    bad = torch.isnan(got.out.cpu())
    assert bool(bad[0, :, :2, 7].all()) and int(bad.sum()) == R * 2
    p = problem(R=R, live=[R, R], lens=[200, 90])
    p.v[1, 0, 1, 3] = math.inf
    got = p.run(G)
    inf = torch.isinf(got.out.cpu())
    assert bool(inf[1, :, 2:, 3].all()) and int(inf.sum()) == R * 2 and not bool(torch.isnan(got.out).any())


def test_minus_infinity_scores_carry_no_weight():
    p = problem(R=3, live=[3, 3], lens=[20, 20], causal=True)
    p.q[:] = p.q.abs() + 0.5
    p.k[0, 1] = -math.inf                                       # row 1 of request 0: scores of -Inf for rows 1 and 2
    p.mask[0, 1:, 1] = False
    check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [3, 60])
def test_large_scores(R):
    """Scores of some thousands, growing along the keys, so that the running maximum rises again and again."""
    p = problem(R=R, live=[R, R], lens=[700, 300], scale=3.0)
    for b in range(2):
        n = p.lens[b]
        p.K[b] = (p.K[b] * torch.linspace(0.1, 4.0, n, dtype=torch.float64)[:, None, None]).bfloat16().double()
        p.put(0, b, 0, p.K[b].bfloat16())
    check_attention(p, p.run(G))


@pytest.mark.parametrize("k_exp,v_exp", [(0, 0), (3, -2), (-5, 9), (16, 16), (-16, -16)])
@pytest.mark.parametrize("R", [2, 50])
def test_exponents_of_the_four_bit_form(k_exp, v_exp, R):
    p = problem(fp4=True, R=R, live=[R, R], k_exp=k_exp, v_exp=v_exp, lens=[140, 30], scale=0.09 * 2.0 ** min(k_exp, 0))
    p.q = (p.q.float() * 0.25).bfloat16()
    check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [7, 90])
def test_strided_operands_and_outputs(R):
    p = problem(R=R, live=[R - 1, R], lens=[77, 130], heads=2, group=3)
    dev = "cuda"
    B, HQ, H, D = 2, 6, 2, 128
    big = torch.full((B, HQ + 2 * H + 1, R + 2, D), 7.0, dtype=torch.bfloat16, device=dev)    # head-major, one allocation
    view = big.permute(0, 2, 1, 3)
    view[:, :R, :HQ], view[:, :R, HQ:HQ + H], view[:, :R, HQ + H:HQ + 2 * H] = p.q.to(dev), p.k.to(dev), p.v.to(dev)
    out = torch.full((B, HQ, R, D + 8), -3.0, dtype=torch.bfloat16, device=dev)
    o = out.permute(0, 2, 1, 3)[..., :D]
    lse = torch.full((B, R, HQ), 5.0, device=dev)
    got = G.cadd_tree_attention(view[:, :R, :HQ], view[:, :R, HQ:HQ + H], view[:, :R, HQ + H:HQ + 2 * H], p.cache(G), mask_bits=p.mask_bits().to(dev),
                                depth=p.depth.to(dev), n_nodes=torch.tensor([R - 2, R - 1], dtype=torch.int32, device=dev),
                                out=G.Attention(out=o, lse=lse))
    check_attention(p, G.Attention(out=got.out.contiguous(), lse=got.lse), before_out=torch.full((B, R, HQ, D), -3.0))
    assert bool((out[..., D:] == -3.0).all()) and bool((lse[0, R - 1] == 5.0).all())


@pytest.mark.parametrize("R", [1, 40])
def test_no_live_rows_leaves_everything(R):
    p = problem(R=R, live=[R, R])
    dev = "cuda"
    out = G.Attention(out=torch.full((2, R, 4, 128), 9.0, dtype=torch.bfloat16, device=dev), lse=torch.full((2, R, 4), 9.0, device=dev),
                      status=torch.full((2,), -7, dtype=torch.int32, device=dev))
    G.cadd_tree_attention(p.q.to(dev), p.k.to(dev), p.v.to(dev), p.cache(G), n_nodes=torch.tensor([-1, -1], dtype=torch.int32, device=dev), out=out)
    assert bool((out.out == 9.0).all()) and bool((out.lse == 9.0).all()) and out.status.tolist() == [0, 0]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("R", [2, 50])
def test_bad_pages_lengths_and_row_counts_are_flagged_and_not_followed(fp4, R):
    p = problem(fp4=fp4, R=R, live=[R, R], lens=[100, 60], page=16)
    keep = torch.ones(100, dtype=torch.bool)
    table = p.block_table.clone()
    table[0, 2], table[0, 5] = -1, p.n_pages                     # places 32..47 and 80..95 are nowhere
    keep[32:48] = False
    keep[80:96] = False
    c = p.cache(G)
    dev = "cuda"
    bad = G.KvCache(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, block_table=table.to(dev), length=c.length)
    got = p.run(G, cache=bad)
    assert got.status.tolist() == [G.STATUS_BAD_PAGE, 0]
    p.K[0], p.V[0] = p.K[0][keep], p.V[0][keep]
    p.lens[0] = int(keep.sum())
    check_attention(p, got)
    # a length outside the table, a row count outside the rows
    p = problem(fp4=fp4, R=R, live=[R, R], lens=[64, 64], page=16)
    c = p.cache(G)
    odd = G.KvCache(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, block_table=c.block_table,
                    length=torch.tensor([64 + 1000, -5], dtype=torch.int32, device=dev))
    got = G.cadd_tree_attention(p.q.to(dev), p.k.to(dev), p.v.to(dev), odd, n_nodes=torch.tensor([R + 7, -9], dtype=torch.int32, device=dev),
                                mask_bits=p.mask_bits().to(dev))
    assert got.status.tolist() == [G.STATUS_BAD_LENGTH | G.STATUS_BAD_N_NODES] * 2
    p.live = [R, 0]
    p.lens = [64, 0]
    p.K[1] = p.K[1][:0]; p.V[1] = p.V[1][:0]
    check_attention(p, got)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("R", [1, 30])
def test_a_length_that_fills_its_pages_and_ragged_batches(fp4, R):
    lens = [0, 1, 16, 31, 32, 500, 64, 0, 77, 128, 1300]
    p = problem(fp4=fp4, batch=len(lens), lens=lens, R=R, live=[1 + (7 * i) % R for i in range(len(lens))], group=4, heads=1)
    check_attention(p, p.run(G))


@pytest.mark.parametrize("R", [1, 60])
def test_repeated_and_captured_calls_give_the_same_bits(R):
    p = problem(fp4=True, R=R, live=[R, R], lens=[3000, 1111], group=4)
    dev = "cuda"
    c = p.cache(G)
    n = G.cadd_tree_attention_workspace_bytes(2, R, 8, c)
    q, k, v, mask, depth = (x.to(dev) for x in (p.q, p.k, p.v, p.mask_bits(), p.depth))
    outs = [G.Attention(out=torch.zeros(2, R, 8, 128, dtype=torch.bfloat16, device=dev), lse=torch.zeros(2, R, 8, device=dev)) for _ in range(4)]
    ws = [torch.full((n,), fill, dtype=torch.uint8, device=dev) for fill in (0, 255, 7, 90)]

    def call(i, stream=None):
        G.cadd_tree_attention(q, k, v, c, mask_bits=mask, depth=depth, out=outs[i], workspace=ws[i], stream=stream)
    call(0)
    call(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(3)
    for _ in range(3):
        outs[3].out.zero_()
        graph.replay()
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o.out, outs[0].out) and torch.equal(o.lse, outs[0].lse)
    check_attention(p, outs[0])


@pytest.mark.parametrize("fp4", [False, True])
def test_two_calls_at_once_on_two_streams(fp4):
    ps = [problem(fp4=fp4, R=40, live=[40, 30], lens=[2500, 900], group=4, seed=s) for s in (1, 2)]
    caches = [p.cache(G) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    outs = []
    for p, c, s in zip(ps, caches, streams):
        with torch.cuda.stream(s):
            outs.append(p.run(G, cache=c))
    torch.cuda.synchronize()
    for p, o in zip(ps, outs):
        check_attention(p, o)


def test_places_behind_two_to_the_thirty_one_bytes():
    """A pool of more than 2^32 bytes, its last pages in use: row offsets need 64 bits."""
    dev = "cuda"
    H, P, D = 8, 64, 128
    n_pages = (1 << 32) // (H * P * D * 2) + 40
    k = torch.zeros(n_pages, H, P, D, dtype=torch.bfloat16, device=dev)
    v = torch.zeros(n_pages, H, P, D, dtype=torch.bfloat16, device=dev)
    p = problem(heads=H, group=1, page=P, lens=[130, 70], R=20, live=[20, 20])
    last = torch.arange(n_pages - 6, n_pages, dtype=torch.int32).reshape(2, 3)
    for b in range(2):
        for i in range(3):
            k[int(last[b, i])] = p.pools[0][int(p.block_table[b, i])].to(dev)
            v[int(last[b, i])] = p.pools[1][int(p.block_table[b, i])].to(dev)
    c = G.KvCache(k=k, v=v, block_table=last.to(dev), length=torch.tensor(p.lens, dtype=torch.int32, device=dev))
    check_attention(p, p.run(G, cache=c))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("R,group", [(1, 4), (20, 4), (150, 1)])
def test_many_more_items_than_the_device_holds_at_once(fp4, R, group):
    """Hundreds of requests with a few keys each: every range goes through several whole items and parts of others."""
    batch = 160
    g = torch.Generator().manual_seed(R)
    lens = torch.randint(0, 300, (batch,), generator=g).tolist()
    live = torch.randint(0, R + 1, (batch,), generator=g).tolist()
    p = problem(fp4=fp4, batch=batch, heads=8, dim=64, group=group, lens=lens, R=R, live=live, page=64)
    got = p.run(G)
    status = got.status.clone()
    for _ in range(3):
        again = p.run(G)
        assert torch.equal(again.out, got.out) and torch.equal(again.lse, got.lse)
    assert int(status.abs().max()) == 0
    pick = Problem(**{f: getattr(p, f) for f in ("batch", "heads", "group", "dim", "page", "fp4", "lens", "R", "live", "causal", "seed")})
    for b in list(range(0, batch, 16)) + [batch - 1]:
        want, wlse, amass, size = pick.attention(b)
        tol, tol_lse = attention_tolerance(pick, want, wlse, amass, size, pick.lens[b] + pick.live[b])
        n = pick.live[b]
        assert bool(((got.out[b, :n].cpu().double() - want).abs() <= tol).all())
        assert bool(((got.lse[b, :n].cpu().double() - wlse).abs() <= tol_lse).all())
        assert bool((got.out[b, n:] == 0).all())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R,group,length", [(1, 1, 5000), (1, 16, 333), (2, 8, 1000), (16, 1, 77), (5, 3, 640), (1, 7, 0)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_both_kernels_for_few_rows_over_four_bits(dim, R, group, length, window, sinks):
    p = problem(fp4=True, dim=dim, R=R, live=[R, R], group=group, lens=[length, 130], window=window, sinks=sinks, page=16, seed=R)
    few, tiled = p.run(G), p.run(G, flags=G.ATTENTION_TILED_PATH)
    check_attention(p, few)
    check_attention(p, tiled)


def test_few_rows_see_what_they_see():
    """Values that are not finite in the tree of a small call over a 4-bit cache: no influence on rows that do not see them."""
    p = problem(fp4=True, R=4, live=[4, 4], group=4, lens=[90, 10])
    p.mask[0, :, 3] = False
    p.mask[0, 3, 3] = True
    clean = p.run(G)
    p.v[0, 3], p.k[0, 3] = math.nan, math.inf
    dirty = p.run(G)
    want, wlse, amass, size = p.attention(1)
    assert bool(torch.isfinite(dirty.out[0, :3]).all()) and bool(torch.isnan(dirty.out[0, 3]).any())
    assert bool(((dirty.out[0, :3].double() - clean.out[0, :3].double()).abs() <= 2.0 ** -6 * clean.out[0, :3].double().abs() + 2.0 ** -6).all())
    assert torch.equal(dirty.out[1], clean.out[1])
