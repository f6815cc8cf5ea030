"""cadd_distill_loss and cadd_distill_grad against their definition in 64 bits (logits_util), whose gradient comes from autograd, and a
whole round: adjust, verify, the target's lists, the drafter's gradient."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from paper_2606_01813_b200 import synth
from logits_util import Adjust, Distill, check_adjust, check_grad, check_loss, pack_bits, plain_distill, random_distill, row_loss, teacher_rows

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32)


def put(d: Distill):
    return (d.logits.cuda(), d.teacher_token.cuda(), d.teacher_logit.cuda()), d.args("cuda")


def every(d: Distill, expected=None):
    """Loss alone, loss with gradient, gradient alone, and the latter two in place."""
    expected = expected or plain_distill(d)
    (x, t, v), kw = put(d)
    r = G.cadd_distill_loss(x, t, v, **kw)
    assert r.grad is None
    check_loss(r.loss, r.stats, d, expected)
    both = G.cadd_distill_loss(x, t, v, grad=True, **kw)
    check_loss(both.loss, both.stats, d, expected)
    check_grad(both.grad, expected)
    alone = G.cadd_distill_grad(x, t, v, r.stats, **kw)
    check_grad(alone, expected)
    assert torch.equal(x.view(torch.uint8), d.logits.cuda().view(torch.uint8))
    y = x.clone()
    out = G.Distilled(loss=torch.full_like(r.loss, 5.0), grad=y)
    G.cadd_distill_loss(y, t, v, out=out, **kw)
    assert torch.equal(y, both.grad) and torch.equal(out.loss, both.loss)
    y = x.clone()
    assert G.cadd_distill_grad(y, t, v, r.stats, grad=y, **kw) is y
    assert torch.equal(y, alone)
    return both


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("B,L,V,K", [(1, 1, 1, 1), (2, 3, 7, 9), (1, 2, 33, 256), (3, 4, 1000, 8), (2, 5, 8192, 64), (1, 3, 50257, 20), (2, 2, 32001, 256)])
def test_sizes(dtype, rest, B, L, V, K):
    every(random_distill(B, L, V, K, dtype, seed=B + V + K, rest=rest))


@pytest.mark.parametrize("V", [2048 * 8 - 3, 2048 * 8, 131072 + 5, 300007, 2000000])
def test_segments_of_every_size(V):
    every(random_distill(1, 2, V, 32, torch.bfloat16, seed=V, rest=True))


@pytest.mark.parametrize("rows", [1, 5, 20, 100, 200])
def test_numbers_of_rows(rows):
    every(random_distill(rows, 1, 20000, 8, torch.bfloat16, seed=rows, rest=True))


@pytest.mark.parametrize("T", [0.25, 1.7, 30.0])
@pytest.mark.parametrize("rest", [False, True])
def test_temperatures(T, rest):
    for dtype in (torch.bfloat16, torch.float32):
        every(random_distill(2, 3, 3000, 12, dtype, seed=5, rest=rest, temperature=T, lse=rest))


@pytest.mark.parametrize("rest", [False, True])
def test_paths(rest):
    d = random_distill(6, 8, 2000, 10, torch.float32, seed=3, rest=rest, path=True)
    d.path_len[0], d.path_len[1] = 0, 7
    d.path[1] = torch.arange(1, 9)
    every(d)
    d.path = d.path[:, :4].contiguous()                                   # fewer columns than positions
    d.path_len.clamp_(max=4)
    every(d)


def test_a_token_listed_twice():
    for rest in (False, True):
        every(random_distill(3, 4, 700, 9, torch.float32, seed=8, rest=rest, twice=True))


def test_rows_that_start_anywhere():
    for dtype in (torch.bfloat16, torch.float32):
        for V, shift_in, shift_out, pad in ((5003, 0, 0, 5), (5003, 1, 1, 0), (20001, 3, 3, 8), (5003, 1, 2, 1), (20001, 0, 7, 6), (6, 1, 3, 0)):
            d = random_distill(2, 4, V, 5, dtype, seed=V + shift_in, rest=True)
            expected = plain_distill(d)
            (x, t, v), kw = put(d)
            n = 2 * 4 * (V + pad)
            a, b = torch.zeros(n + 64, dtype=dtype, device="cuda"), torch.full((n + 64,), 7.0, dtype=dtype, device="cuda")
            view = lambda z, s: z[s:s + n].view(2, 4, V + pad)
            view(a, shift_in)[:, :, :V] = x
            out = G.Distilled(loss=torch.zeros(2, 4, device="cuda"), stats=torch.zeros(2, 4, 4, device="cuda"), grad=view(b, shift_out)[:, :, :V])
            G.cadd_distill_loss(view(a, shift_in)[:, :, :V], t, v, out=out, **kw)
            check_loss(out.loss, out.stats, d, expected)
            check_grad(out.grad, expected)
            first = out.grad.clone()
            out.grad.fill_(3.0)
            G.cadd_distill_grad(view(a, shift_in)[:, :, :V], t, v, out.stats, grad=out.grad, **kw)
            check_grad(out.grad, expected)
            assert bool((view(b, shift_out)[:, :, V:] == 7.0).all()) and bool((b[:shift_out] == 7.0).all()) and bool((b[shift_out + n:] == 7.0).all())
            assert first.shape == out.grad.shape


def test_axes_in_another_order_and_broadcast_input():
    d = random_distill(3, 4, 4500, 6, torch.bfloat16, seed=8)
    d.logits = d.logits[:1].expand(3, -1, -1).contiguous()
    expected = plain_distill(d)
    (x, t, v), kw = put(d)
    grad = torch.zeros(4, 3, 4500, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    r = G.cadd_distill_loss(x[:1].expand(3, -1, -1), t, v, out=G.Distilled(loss=torch.zeros(3, 4, device="cuda"), grad=grad), **kw)
    check_loss(r.loss, None, d, expected)
    check_grad(r.grad, expected)


def test_rows_left_out_do_not_matter():
    """Weights of zero, rows behind n_rows, lists without a token: zeros, even where the logits are NaN."""
    d = random_distill(3, 6, 9000, 4, torch.bfloat16, seed=2, rest=True)
    d.n_rows = i32([6, 2, 0])
    d.weight[0, 1] = 0.0
    d.teacher_token[0, 3] = -1
    for b, i in ((0, 1), (0, 3), (1, 2), (2, 0)):
        d.logits[b, i] = math.nan
    expected = plain_distill(d)
    r = every(d, expected)
    for b, i in ((0, 1), (0, 3), (1, 2), (2, 0)):
        assert float(r.loss[b, i]) == 0.0 and int(r.grad[b, i].count_nonzero()) == 0 and int(r.stats[b, i].count_nonzero()) == 0
    e = random_distill(1, 2, 500, 4, torch.float32, seed=2)                # no mass in the list
    e.teacher_logit[0, 1] = -math.inf
    r = every(e)
    assert float(r.loss[0, 1]) == 0.0


def test_masked_logits():
    """-Inf in the drafter's row: tokens without probability, listed or not; all but the listed ones; a lowest value as mask."""
    for dtype in (torch.bfloat16, torch.float32):
        d = random_distill(1, 5, 9000, 6, dtype, seed=4, weight=False)
        d.n_rows = None
        tok = d.teacher_token
        d.logits[0, 0, ::2] = -math.inf
        d.logits[0, 0, tok[0, 0].clamp(min=0).long()] = 1.0
        d.logits[0, 1] = torch.finfo(dtype).min
        d.logits[0, 1, tok[0, 1].clamp(min=0).long()] = 0.5
        d.logits[0, 2, 100:] = torch.finfo(dtype).min
        d.logits[0, 2, tok[0, 2].clamp(min=0).long()] = 0.5
        exact = plain_distill(Distill(torch.where(d.logits < -1e30, -math.inf, d.logits.float()).to(dtype), d.teacher_token, d.teacher_logit))
        every(d, exact)
    d = random_distill(1, 3, 3000, 3, torch.float32, seed=4, rest=True, weight=False)
    d.n_rows = None
    d.teacher_token[:] = i32([5, 6, 7])
    d.teacher_logit[0] = torch.log(torch.tensor([0.5, 0.25, 0.125], dtype=torch.float64))
    d.logits[0, 0, 10:] = -math.inf                                        # a rest of seven tokens
    d.logits[0, 1, 5] = -math.inf                                          # a listed token without probability: the loss is infinite
    d.logits[0, 2, :5] = d.logits[0, 2, 8:] = -math.inf                    # no rest
    (x, t, v), kw = put(d)
    r = G.cadd_distill_loss(x, t, v, grad=True, **kw)
    want = plain_distill(d)
    assert abs(float(r.loss[0, 0]) - float(want[0][0, 0])) <= float(want[3][0, 0])
    assert float(r.loss[0, 1]) == math.inf and float(r.loss[0, 2]) == math.inf
    assert bool(torch.isfinite(r.grad).all())
    d.teacher_logit[0, 2] = torch.log(torch.tensor([0.5, 0.25, 0.25 - 2.0 ** -21], dtype=torch.float64))    # a rest that is rounding
    (x, t, v), kw = put(d)
    assert math.isfinite(float(G.cadd_distill_loss(x, t, v, **kw).loss[0, 2]))


def test_what_is_not_finite():
    d = random_distill(1, 6, 9000, 4, torch.float32, seed=3, weight=False)
    d.n_rows = None
    d.logits[0, 0, 4000] = math.nan
    d.logits[0, 1, 4000] = math.inf
    d.logits[0, 2] = -math.inf
    d.logits[0, 3, int(d.teacher_token[0, 3, 0])] = math.nan
    d.teacher_logit[0, 4, 0] = math.nan
    (x, t, v), kw = put(d)
    for rest in (False, True):
        r = G.cadd_distill_loss(x, t, v, grad=True, rest=rest)
        assert torch.isnan(r.loss[0]).tolist() == [True] * 5 + [False]
        assert bool(torch.isnan(r.grad[0, :5]).all()) and not bool(torch.isnan(r.grad[0, 5]).any())
        g = G.cadd_distill_grad(x, t, v, r.stats, rest=rest)
        assert bool(torch.isnan(g[0, :5]).all()) and not bool(torch.isnan(g[0, 5]).any())


def test_large_common_offsets_and_wide_ranges():
    for dtype in (torch.bfloat16, torch.float32):
        d = random_distill(2, 3, 9000, 6, dtype, seed=9, rest=True, sharp=30.0)
        every(d)
        d = random_distill(2, 3, 9000, 6, torch.float32, seed=9, rest=True)
        d.logits += 512.0
        every(d)
    d = random_distill(1, 2, 9000, 6, torch.float32, seed=9, rest=True)    # listed tokens 200 above the rest: a rest of e^-200
    for i in range(2):
        ids = d.teacher_token[0, i]
        d.logits[0, i, ids[ids >= 0].long()] += 200.0
    every(d)


def test_status():
    d = random_distill(5, 4, 300, 3, torch.float32, seed=2, path=True)
    d.path_len = i32([4, -1, 3, 1, 2])
    d.path[2] = i32([3, 9, 1, -1])
    d.path[3, 0], d.path[4, :2] = 2, i32([1, 2])
    d.teacher_token[3, 2, 1] = 300
    d.teacher_token[4, 2, 1] = -5
    d.path[0] = i32([1, 2, 3, 4])
    (x, t, v), kw = put(d)
    r = G.cadd_distill_loss(x, t, v, grad=True, **kw)
    assert r.status.tolist() == [G.STATUS_BAD_LENGTH, G.STATUS_BAD_LENGTH, G.STATUS_BAD_PATH, G.STATUS_BAD_TOKEN, G.STATUS_BAD_TOKEN]
    expected = plain_distill(d)
    check_loss(r.loss, r.stats, d, expected)
    check_grad(r.grad, expected)
    st = torch.full((5,), -1, dtype=torch.int32, device="cuda")
    G.cadd_distill_grad(x, t, v, r.stats, status=st, **kw)
    assert torch.equal(st, r.status)


@pytest.mark.parametrize("V", [60000, 3000])
def test_wait_that_runs_out(V):
    """A copy that is never made: NaN and the status bit, and the next call is right (nothing hangs or faults)."""
    d = random_distill(2, 3, V, 5, torch.bfloat16, seed=2, rest=True)
    d.n_rows = None
    (x, t, v), kw = put(d)
    r = G.cadd_distill_loss(x, t, v, grad=True, flags=G.FLAG_TEST_DROP_TILE, **kw)
    torch.cuda.synchronize()
    assert r.status.tolist() == [G.STATUS_INTERNAL_TIMEOUT] * 2
    assert bool(torch.isnan(r.loss).all()) and bool(torch.isnan(r.grad).all())
    good = every(d)
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    g = G.cadd_distill_grad(x, t, v, good.stats, status=st, flags=G.FLAG_TEST_DROP_TILE, **kw)
    assert st.tolist() == [G.STATUS_INTERNAL_TIMEOUT] * 2 and bool(torch.isnan(g).any())
    every(d)


def test_rows_behind_four_billion_bytes():
    B, L, V = 230, 64, 151936                                              # 2.2 billion elements
    x = torch.zeros(B, L, V, dtype=torch.bfloat16, device="cuda")
    t, v = torch.zeros(B, L, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, L, 1, dtype=torch.float64, device="cuda")
    t[:, :, 0] = torch.arange(B * L, device="cuda").view(B, L) % V
    r = G.cadd_distill_loss(x, t, v, out=G.Distilled(loss=torch.zeros(B, L, device="cuda"), grad=x))
    assert bool(((r.loss - math.log(V)).abs() < 1e-5).all())
    at = t.long()
    assert bool((torch.gather(x, 2, at) == -1.0).all())
    x.scatter_(2, at, 0.0)
    top = x.view(torch.int16).amax(-1)
    assert int(top.min()) == int(top.max()) == int(torch.tensor(1.0 / V).bfloat16().view(torch.int16))


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    a, b = (random_distill(3, 4, 30000, 9, torch.bfloat16, seed=s, rest=True) for s in (1, 2))
    b.n_rows = a.n_rows = None
    (x, t, v), kw = put(a)
    first = G.cadd_distill_loss(x, t, v, grad=True, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    second = G.cadd_distill_loss(x, t, v, grad=True, stream=s, **kw)
    s.synchronize()
    for f in ("loss", "stats", "grad"):
        assert torch.equal(getattr(first, f), getattr(second, f))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.cadd_distill_loss(x, t, v, out=second, **kw)
        alone = G.cadd_distill_grad(x, t, v, second.stats, **kw)
    (x2, t2, v2), kw2 = put(b)
    for dst, src in ((x, x2), (t, t2), (v, v2)):
        dst.copy_(src)
    for k in kw:
        if isinstance(kw[k], torch.Tensor):
            kw[k].copy_(kw2[k])
    graph.replay()
    torch.cuda.synchronize()
    expected = plain_distill(b)
    check_loss(second.loss, second.stats, b, expected)
    check_grad(second.grad, expected)
    check_grad(alone, expected)


def test_a_round_that_teaches_the_drafter():
    """Trees from the drafter's logits; the target's logits under penalties and a grammar; the verdict; the target's own lists of the
    accepted rows; the drafter's gradient, which autograd takes on to hidden states and weight."""
    cfg = synth.scaled(synth.CONFIGS["c2"], batch=4, V=5000, L=8, B_max=24, K=4)
    d, c = synth.make_draft_inputs(cfg, 3), synth.make_cost_inputs(cfg, 3)
    draft = d.logits.cuda()
    tree = G.cadd_build_tree(draft, cfg.K, cfg.B_max, bonus_token=d.bonus_token, cost_coef=c.coef, flags=G.FLAG_FIXED_BUDGET)
    target = synth.make_target_logits(cfg, 3, d, tree.depth.cpu()).cuda()
    B, R, V, L, K = cfg.batch, cfg.R, cfg.V, cfg.L, 6
    g = torch.Generator().manual_seed(1)
    a = Adjust(target.cpu(), n_nodes=tree.n_nodes.cpu(), token_ids=tree.token_ids.cpu(), parent_idx=tree.parent_idx.cpu(),
               history=torch.randint(0, V, (B, 60), generator=g).int(), repetition=torch.full((B,), 1.1), frequency=torch.full((B,), 0.2),
               allowed=pack_bits(torch.rand(3, V, generator=g) < 0.9), allowed_row=torch.randint(-1, 3, (B, R), generator=g).int())
    G.cadd_adjust_logits(target, **a.args("cuda"))
    check_adjust(target, a)
    verdict = G.cadd_verify_tree(target, L, tree.n_nodes, tree.token_ids, tree.parent_idx)
    y = target.float().cpu()
    for b in range(B):
        for j in range(int(tree.n_nodes[b]) + 1):
            assert int(verdict.node_argmax[b, j]) == int(y[b, j].argmax())
    u = torch.rand(B, R, dtype=torch.float64, generator=g).cuda()
    drawn = G.cadd_verify_tree_sampled(target, u, L, tree.n_nodes, tree.token_ids, tree.parent_idx)
    for b in range(B):
        for j in range(int(tree.n_nodes[b]) + 1):
            assert math.isfinite(float(y[b, j, int(drawn.node_argmax[b, j])]))
    lists = G.cadd_build_tree(target.view(B * R, 1, V), K, 0, cost_coef=torch.ones(B * R, 4), flags=G.FLAG_EMIT_TOPK)
    tok, logp = lists.topk_token.view(B, R, K), lists.topk_logprob.view(B, R, K)
    hidden, w = torch.randn(B * L, 16, device="cuda", requires_grad=True), torch.randn(16, V, device="cuda", requires_grad=True)
    logits = (hidden @ w).view(B, L, V)
    kw = dict(rest=True, path=verdict.accepted_nodes, path_len=verdict.accepted_len)
    r = G.cadd_distill_loss(logits.detach(), tok, logp, grad=True, **kw)
    logits.backward(r.grad)
    q = Distill(logits.detach().cpu(), tok.cpu(), logp.cpu(), rest=True, path=verdict.accepted_nodes.cpu(), path_len=verdict.accepted_len.cpu())
    expected = plain_distill(q)
    check_loss(r.loss, r.stats, q, expected)
    check_grad(r.grad, expected)
    assert int(r.status.max()) == 0
    want = r.grad.view(B * L, V).double() @ w.detach().double().t()
    assert torch.allclose(hidden.grad.double(), want, rtol=1e-3, atol=1e-3)
    assert int((r.grad.abs().amax(-1) > 0).sum()) == int((verdict.accepted_len.clamp(max=L - 1) + 1).sum())


def test_refusals_of_the_binding():
    x, t = torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 3, 5, dtype=torch.int32, device="cuda")
    v, s, n = torch.zeros(2, 3, 5, dtype=torch.float64, device="cuda"), torch.zeros(2, 3, 4, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for args, kw in (((x, t.long(), v), {}), ((x, t, v.float()), {}), ((x, t[:1], v), {}), ((x, t, v[:, :, :4]), {}), ((x, t, v), dict(path=t[:, :, 0].contiguous())),
                     ((x, t, v), dict(path_len=n)), ((x, t, v), dict(path=t[:, :, 0].contiguous(), path_len=n, n_rows=n)), ((x, t, v), dict(weight=s[:, :, 0])),
                     ((x, t, v), dict(teacher_lse=v[:, :, 0].contiguous())), ((x, t, v), dict(n_rows=n.cpu())),
                     ((x, t, v), dict(out=G.Distilled(loss=torch.zeros(2, 3, device="cuda"), grad=x.bfloat16())))):
        with pytest.raises(ValueError):
            G.cadd_distill_loss(*args, **kw)
    with pytest.raises(ValueError):
        G.cadd_distill_grad(x, t, v, s[:, :, :2])
    with pytest.raises(TypeError):
        G.cadd_distill_loss(x.half(), t, v)
    for bad, kw in ((t[:, :2].contiguous(), {}), (t, dict(temperature=0.0)), (t, dict(out=G.Distilled()))):
        with pytest.raises(G.CaddError):
            G.cadd_distill_loss(x, bad, torch.zeros(bad.shape, dtype=torch.float64, device="cuda"), **kw)


@pytest.mark.parametrize("rest,T", [(False, 1.0), (True, 1.0), (True, 1.7), (False, 0.5)])
def test_gradient_against_differences(rest, T):
    """Central differences of the plain loss in 64 bits, step h: their error is h^2 / 6 times a third derivative of at most w / T^3 (a
    softmax's is at most 1, and with p_rest / q_rest it has the rest's own softmax besides: 2), and 2^-50 / h of rounding."""
    d = random_distill(2, 3, 40, 6, torch.float32, seed=21, rest=rest, temperature=T, lse=rest)
    (x, t, v), kw = put(d)
    got = G.cadd_distill_loss(x, t, v, grad=True, **kw).grad.double().cpu()
    tol, h, rows = plain_distill(d)[4], 2.0 ** -14, teacher_rows(d)
    for b in range(2):
        for i in range(3):
            r = int(rows[b, i])
            if r < 0:
                assert int(got[b, i].count_nonzero()) == 0
                continue
            f = lambda s: float(row_loss(s, d.teacher_token[b, r], d.teacher_logit[b, r], float(d.teacher_lse[b, r]) if rest else 0.0, rest, T))
            s, w = d.logits[b, i].double(), float(d.weight[b, i]) * float(d.grad_loss[b, i])
            for k in range(40):
                step = torch.zeros(40, dtype=torch.float64)
                step[k] = h
                want = w * (f(s + step) - f(s - step)) / (2 * h)
                assert abs(float(got[b, i, k]) - want) <= float(tol[b, i, k]) + abs(w) * (3 * h * h / (6 * T ** 3) + 2.0 ** -46 / h), (b, i, k)


@pytest.mark.parametrize("B,L,V,path", [(700, 3, 130, False), (3000, 2, 64, True), (1025, 2, 9000, False)])
def test_many_requests_of_few_rows(B, L, V, path):
    """More requests than the map of live rows has groups, some of them without any."""
    d = random_distill(B, L, V, 3, torch.bfloat16, seed=B, rest=True, path=path)
    if not path:
        d.n_rows[100:400] = 0
    every(d)


def test_no_row_is_left():
    d = random_distill(3, 4, 5000, 3, torch.float32, seed=1)
    d.n_rows[:] = 0
    r = every(d)
    assert int(r.grad.count_nonzero()) == 0


def test_calls_on_two_streams_and_graphs_of_both():
    """Calls share nothing: two at once, captured and not, each with its own answers."""
    sets = [random_distill(20, 8, 40000, 16, torch.bfloat16, seed=s, rest=True) for s in (5, 6)]
    args = [put(d) for d in sets]
    alone = [G.cadd_distill_loss(*a, grad=True, **kw) for a, kw in args]
    outs = [G.Distilled(loss=torch.zeros_like(r.loss), stats=torch.zeros_like(r.stats), grad=torch.zeros_like(r.grad)) for r in alone]
    streams, graphs = [torch.cuda.Stream() for _ in args], []
    torch.cuda.synchronize()
    for (a, kw), out in zip(args, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            G.cadd_distill_loss(*a, out=out, **kw)
        graphs.append(g)
    for again in range(3):
        for out in outs:
            out.loss.zero_(), out.grad.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        plain = [G.cadd_distill_loss(*a, grad=True, stream=s, **kw) for (a, kw), s in zip(args, reversed(streams))]
        torch.cuda.synchronize()
        for r, out, p in zip(alone, outs, plain):
            for f in ("loss", "stats", "grad"):
                assert torch.equal(getattr(r, f), getattr(out, f)) and torch.equal(getattr(r, f), getattr(p, f))


def test_listed_tokens_at_every_place():
    """Lists of 256 neighbouring tokens: over the head, the boundaries of chunks, warps and tiles, the tail."""
    V = 2 * 20480 + 37
    d = random_distill(1, 12, V, 256, torch.bfloat16, seed=9, rest=True)
    d.n_rows = None
    starts = [0, 1, 7, 250, 5100, 20480 - 128, 20480 - 255, 20480, 2 * 20480 - 100, V - 256, V - 300, 10000]
    for i, s in enumerate(starts):
        d.teacher_token[0, i] = torch.randperm(256).int() + s
    d.teacher_logit = torch.log_softmax(torch.randn(1, 12, 256, dtype=torch.float64), -1) - 0.1
    every(d)
    (x, t, v), kw = put(d)
    big = torch.zeros(12 * V + 3, dtype=torch.bfloat16, device="cuda")
    y = big[3:].view(1, 12, V)                                             # rows that start anywhere
    y.copy_(x)
    check_grad(G.cadd_distill_loss(y, t, v, grad=True, **kw).grad, plain_distill(d))


def test_lists_over_all_parts_of_rows_in_turn():
    """Several rows a CTA, each with a list in every part of it: what a list leaves in its place is not seen by the row two behind it, and
    all of a row's entries are found, call after call."""
    B, L, V, K = 40, 9, 60000, 256
    d = random_distill(B, L, V, K, torch.bfloat16, seed=31, rest=True)
    d.n_rows = None
    g = torch.Generator().manual_seed(31)
    d.teacher_token = (torch.arange(K) * (V // K) + torch.randint(0, V // K, (B, L, K), generator=g)).int()
    d.teacher_logit = torch.log_softmax(torch.randn(B, L, K, generator=g, dtype=torch.float64), -1) - 0.2
    first = every(d)
    (x, t, v), kw = put(d)
    for _ in range(20):
        r = G.cadd_distill_loss(x, t, v, grad=True, **kw)
        for f in ("loss", "stats", "grad"):
            assert torch.equal(getattr(r, f), getattr(first, f))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("equal", [False, True])
def test_sums_of_few_large_terms(dtype, equal):
    """Rows of which one token beside the list, or equal ones, make up the sum: nothing averages out.  The argument of the exponential of a large
    term is at most 4 in magnitude, in log2 units, so that its rounding is off by 2^-23 at most (ln 2 of that relative); ex2 by 2^-22; the factor that
    centres ex2, the statistics' fp32 and two roundings of a sum of up to eight equal terms by 2^-24 each."""
    tol = math.log(2.0) * 2.0 ** -23 + 2.0 ** -22 + 4 * 2.0 ** -24
    B, L, V = 30, 8, 4096 if equal else 45056
    g = torch.Generator().manual_seed(17)
    top = (6 * torch.randn(B, L, 1, generator=g)).to(dtype)
    if equal:
        x = top.expand(-1, -1, V).clone()
    else:                                                                  # and one below it that its thread meets first
        x = ((torch.randn(B, L, V, generator=g) - 60.0).to(dtype) + top).to(dtype)
        x[:, :, 1234], x[:, :, 1234 + 20480] = top[:, :, 0] - 2.5, top[:, :, 0]
    t, v = torch.zeros(B, L, 1, dtype=torch.int32), torch.full((B, L, 1), math.log(0.25), dtype=torch.float64)
    x[:, :, 0] = top[:, :, 0] - 8
    for T in (1.0, 0.7):
        r = G.cadd_distill_loss(x.cuda(), t.cuda(), v.cuda(), rest=True, temperature=T)
        z, m = x[..., 1:].double(), top.double()
        want = torch.exp((z - m) / T).sum(-1)
        assert torch.equal(r.stats[..., 2].cpu(), top[..., 0].float())
        err = (r.stats[..., 3].double().cpu() / want - 1.0).abs()
        assert float(err.max()) <= tol, float(err.max())
        logq = torch.log_softmax(x.double() / T, -1)
        p = 0.25 ** (1.0 / T)                                              # (the target's entries are logits, too)
        loss = p * (math.log(p) - logq[..., 0]) + (1.0 - p) * (math.log(1.0 - p) - torch.logsumexp(logq[..., 1:], -1))
        assert bool(((r.loss.double().cpu() - loss).abs() <= 2 * tol + 2.0 ** -24 * loss.abs()).all())


@pytest.mark.parametrize("rest", [False, True])
def test_a_path_without_columns(rest):
    """Accepted nodes cut to the longest accepted length, of a batch in which nothing was accepted: only the first position is learnt from."""
    for L in (1, 5):
        d = random_distill(3, L, 2000, 6, torch.float32, seed=19, rest=rest, path=True)
        d.path, d.path_len = d.path[:, :0].contiguous(), i32([0, 0, 0])
        assert d.teacher_token.shape[1] >= L                               # (rows of lists for all positions are there)
        r = every(d)
        assert r.status.tolist() == [0, 0, 0] and int(r.loss[:, 1:].count_nonzero()) == 0 and int(r.grad[:, 1:].count_nonzero()) == 0
        assert int((r.loss[:, 0] != 0).sum()) == 3
    d.teacher_token, d.teacher_logit = d.teacher_token[:, :2].contiguous(), d.teacher_logit[:, :2].contiguous()      # fewer rows than positions
    every(d)


@pytest.mark.parametrize("V", [60000, 3000])
def test_gradient_alone_when_a_wait_runs_out(V):
    """All of its rows are lost."""
    d = random_distill(2, 3, V, 5, torch.bfloat16, seed=2, rest=True)
    d.n_rows = None
    (x, t, v), kw = put(d)
    stats, st = G.cadd_distill_loss(x, t, v, **kw).stats, torch.zeros(2, dtype=torch.int32, device="cuda")
    g = G.cadd_distill_grad(x, t, v, stats, status=st, flags=G.FLAG_TEST_DROP_TILE, grad=torch.zeros_like(x), **kw)
    assert st.tolist() == [G.STATUS_INTERNAL_TIMEOUT] * 2 and bool(torch.isnan(g).all())


def test_lists_of_the_accepted_rows_alone():
    """The target's rows along the accepted path gathered first, and their lists made: the same tokens as in the lists of all rows by the path (log-probabilities
    differ in how a row's sum was cut), and the loss and gradient that they stand for."""
    batch, R, L, V, K = 5, 17, 6, 4001, 7
    g = torch.Generator().manual_seed(23)
    target, draft = torch.randn(batch, R, V, generator=g).cuda(), torch.randn(batch, L, V, generator=g).cuda().requires_grad_(True)
    nodes, lens = torch.full((batch, L), -1, dtype=torch.int32, device="cuda"), i32([0, 1, 4, 6, 5]).cuda()
    for b, n in enumerate(lens.tolist()):
        nodes[b, :n] = torch.randperm(R - 1, generator=g)[:n].sort().values.int().cuda() + 1
    rows = torch.cat([nodes.new_zeros(batch, 1), nodes[:, :L - 1].clamp(min=0)], 1).long()
    accepted = target[torch.arange(batch, device=rows.device)[:, None], rows]
    lists = G.cadd_build_tree(accepted.view(batch * L, 1, V), K, 0, cost_coef=torch.ones(batch * L, 4), flags=G.FLAG_EMIT_TOPK)
    tok, logp, n_rows = lists.topk_token.view(batch, L, K), lists.topk_logprob.view(batch, L, K), (lens + 1).clamp(max=L)
    d = G.cadd_distill_loss(draft.detach(), tok, logp, rest=True, n_rows=n_rows, grad=True)
    q = Distill(draft.detach().cpu(), tok.cpu(), logp.cpu(), rest=True, n_rows=n_rows.cpu())
    expected = plain_distill(q)
    check_loss(d.loss, d.stats, q, expected)
    check_grad(d.grad, expected)
    assert d.status.tolist() == [0] * batch and int((d.loss != 0).sum()) == int(n_rows.sum())
    draft.backward(d.grad)
    assert torch.equal(draft.grad, d.grad)
    every_row = G.cadd_build_tree(target.view(batch * R, 1, V), K, 0, cost_coef=torch.ones(batch * R, 4), flags=G.FLAG_EMIT_TOPK)
    all_tok, all_logp = every_row.topk_token.view(batch, R, K), every_row.topk_logprob.view(batch, R, K)
    assert torch.equal(torch.gather(all_tok, 1, rows[..., None].expand(-1, -1, K)), tok)
    by_path = G.cadd_distill_loss(draft.detach(), all_tok, all_logp, rest=True, path=nodes, path_len=lens, grad=True)
    check_grad(by_path.grad, plain_distill(Distill(draft.detach().cpu(), all_tok.cpu(), all_logp.cpu(), rest=True, path=nodes.cpu(), path_len=lens.cpu())))
    assert torch.equal(by_path.loss != 0, d.loss != 0)
