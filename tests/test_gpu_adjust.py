"""cadd_adjust_logits against its definition in 64 bits (logits_util), at the sizes, layouts and masks where it can go wrong."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from logits_util import Adjust, check_adjust, pack_bits, plain_adjust, random_adjust

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(x, dtype=torch.int32)


def both(a: Adjust):
    """The call into another array (rows that are not live keep what it held) and in place: the same bits."""
    want = plain_adjust(a)
    x, kw = a.logits.cuda(), a.args("cuda")
    out = x.clone()
    assert G.cadd_adjust_logits(x, out=out, **kw) is out
    check_adjust(out, a, want)
    assert torch.equal(x.cpu().view(torch.uint8), a.logits.view(torch.uint8))
    assert G.cadd_adjust_logits(x, **kw) is x
    assert torch.equal(x.view(torch.uint8), out.view(torch.uint8))
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V", [(1, 1, 1), (2, 3, 7), (1, 1, 4096), (3, 5, 4097), (2, 33, 1000), (1, 70, 12289), (5, 1, 32001), (2, 9, 8200)])
def test_sizes(dtype, B, R, V):
    both(random_adjust(B, R, V, dtype, seed=B + R + V, tree=R > 1))


@pytest.mark.parametrize("part", ["masks", "penalties", "n_bias", "history", "tree"])
@pytest.mark.parametrize("alone", [False, True])
def test_each_part_alone_and_left_out(part, alone):
    every = ("masks", "penalties", "n_bias", "history", "tree")
    kw = {p: (p == part) == alone for p in every}
    if alone and part in ("history", "tree"):
        kw["penalties"] = True
    kw["n_bias"], kw["history"] = 9 * kw["n_bias"], 40 * kw["history"]
    both(random_adjust(2, 6, 5000, torch.bfloat16, seed=3, **kw))


@pytest.mark.parametrize("which", ["repetition", "presence", "frequency"])
def test_one_penalty_alone(which):
    a = random_adjust(2, 6, 300, torch.float32, seed=4, n_bias=0, masks=False)
    for k in ("repetition", "presence", "frequency"):
        if k != which:
            setattr(a, k, None)
    both(a)


def test_nothing_to_do():
    a = Adjust(torch.randn(2, 3, 5000).bfloat16())
    both(a)
    a = random_adjust(2, 3, 500, torch.float32, seed=1, history=0, tree=False, n_bias=0, masks=False)     # penalties without anything to count
    both(a)


def test_rows_that_start_anywhere():
    for dtype in (torch.bfloat16, torch.float32):
        for shift_in, shift_out, pad in ((0, 0, 5), (1, 1, 3), (3, 3, 8), (1, 2, 1), (0, 7, 6)):
            a = random_adjust(2, 4, 5003, dtype, seed=shift_in + pad)
            V = a.logits.shape[2]
            big = torch.zeros(2 * 4 * (V + pad) + 64, dtype=dtype, device="cuda")
            x = big[shift_in:shift_in + 2 * 4 * (V + pad)].view(2, 4, V + pad)[:, :, :V]
            x.copy_(a.logits)
            big2 = torch.full_like(big, 7.0)
            out = big2[shift_out:shift_out + 2 * 4 * (V + pad)].view(2, 4, V + pad)[:, :, :V]
            out.copy_(a.logits)
            G.cadd_adjust_logits(x, out=out, **a.args("cuda"))
            check_adjust(out, a)
            rest = big2[shift_out:shift_out + 2 * 4 * (V + pad)].view(2, 4, V + pad)[:, :, V:]
            assert bool((rest == 7.0).all()) and bool((big2[:shift_out] == 7.0).all())
            kept = big.clone()
            G.cadd_adjust_logits(x, **a.args("cuda"))
            assert torch.equal(x, out)
            x.copy_(kept[shift_in:shift_in + 2 * 4 * (V + pad)].view(2, 4, V + pad)[:, :, :V])
            assert torch.equal(big, kept)


def test_axes_in_another_order_and_broadcast_input():
    a = random_adjust(3, 4, 4500, torch.bfloat16, seed=8)
    x = a.logits.cuda().transpose(0, 1).contiguous().transpose(0, 1)           # [R, batch, V] in memory
    out = torch.zeros(4, 3, 4500, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    out.copy_(x)
    G.cadd_adjust_logits(x, out=out, **a.args("cuda"))
    check_adjust(out, a)
    G.cadd_adjust_logits(x, **a.args("cuda"))
    assert torch.equal(x, out)
    a.logits = a.logits[:1].expand(3, -1, -1)                                  # every request from the same logits
    x = a.logits[:1].cuda().expand(3, -1, -1)
    out = x.clone()
    G.cadd_adjust_logits(x, out=out, **a.args("cuda"))
    a.logits = a.logits.contiguous()
    check_adjust(out, a)
    with pytest.raises(G.CaddError) as e:                                      # in place there: rows that lie in one another
        G.cadd_adjust_logits(x, **a.args("cuda"))
    assert e.value.code == G.ERR_SHAPE


def test_histories_of_every_length():
    for n in (1, 255, 256, 257, 5000):
        a = random_adjust(4, 2, 600, torch.float32, seed=n, history=n, tree=False, masks=False)
        a.history_len[1], a.prompt_len[1] = 0, 0
        a.prompt_len[2] = a.history_len[2]
        both(a)
        a.history_len = a.prompt_len = None                                    # all of it was said
        both(a)
    wide = random_adjust(2, 2, 600, torch.float32, seed=5, history=40)
    big = torch.full((2, 100), 3, dtype=torch.int32)
    big[:, :40] = wide.history
    wide.history = big[:, :40]                                                 # rows apart
    want = plain_adjust(wide)
    x = wide.logits.cuda()
    kw = wide.args("cuda")
    kw["history"] = big.cuda()[:, :40]
    check_adjust(G.cadd_adjust_logits(x, **kw), wide, want)


def test_tokens_out_of_range_have_no_effect():
    a = random_adjust(2, 6, 100, torch.float32, seed=9, spread=100)
    a.history[:, ::3] = i32([-1, 100, 2 ** 31 - 1, -2 ** 31, 4096, 105])[torch.arange(17) % 6]
    a.token_ids[:, 2] = -1
    a.token_ids[:, 3] = 100
    a.bias_token[0, :4] = i32([-1, 100, 2 ** 31 - 1, -7])
    both(a)


def test_the_same_token_in_every_list():
    for V in (50, 9000):
        a = random_adjust(3, 12, V, torch.float32, seed=V, spread=3, n_bias=64, history=300)
        both(a)
    a = random_adjust(1, 3, 9000, torch.float32, seed=2, spread=9000, n_bias=6000, history=0, masks=False, tree=False)
    both(a)                                                                    # more biases than a tile has tokens


def test_the_same_inputs_give_the_same_bits():
    a = random_adjust(2, 40, 9000, torch.float32, seed=2, spread=30, n_bias=500, history=3000)
    x, kw = a.logits.cuda(), a.args("cuda")
    first = G.cadd_adjust_logits(x, out=x.clone(), **kw)
    for _ in range(5):
        assert torch.equal(G.cadd_adjust_logits(x, out=x.clone(), **kw), first)


def test_masks():
    V = 4100
    for dtype in (torch.bfloat16, torch.float32):
        a = random_adjust(2, 5, V, dtype, seed=6, masks=False, dead=False)
        m = torch.zeros(6, V, dtype=torch.bool)
        m[1, V - 1] = True
        m[2, 0] = True
        m[3] = True
        m[4, ::2] = True
        m[5, 4000:] = True
        a.allowed, a.allowed_row = pack_bits(m), i32([[0, 1, 2, 3, 4], [5, -1, 1, 1, 0]])
        out = both(a)
        assert bool((out[0, 0] == -math.inf).all())
        st = torch.full((2,), -1, dtype=torch.int32, device="cuda")
        G.cadd_adjust_logits(a.logits.cuda(), status=st, **a.args("cuda"))
        assert st.tolist() == [G.STATUS_NOTHING_ALLOWED, G.STATUS_NOTHING_ALLOWED]
        a.allowed[:, -1] |= -1 << (V % 32)                                     # bits behind the vocabulary mean nothing
        both(a)
        G.cadd_adjust_logits(a.logits.cuda(), status=st, **a.args("cuda"))
        assert st.tolist() == [G.STATUS_NOTHING_ALLOWED, G.STATUS_NOTHING_ALLOWED]


def test_what_is_not_finite():
    a = random_adjust(2, 6, 4200, torch.float32, seed=12, spread=40, n_bias=30)
    inf = math.inf
    for v in range(60):
        a.logits[:, :, v] = [math.nan, inf, -inf, -0.0, 0.0, 3.4e38, -3.4e38, 1e-42][v % 8]
    a.logits[:, :, -9:] = math.nan
    a.bias[0, :3] = torch.tensor([inf, -inf, math.nan])
    both(a)
    b = random_adjust(2, 6, 4200, torch.bfloat16, seed=12, spread=40, n_bias=30)
    b.logits[:, :, :16] = torch.tensor([math.nan, inf, -inf, -0.0] * 4).bfloat16()
    both(b)


def test_status():
    a = random_adjust(6, 80, 50, torch.float32, seed=1, n_bias=0, dead=False, masks=False)
    n = 80
    a.parent_idx[1] = torch.arange(-1, n - 1)                                  # a chain: 64 nodes above a node are followed
    a.parent_idx[2, 5] = 5
    a.parent_idx[2, 6] = 70
    a.history_len[3] = 51
    a.history_len[4], a.prompt_len[4] = 10, 11
    a.n_nodes[5] = 80
    a.allowed, a.allowed_row = pack_bits(torch.ones(2, 50, dtype=torch.bool)), torch.full((6, n), -1, dtype=torch.int32)
    a.allowed_row[0, 3] = 2
    a.allowed_row[1, 3] = -2
    st = torch.full((6,), -1, dtype=torch.int32, device="cuda")
    x = a.logits.cuda()
    out = G.cadd_adjust_logits(x, out=x.clone(), status=st, **a.args("cuda"))
    check_adjust(out, a)
    assert st.tolist() == [G.STATUS_BAD_MASK, G.STATUS_BAD_MASK | G.STATUS_BAD_PATH, G.STATUS_BAD_PATH, G.STATUS_BAD_LENGTH, G.STATUS_BAD_LENGTH, G.STATUS_BAD_N_NODES]
    a = random_adjust(2, 8, 50, torch.float32, seed=1, masks=False)
    G.cadd_adjust_logits(a.logits.cuda(), status=st[:2], **a.args("cuda"))
    assert st[:2].tolist() == [0, 0]


def test_rows_and_requests_behind_four_billion_bytes():
    """In place on 2.6 billion elements: the last request's rows, and no other."""
    B, R, V = 17, 1000, 151936
    x = torch.zeros(B, R, V, dtype=torch.bfloat16, device="cuda")
    rows = torch.full((B, R), -1, dtype=torch.int32, device="cuda")
    rows[16, 999] = rows[15, 0] = 0
    bits = torch.full((1, V // 32), 1 << 5, dtype=torch.int32, device="cuda")
    n = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    n[15:] = R - 1
    hist = torch.full((B, 2), V - 1, dtype=torch.int32, device="cuda")
    G.cadd_adjust_logits(x, n_nodes=n, allowed=bits, allowed_row=rows, history=hist, presence=torch.full((B,), 2.0, device="cuda"))
    keep = torch.arange(V, device="cuda") % 32 == 5
    for b, j in ((16, 999), (15, 0)):
        want = torch.where(keep, 0.0, -math.inf)
        assert torch.equal(x[b, j].float(), want)
        x[b, j] = 0
    assert bool((x[15:, :, V - 1] == -2.0).sum() == 2 * R - 2)
    x[15:, :, V - 1] = 0
    assert int(x.view(torch.int16).count_nonzero()) == 0


def test_other_stream_and_graph():
    a, b = random_adjust(2, 9, 9000, torch.bfloat16, seed=1), random_adjust(2, 9, 9000, torch.bfloat16, seed=2)
    x, kw, out = a.logits.cuda(), a.args("cuda"), torch.zeros(2, 9, 9000, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out.copy_(x)
    s.wait_stream(torch.cuda.current_stream())
    G.cadd_adjust_logits(x, out=out, stream=s, **kw)
    s.synchronize()
    check_adjust(out, a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.cadd_adjust_logits(x, out=out, **kw)
    x.copy_(b.logits.cuda())
    for k, v in b.args("cuda").items():
        kw[k].copy_(v)
    out.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    check_adjust(out, b)


def test_refusals_of_the_binding():
    x, t = torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    f = torch.ones(2, device="cuda")
    for kw in (dict(token_ids=t), dict(history=t.long(), presence=f), dict(history_len=t[:, 0].contiguous()), dict(bias=x[:, :, 0]), dict(allowed=t), dict(repetition=f.double()),
               dict(repetition=torch.ones(3, device="cuda")), dict(n_nodes=torch.zeros(2, dtype=torch.int32)), dict(out=x.bfloat16()), dict(out=x[:, :2]),
               dict(allowed=t[:, :1], allowed_row=t), dict(history=t.t(), presence=f)):
        with pytest.raises(ValueError):
            G.cadd_adjust_logits(x, **kw)
    with pytest.raises(ValueError):
        G.cadd_adjust_logits(x[:, :, ::2])
    with pytest.raises(TypeError):
        G.cadd_adjust_logits(x.half())


def test_wait_that_runs_out():
    """Copies that are never made: NaN and the status bit, and the next call is right (nothing hangs or faults)."""
    a = random_adjust(2, 9, 9000, torch.bfloat16, seed=5, dead=False)
    x, st, kw = a.logits.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda"), a.args("cuda")
    out = G.cadd_adjust_logits(x, out=torch.zeros_like(x), status=st, flags=G.FLAG_TEST_DROP_TILE, **kw)
    torch.cuda.synchronize()
    assert st.tolist() == [G.STATUS_INTERNAL_TIMEOUT] * 2 and bool(torch.isnan(out).all())
    both(a)
    out = G.cadd_adjust_logits(x, out=torch.zeros_like(x), status=st, flags=G.FLAG_TEST_DROP_TILE, allowed=kw["allowed"], allowed_row=kw["allowed_row"])
    torch.cuda.synchronize()
    assert st.tolist() == [G.STATUS_INTERNAL_TIMEOUT] * 2 and bool(torch.isnan(out).all())


@pytest.mark.parametrize("V,history", [(4097, 1025), (40000, 3000), (2048 * 9, 5000), (30000, 14000), (9000, 40000)])
@pytest.mark.parametrize("R", [3, 10])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_histories_of_many_tokens(V, history, R, dtype):
    """Into another array and in place; beyond 12288 tokens several CTAs share a request's."""
    both(random_adjust(2, R, V, dtype, seed=V, history=history, spread=V, n_bias=20))


def test_wait_that_runs_out_with_more_pieces_to_come():
    """A warp whose copy never comes loses the pieces it would have taken after it, too: no request is left as it was without its bit."""
    B, V = 100, 40 * 4096                                                      # 4000 pieces for 3552 warps
    x, st = torch.zeros(B, 1, V, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    out = G.cadd_adjust_logits(x, out=torch.zeros_like(x), status=st, flags=G.FLAG_TEST_DROP_TILE)
    torch.cuda.synchronize()
    assert bool((st == G.STATUS_INTERNAL_TIMEOUT).all()) and bool(torch.isnan(out).all())
    assert torch.equal(G.cadd_adjust_logits(x, out=out, status=st), x) and not bool(st.any())


@pytest.mark.parametrize("n_bias,spread", [(31, 1), (33, 2), (1024, 3), (4096, 2000), (65536, 65536), (65536, 20000)])
@pytest.mark.parametrize("R", [1, 8])
def test_biases_listed_many_times(n_bias, spread, R):
    both(random_adjust(1, R, 70000, torch.float32, seed=n_bias + R, spread=spread, n_bias=n_bias, history=20, masks=False))


def test_unused_biases_filled_with_one_token():
    """Lists padded with a token and nothing to add, as well as with none."""
    a = random_adjust(2, 9, 9000, torch.float32, seed=4, n_bias=300)
    a.bias_token[:, 100:], a.bias[:, 100:] = 17, 0.0
    a.bias_token[1, 50:], a.bias[1, 50:] = -1, math.nan
    both(a)
    a.bias_token[0, :3], a.bias[0, :3] = 17, torch.tensor([1e8, -1e8, 1.0])      # a sum that 32 bits would lose on the way
    both(a)


@pytest.mark.parametrize("R,batch", [(1, 2), (1, 40), (2, 90), (9, 3), (65, 2)])
def test_calls_on_two_streams_and_graphs_of_both(R, batch):
    """Calls share nothing: two at once, captured and not, into other arrays and in place."""
    sets = [random_adjust(batch, R, 30000, torch.bfloat16, seed=s, history=500, tree=R > 1) for s in (3, 4)]
    xs, kws = [a.logits.cuda() for a in sets], [a.args("cuda") for a in sets]
    alone = [G.cadd_adjust_logits(x, out=x.clone(), **kw) for x, kw in zip(xs, kws)]
    outs, placed, streams, graphs = [x.clone() for x in xs], [x.clone() for x in xs], [torch.cuda.Stream() for _ in xs], []
    torch.cuda.synchronize()
    for x, kw, out, y in zip(xs, kws, outs, placed):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            G.cadd_adjust_logits(x, out=out, **kw)
            y.copy_(x)
            G.cadd_adjust_logits(y, **kw)
        graphs.append(g)
    for again in range(3):
        for out, x in zip(outs, xs):
            out.copy_(x)
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for r, out, y in zip(alone, outs, placed):
            assert torch.equal(r, out) and torch.equal(r, y)


def test_results_are_there_for_the_next_kernel():
    """What reads the rows next on the stream reads them as they are when the call is done, with and without live rows."""
    for batch, live in ((64, 0), (64, -1)):
        x = torch.zeros(batch, 1, 151936, dtype=torch.bfloat16, device="cuda")
        n = torch.full((batch,), live, dtype=torch.int32, device="cuda")
        n[0] = 0
        hist = torch.arange(1000, dtype=torch.int32, device="cuda").repeat(batch, 1)
        kw = dict(history=hist, presence=torch.full((batch,), 2.0, device="cuda"), n_nodes=n)
        for _ in range(20):
            out = torch.full_like(x, 1.0)
            total = G.cadd_adjust_logits(x, out=out, **kw).float().sum(-1)[:, 0]
            assert total.tolist() == [-2000.0 if live == 0 or b == 0 else 151936.0 for b in range(batch)]


def test_many_rows():
    """As many rows as a call can have: a tree whose nodes all follow the root."""
    R, V = 65536, 40
    a = Adjust(torch.randn(1, R, V).bfloat16(), token_ids=(torch.arange(R) % 50).int()[None], parent_idx=torch.zeros(1, R, dtype=torch.int32),
               presence=torch.ones(1), history=i32([[3, 3, 7]]), bias_token=i32([[5]]), bias=torch.tensor([[0.5]]))
    a.parent_idx[0, 0] = -1
    x = a.logits.double()
    for t, n in ((0, 1), (3, 1), (7, 1)):
        x[0, :, t] -= n
    at = torch.arange(R)
    own = (at % 50 < V) & (at > 0)
    for t in (0, 3, 7):
        own &= at % 50 != t
    x[0, at[own], (at % 50)[own]] -= 1
    x[0, :, 5] += 0.5
    y = a.logits.cuda()
    assert torch.equal(G.cadd_adjust_logits(y, out=torch.zeros_like(y), **a.args("cuda")).cpu(), x.bfloat16())
    assert torch.equal(G.cadd_adjust_logits(y, **a.args("cuda")).cpu(), x.bfloat16())


@pytest.mark.parametrize("B,R,V,dtype,history,n_bias", [(40, 1, 70001, torch.bfloat16, 50, 7), (40, 3, 70000, torch.bfloat16, 3000, 40), (70, 2, 20000, torch.float32, 14000, 20),
                                                        (30, 3, 65000, torch.float32, 500, 0), (700, 1, 5000, torch.float32, 5, 3)])
@pytest.mark.parametrize("masks", [False, True])
def test_few_rows_of_many_requests(B, R, V, dtype, history, n_bias, masks):
    """More tiles than the device has room for at once: copied and masked first, then token by token."""
    both(random_adjust(B, R, V, dtype, seed=B + R, history=history, n_bias=n_bias, tree=R > 1, masks=masks, spread=V if history > 1000 else None))


def test_many_rows_in_place_with_few_tokens():
    both(random_adjust(40, 25, 40000, torch.bfloat16, seed=2, history=50, masks=False))


@pytest.mark.parametrize("R", [1, 5])
def test_a_history_of_more_uses_than_a_word_counts(R):
    a = random_adjust(1, R, 6000, torch.float32, seed=R, history=600000, spread=6000, tree=R > 1)
    a.history[:, 100000:] = 7                                                  # half a million uses of one token
    a.prompt_len[0] = 1000
    both(a)


def test_one_history_for_all_requests():
    a = random_adjust(5, 3, 9000, torch.bfloat16, seed=6, history=300)
    a.history = a.history[:1].expand(5, -1)
    want = plain_adjust(a)
    kw = a.args("cuda")
    kw["history"] = kw["history"][:1].expand(5, -1)
    assert kw["history"].stride(0) == 0
    x = a.logits.cuda()
    check_adjust(G.cadd_adjust_logits(x, out=x.clone(), **kw), a, want)


def test_wait_that_runs_out_before_single_tokens():
    """Rows whose copies never come hold NaN but where single tokens are replaced afterwards, and every request has its bit."""
    a = random_adjust(50, 1, 70000, torch.bfloat16, seed=7, tree=False, dead=False, history=40, masks=False)
    x, st, kw = a.logits.cuda(), torch.zeros(50, dtype=torch.int32, device="cuda"), a.args("cuda")
    out = G.cadd_adjust_logits(x, out=torch.zeros_like(x), status=st, flags=G.FLAG_TEST_DROP_TILE, **kw)
    torch.cuda.synchronize()
    assert bool((st == G.STATUS_INTERNAL_TIMEOUT).all())
    _, touched, _ = plain_adjust(a)
    assert bool(torch.isnan(out.cpu()[~touched]).all())
    both(a)
