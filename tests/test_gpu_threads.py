"""Calls from several host threads at once, each on a stream of its own: a large call and a small one of the same kernel.  Kernels' limits of shared memory
belong to the process, so no call may set one by its own size."""
import threading

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from paper_2606_01813_b200 import synth
from logits_util import random_adjust, random_distill

pytestmark = pytest.mark.gpu
CALLS = 1500


def together(*calls):
    """Each call CALLS times in a thread and on a stream of its own; returns what the last ones gave."""
    failed, results, start = [], [None] * len(calls), threading.Barrier(len(calls))

    def work(k):
        s = torch.cuda.Stream()
        start.wait()
        try:
            for _ in range(CALLS):
                results[k] = calls[k](s)
        except Exception as e:                                                # noqa: BLE001 (told to the test)
            failed.append(e)
        s.synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed[:2]
    return results


def distill_call(V, K, grad):
    d = random_distill(1, 2, V, K, torch.bfloat16, seed=V, rest=True)
    x, t, v, kw = d.logits.cuda(), d.teacher_token.cuda(), d.teacher_logit.cuda(), d.args("cuda")
    want = G.cadd_distill_loss(x, t, v, grad=grad, **kw)
    out = G.Distilled(*(None if y is None else torch.zeros_like(y) for y in (want.loss, want.stats, want.grad, want.status)))
    return lambda s: G.cadd_distill_loss(x, t, v, out=out, stream=s, **kw), want


@pytest.mark.parametrize("grad", [False, True])
def test_distillation(grad):
    (large, a), (small, b) = distill_call(150000, 256, grad), distill_call(500, 1, grad)
    torch.cuda.synchronize()
    for r, want in zip(together(large, small), (a, b)):
        assert torch.equal(r.loss, want.loss) and torch.equal(r.stats, want.stats) and (not grad or torch.equal(r.grad, want.grad))


def adjust_call(history, n_bias, R, batch, V):
    a = random_adjust(batch, R, V, torch.bfloat16, seed=history, history=history, n_bias=n_bias, tree=False, masks=False, dead=False)
    x, kw = a.logits.cuda(), a.args("cuda")
    want, out = G.cadd_adjust_logits(x, out=torch.zeros_like(x), **kw), torch.zeros_like(x)
    return lambda s: G.cadd_adjust_logits(x, out=out, stream=s, **kw), want


@pytest.mark.parametrize("R,batch,V", [(1, 64, 50000), (9, 2, 9000)])          # by single tokens, by tables
def test_adjustment(R, batch, V):
    (large, a), (small, b) = adjust_call(9000, 5000, R, batch, V), adjust_call(10, 0, R, batch, V)
    torch.cuda.synchronize()
    for r, want in zip(together(large, small), (a, b)):
        assert torch.equal(r, want)


def build_call(L, K, B_max):
    """The C call alone, so that threads are in it most of the time."""
    cfg = synth.scaled(synth.CONFIGS["c2"], batch=2, V=2000, L=L, B_max=B_max, K=K)
    x, coef = synth.make_draft_inputs(cfg, 3).logits.cuda(), synth.make_cost_inputs(cfg, 3).coef.double().cuda().contiguous()
    call, given = G.lib().cadd_build_tree, []
    want, out = (G.cadd_build_tree(x, K, B_max, cost_coef=coef) for _ in range(2))
    ws = torch.empty(G.cadd_build_workspace_bytes(2, L, 2000, K, B_max, B_max + 1, x.dtype), dtype=torch.uint8, device="cuda")
    G.lib().cadd_build_tree = lambda args, stream: given.append(args) or call(args, stream)
    try:
        G.cadd_build_tree(x, K, B_max, cost_coef=coef, out=out, workspace=ws)
    finally:
        G.lib().cadd_build_tree = call
    assert given[0]._obj.cost_coef == coef.data_ptr()

    def again(s):
        for _ in range(5):
            if call(given[0], s.cuda_stream) != G.OK:
                raise G.CaddError(G.ERR_LAUNCH)
        return x, coef, ws, out
    return again, want


def test_construction():
    calls = [build_call(32, 32, b) for b in (2048, 1400, 2048, 1400)]
    torch.cuda.synchronize()
    for (*_, r), (_, want) in zip(together(*(c for c, _ in calls)), calls):
        assert torch.equal(r.token_ids, want.token_ids) and torch.equal(r.parent_idx, want.parent_idx) and torch.equal(r.n_nodes, want.n_nodes)
