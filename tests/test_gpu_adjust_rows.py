"""Rows of cadd_adjust_logits that are not live, and what lies between rows: other arrays keep exactly what they held, whichever kernels take the call."""
import pytest
import torch

from paper_2606_01813_b200 import binding as G
from logits_util import check_adjust, plain_adjust, random_adjust

pytestmark = pytest.mark.gpu
HELD = 768.0                                                                  # what the arrays hold before: no logit of these problems


def problem(B, R, V, dtype, history, n_bias, masks, penalties, seed):
    a = random_adjust(B, R, V, dtype, seed=seed, history=history, n_bias=n_bias, masks=masks, penalties=penalties, tree=R > 1)
    a.n_nodes[0] = -1                                                         # a request without a live row
    if B > 2:
        a.n_nodes[1] = (R - 1) // 2
    live = torch.arange(R) <= a.n_nodes[:, None]
    assert bool((a.logits != HELD).all()) and bool(live.any()) and not bool(live.all())
    return a, live


@pytest.mark.parametrize("B,R,V,dtype,history,n_bias,masks,penalties", [
    (3, 33, 9001, torch.bfloat16, 60, 9, True, True), (3, 40, 4100, torch.float32, 300, 0, False, True),      # by tables
    (40, 1, 70001, torch.bfloat16, 50, 7, True, True), (40, 3, 70000, torch.float32, 40, 0, False, True),     # copied, then token by token
    (5, 7, 20011, torch.bfloat16, 0, 0, True, False), (3, 6, 5003, torch.float32, 0, 0, False, False)])       # masks alone, and nothing at all
@pytest.mark.parametrize("shift_in,shift_out,pad", [(0, 0, 0), (1, 1, 3), (3, 2, 8)])
def test_rows_that_are_not_live_keep_what_they_held(B, R, V, dtype, history, n_bias, masks, penalties, shift_in, shift_out, pad):
    a, live = problem(B, R, V, dtype, history, n_bias, masks, penalties, seed=V + pad)
    want, kw, n = plain_adjust(a), a.args("cuda"), B * R * (V + pad)
    area = lambda fill: torch.full((n + 64,), fill, dtype=dtype, device="cuda")
    view = lambda z, s: z[s:s + n].view(B, R, V + pad)
    src, dst = area(5.0), area(HELD)
    x, out = view(src, shift_in)[:, :, :V], view(dst, shift_out)[:, :, :V]
    x.copy_(a.logits)
    given = src.clone()
    G.cadd_adjust_logits(x, out=out, **kw)
    assert torch.equal(src, given)
    got = out.cpu()
    assert bool((got[~live] == HELD).all())
    check_adjust(torch.where(live[..., None], got, a.logits), a, want)
    view(dst, shift_out)[:, :, :V] = HELD
    assert bool((dst == HELD).all())                                          # before, between and behind the rows
    G.cadd_adjust_logits(x, **kw)                                             # in place: the same
    assert torch.equal(x.cpu()[live].view(torch.uint8), got[live].view(torch.uint8)) and torch.equal(x.cpu()[~live], a.logits[~live])
    x.copy_(a.logits)
    assert torch.equal(src, given)
