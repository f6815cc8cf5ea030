"""cadd_distill_loss and cadd_distill_grad where logits are far from one another or from zero: finite masks, offsets and temperatures at
which s / T is far beyond the integers that fp32 holds.

The expected gradient of rows with a rest is the formula itself, w / T (S q - p) and w / T (S q - p_rest r) with r the softmax over the rest alone: autograd
passes by log q, which in 64 bits has no digits left for log q_rest once the rest is some 1e12 T below the list.  The tolerances are logits_util's, whose share of
the rest, q p_rest / q_rest, is 0 / 0 there, and is r p_rest here, with its own distances from the rest's largest logit:
|g w / T| r p_rest (2 Z_TOL + |s - m'| / T * 2 * 2^-24)."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from logits_util import HALF, Z_TOL, Distill, check_grad, check_loss, plain_distill, random_distill, teacher_rows

pytestmark = pytest.mark.gpu
LOWEST = float(torch.tensor(-1e30))                                       # in fp32; what is below counts as -Inf


def expected_of(d: Distill):
    loss, stats, grad, tol_loss, tol_grad = plain_distill(d)
    rows, T = teacher_rows(d), d.temperature
    for b in range(d.logits.shape[0]):
        for i in range(d.logits.shape[1]):
            r = int(rows[b, i])
            if r < 0 or not d.rest:
                continue
            tok, v = d.teacher_token[b, r], d.teacher_logit[b, r]
            keep = tok >= 0
            others = torch.ones(d.logits.shape[2], dtype=torch.bool)
            others[tok[keep].long()] = False
            lse = float(d.teacher_lse[b, r]) if d.teacher_lse is not None else 0.0
            left = max(0.0, 1.0 - float(torch.exp(v[keep] / T - lse).sum()))
            x = d.logits[b, i].double()
            x = torch.where(x < LOWEST, -torch.inf, x)
            up = float(d.weight[b, i]) * float(d.grad_loss[b, i]) if d.weight is not None else 1.0
            p = torch.exp(v[keep] / T - lse)
            if left == 0.0 or len(p) == 0:
                continue
            ids, total = tok[keep].long(), float(p.sum()) + left
            q, r = torch.softmax(x / T, 0), torch.softmax(torch.where(others, x, -torch.inf) / T, 0)
            far = lambda m: 2 * Z_TOL + torch.nan_to_num((m - x) / T, posinf=0.0).clamp(min=0.0) * 2.0 ** -23
            grad[b, i] = up / T * (q * total - left * r)
            grad[b, i].index_add_(0, ids, -up / T * p)
            tol_grad[b, i] = abs(up) / T * (q * total * far(x.max()) + r * left * far(x[others].max()) + 2.0 ** -120) + HALF[d.logits.dtype] * grad[b, i].abs()
            tol_grad[b, i][ids] += abs(up) / T * total * 2.0 ** -24
    return loss, stats, grad, tol_loss, tol_grad


def every(d: Distill):
    expected = expected_of(d)
    x, t, v, kw = d.logits.cuda(), d.teacher_token.cuda(), d.teacher_logit.cuda(), d.args("cuda")
    r = G.cadd_distill_loss(x, t, v, **kw)
    check_loss(r.loss, r.stats, d, expected)
    both = G.cadd_distill_loss(x, t, v, grad=True, **kw)
    check_loss(both.loss, both.stats, d, expected)
    check_grad(both.grad, expected)
    check_grad(G.cadd_distill_grad(x, t, v, r.stats, **kw), expected)


def masked_rows(dtype, V, L, K, fill, rest, T, seed, B=1):
    """Rows of which a mask has left: the first hundred tokens and the list; the list alone; every other token; the last token and the list;
    all but the list; the first tokens of a row and nothing listed; nothing."""
    d = random_distill(B, L, V, K, dtype, seed=seed, rest=rest, temperature=T, lse=rest)
    d.n_rows = None
    for b in range(B):
        for i in range(L):
            x, ids = d.logits[b, i], d.teacher_token[b, i]
            ids = ids[ids >= 0].long()
            kept, kind = x.clone(), i % 7
            if kind == 2:
                x[::2] = fill
            elif kind == 4:
                x[ids] = fill
            else:
                x[:] = fill
                if kind == 0:
                    x[:100] = kept[:100]
                elif kind == 3:
                    x[-1] = kept[-1]
                elif kind == 5:
                    x[:50] = kept[:50]
                    x[ids] = fill
                if kind in (0, 1, 3):
                    x[ids] = kept[ids]
            if kind == 6 and abs(float(x[0])) / T > 5e29:              # (a row whose largest logit is that far out is no one's)
                x[:] = kept
    return d


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fill", [-1e4, -1e7, -1e10, -1e12, -1e20, -8e29, -1e30])
def test_finite_masks(dtype, fill):
    fill = float(torch.tensor(fill).to(dtype)) if fill > -1e30 or dtype == torch.float32 else -9.9e29      # (bf16 rounds -1e30 to a value below it)
    for T in (0.5, 1.0, 2.0):
        for rest in (False, True):
            every(masked_rows(dtype, 9001, 7, 6, fill, rest, T, seed=int(T * 4)))          # one CTA a row
    every(masked_rows(dtype, 70003, 7, 6, fill, True, 1.0, seed=3))                         # four
    every(masked_rows(dtype, 45000, 7, 6, fill, True, 1.0, seed=3, B=24))                   # more rows than SMs


@pytest.mark.parametrize("T", [2.0 ** -20, 1e-4, 0.01, 1000.0, 2.0 ** 20])
@pytest.mark.parametrize("rest", [False, True])
def test_temperatures_far_from_one(T, rest):
    for dtype in (torch.bfloat16, torch.float32):
        for sharp in (2.0, 3000.0):
            every(random_distill(2, 3, 9000, 6, dtype, seed=11, rest=rest, temperature=T, lse=rest, sharp=sharp))


@pytest.mark.parametrize("offset,T", [(181704.0, 1.0), (-181704.0, 1.0), (3e6, 1.0), (-3e6, 1.0), (1e8, 20.0), (-1e8, 20.0), (1e10, 3000.0), (-1e20, 1.0), (1e20, 1.0), (4e29, 1.0)])
def test_offsets_common_to_a_row(offset, T):
    """The loss does not depend on an offset but through the rounding of its logits; at 1e20 all of them are equal.  At 2^18 ln 2 = 181704.4 some
    of a row's logits are on either side of where sums change their kind of reference."""
    for rest in (False, True):
        for V in (9000, 60000):
            d = random_distill(2, 3, V, 6, torch.float32, seed=12, rest=rest, temperature=T, lse=rest, sharp=T)
            d.logits += offset
            every(d)


def test_single_logits_far_above_all_others():
    """Where a thread, a warp or a CTA of a row meets them, in the list and beside it, early and late."""
    for dtype in (torch.bfloat16, torch.float32):
        for high in (2e6, 5e6, 1e10, 1e25):
            d = random_distill(1, 12, 61000, 6, dtype, seed=13, rest=True)
            d.n_rows = None
            for i, at in enumerate((0, 1, 100, 5000, 20479, 20480, 40000, 60998, 60999)):
                d.logits[0, i, at] = high
                d.logits[0, i, (at + 7919) % 61000] = high / 2             # and another between them and the others
            for i in (9, 10):
                ids = d.teacher_token[0, i]
                d.logits[0, i, ids[ids >= 0][0].long()] = high
            every(d)


def test_masked_rows_repeat_bit_for_bit_and_keep_nan():
    """Which of a row's threads have met a mask before they learn of larger logits is not the same from call to call; what they give is."""
    for dtype, fill in ((torch.bfloat16, -1e9), (torch.float32, -1e12)):
        d = random_distill(20, 12, 45000, 6, dtype, seed=41, rest=True)
        d.n_rows = None
        kept = torch.rand(45000, generator=torch.Generator().manual_seed(2)) < 0.01
        ids = d.teacher_token.clamp(min=0).long()
        listed = torch.gather(d.logits, 2, ids)
        d.logits[:, :, ~kept] = fill
        d.logits.scatter_(2, ids, listed)
        d.logits[3, 4] = fill                                              # a row of nothing else
        x, t, v, kw = d.logits.cuda(), d.teacher_token.cuda(), d.teacher_logit.cuda(), d.args("cuda")
        first = G.cadd_distill_loss(x, t, v, grad=True, **kw)
        for _ in range(30):
            r = G.cadd_distill_loss(x, t, v, grad=True, **kw)
            for f in ("loss", "stats", "grad"):
                assert torch.equal(getattr(r, f), getattr(first, f))
        check = Distill(d.logits[:3], d.teacher_token[:3], d.teacher_logit[:3], rest=True, weight=d.weight[:3], grad_loss=d.grad_loss[:3])
        expected = expected_of(check)
        check_loss(first.loss[:3], first.stats[:3], check, expected)
        check_grad(first.grad[:3], expected)
        masked = [v for v in torch.nonzero(~kept)[:, 0].tolist() if not bool((ids == v).any())]
        for i, at in enumerate((masked[0], masked[len(masked) // 2], masked[-1])):
            x[5, i, at] = math.nan
        r = G.cadd_distill_loss(x, t, v, grad=True, **kw)
        assert torch.isnan(r.loss[5]).tolist() == [True] * 3 + [False] * 9 and bool(torch.isnan(r.grad[5, :3]).all())
        assert torch.equal(r.loss[:5], first.loss[:5]) and torch.equal(r.grad[6:], first.grad[6:])
