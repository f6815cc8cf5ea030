"""Host-side checks of the calls on a round's logits: what they refuse, before anything is launched, and the tests' own plain
forms.  The pointers given here are never followed: every call is refused for another reason, and the good call itself is not made."""
import ctypes as C

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from paper_2606_01813_b200 import build as B
from logits_util import Adjust, pack_bits, plain_adjust, plain_distill, random_distill, row_loss

PTR = 1 << 20


@pytest.fixture(scope="module")
def lib():
    B.build()
    return G.lib()


def fill(a, **kw):
    a.struct_size = C.sizeof(type(a))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def adjust():
    return fill(G.AdjustArgs(), batch=2, R=5, logits_dtype=0, n_bias=3, V=1000, logits=PTR, stride_b=5000, stride_row=1000, out=2 * PTR, out_stride_b=5000,
                out_stride_row=1000, token_ids=PTR, parent_idx=PTR, history=PTR, history_stride=9, history_cols=9, n_allowed=4, repetition=PTR, bias_token=PTR,
                bias=PTR, allowed=PTR, allowed_row=PTR)


def loss():
    return fill(G.DistillArgs(), batch=2, L=4, R=9, K=6, logits_dtype=0, path_cols=4, V=1000, temperature=1.0, logits=PTR, stride_b=4000, stride_l=1000,
                teacher_token=PTR, teacher_logit=PTR, path=PTR, path_len=PTR, loss=PTR, stats=PTR, grad=2 * PTR, grad_stride_b=4000, grad_stride_l=1000)


CALLS = {"adjust": (adjust, "cadd_adjust_logits"), "loss": (loss, "cadd_distill_loss"), "grad": (loss, "cadd_distill_grad")}
DISTILL = [
    (dict(batch=0), G.ERR_SHAPE), (dict(L=0), G.ERR_SHAPE), (dict(V=0), G.ERR_SHAPE), (dict(V=2000001, grad_stride_l=1 << 21, grad_stride_b=1 << 25), G.ERR_SHAPE),
    (dict(K=0), G.ERR_SHAPE), (dict(K=257), G.ERR_SHAPE), (dict(R=0), G.ERR_SHAPE),
    (dict(path=None, path_len=None, R=3), G.ERR_SHAPE), (dict(path_cols=0), G.ERR_SHAPE), (dict(temperature=0.0), G.ERR_SHAPE), (dict(temperature=-1.0), G.ERR_SHAPE),
    (dict(temperature=float("nan")), G.ERR_SHAPE), (dict(temperature=float("inf")), G.ERR_SHAPE), (dict(temperature=2.0 ** 21), G.ERR_SHAPE),
    (dict(logits_dtype=2), G.ERR_DTYPE), (dict(logits=None), G.ERR_NULL), (dict(teacher_token=None), G.ERR_NULL), (dict(teacher_logit=None), G.ERR_NULL),
    (dict(path_len=None), G.ERR_NULL), (dict(logits=PTR + 1), G.ERR_ALIGN), (dict(grad=2 * PTR + 1), G.ERR_ALIGN), (dict(stats=PTR + 8), G.ERR_ALIGN),
    (dict(teacher_logit=PTR + 4), G.ERR_ALIGN), (dict(weight=PTR + 2), G.ERR_ALIGN), (dict(status=PTR + 1), G.ERR_ALIGN), (dict(stride_l=-1000), G.ERR_SHAPE),
    (dict(grad_stride_l=999), G.ERR_SHAPE), (dict(grad_stride_b=3999), G.ERR_SHAPE), (dict(grad_stride_b=0), G.ERR_SHAPE), (dict(grad=PTR, stride_b=8000), G.ERR_SHAPE),
    (dict(grad=PTR, stride_l=2000), G.ERR_SHAPE)]
OWN = {
    "adjust": [
        (dict(batch=0), G.ERR_SHAPE), (dict(R=0), G.ERR_SHAPE), (dict(R=65537), G.ERR_SHAPE), (dict(V=0), G.ERR_SHAPE), (dict(V=1 << 31), G.ERR_SHAPE),
        (dict(logits_dtype=2), G.ERR_DTYPE), (dict(logits_dtype=-1), G.ERR_DTYPE), (dict(n_bias=-1), G.ERR_SHAPE), (dict(n_bias=65537), G.ERR_SHAPE), (dict(history_cols=0), G.ERR_SHAPE), (dict(history_cols=1 << 30), G.ERR_SHAPE),
        (dict(history_stride=-9), G.ERR_SHAPE), (dict(n_allowed=0), G.ERR_SHAPE), (dict(logits=None), G.ERR_NULL), (dict(out=None), G.ERR_NULL),
        (dict(parent_idx=None), G.ERR_NULL), (dict(bias=None), G.ERR_NULL), (dict(bias_token=None), G.ERR_NULL), (dict(allowed_row=None), G.ERR_NULL),
        (dict(logits=PTR + 1), G.ERR_ALIGN), (dict(out=2 * PTR + 1), G.ERR_ALIGN), (dict(logits_dtype=1, out=2 * PTR + 2), G.ERR_ALIGN), (dict(history=PTR + 2), G.ERR_ALIGN),
        (dict(allowed=PTR + 2), G.ERR_ALIGN), (dict(status=PTR + 1), G.ERR_ALIGN), (dict(stride_b=-1), G.ERR_SHAPE), (dict(out_stride_row=999), G.ERR_SHAPE),
        (dict(out_stride_b=4999), G.ERR_SHAPE), (dict(out_stride_b=0), G.ERR_SHAPE), (dict(out=PTR, stride_b=0), G.ERR_SHAPE), (dict(out=PTR, stride_row=2000), G.ERR_SHAPE)],
    "loss": DISTILL + [(dict(loss=None, stats=None, grad=None), G.ERR_NULL)],
    "grad": DISTILL + [(dict(stats=None), G.ERR_NULL), (dict(grad=None), G.ERR_NULL)],
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_calls_refuse_bad_arguments(lib, name):
    make, fn = CALLS[name][0], getattr(lib, CALLS[name][1])
    assert fn(None, None) == G.ERR_NULL
    a = make()
    a.struct_size -= 8
    assert fn(C.byref(a), None) == G.ERR_STRUCT_SIZE
    for change, code in OWN[name]:
        a = make()
        for k, v in change.items():
            setattr(a, k, v)
        assert fn(C.byref(a), None) == code, change


def test_binding_refuses_cpu_tensors():
    x, t = torch.zeros(1, 2, 8), torch.zeros(1, 2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        G.cadd_adjust_logits(x)
    with pytest.raises(ValueError):
        G.cadd_distill_loss(x, t, torch.zeros(1, 2, 3, dtype=torch.float64))
    with pytest.raises(ValueError):
        G.cadd_distill_grad(x, t, torch.zeros(1, 2, 3, dtype=torch.float64), torch.zeros(1, 2, 4))


def test_plain_adjust_by_hand():
    """Two rows of a chain over five tokens, every rule once."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)
    a = Adjust(torch.tensor([[[2.0, -2.0, 1.0, 4.0, 0.5], [2.0, -2.0, 1.0, 4.0, 0.5]]]), token_ids=i32([[1, 3]]), parent_idx=i32([[-1, 0]]),
               history=i32([[0, 2, 2, 9]]), prompt_len=i32([1]), repetition=torch.tensor([2.0]), presence=torch.tensor([0.25]), frequency=torch.tensor([0.5]),
               bias_token=i32([[4, 3, 4]]), bias=torch.tensor([[1.0, 8.0, 0.5]]), allowed=pack_bits(torch.tensor([[True, True, True, True, False]])),
               allowed_row=i32([[-1, 0]]))
    y, _, _ = plain_adjust(a)
    # token 0 in the prompt: 2 / 2; token 1 on the path: -2 * 2 - .75; token 2 twice: 1 / 2 - 1 - .25; token 3 on the second row's path
    assert y[0, 0].tolist() == [1.0, -4.75, -0.75, 12.0, 2.0]
    assert y[0, 1].tolist() == [1.0, -4.75, -0.75, 2.0 - 0.75 + 8.0, -float("inf")]


@pytest.mark.parametrize("rest,T,twice", [(False, 1.0, False), (False, 2.0, True), (True, 1.0, False), (True, 0.5, True)])
def test_plain_gradient_by_formula_and_by_differences(rest, T, twice):
    d = random_distill(2, 3, 12, 5, torch.float32, 7, rest=rest, temperature=T, lse=rest and T != 1.0, twice=twice)
    _, _, grad, _, _ = plain_distill(d)
    for b in range(2):
        for i in range(int(d.n_rows[b])):
            tok, val = d.teacher_token[b, i], d.teacher_logit[b, i]
            lse = float(d.teacher_lse[b, i]) if d.teacher_lse is not None else 0.0
            s = d.logits[b, i].double()
            w = float(d.weight[b, i]) * float(d.grad_loss[b, i])
            q = torch.softmax(s / T, 0)
            have = tok >= 0
            p = torch.exp(val[have] / T - lse) if rest else torch.softmax(val[have] / T, 0)
            left = max(0.0, 1.0 - float(p.sum())) if rest else 0.0
            listed = torch.zeros(12, dtype=torch.bool)
            listed[tok[have].long()] = True
            want = (float(p.sum()) + left) * q - torch.zeros(12, dtype=torch.float64).index_add(0, tok[have].long(), p)
            if rest:
                want = want - torch.where(listed, 0.0, q * left / q[~listed].sum())
            assert torch.allclose(grad[b, i], w / T * want, rtol=1e-9, atol=1e-12)
            for v in range(12):
                e = torch.zeros(12, dtype=torch.float64)
                e[v] = 1e-5
                diff = (row_loss(s + e, tok, val, lse, rest, T) - row_loss(s - e, tok, val, lse, rest, T)) / 2e-5
                assert abs(float(diff) * w - float(grad[b, i, v])) < 1e-7


def test_a_gradient_that_has_no_place_is_refused():
    x, t = torch.zeros(1, 2, 8), torch.zeros(1, 2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="out.grad"):
        G.cadd_distill_loss(x, t, torch.zeros(1, 2, 3, dtype=torch.float64), grad=True, out=G.Distilled(loss=torch.zeros(1, 2)))
