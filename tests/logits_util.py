"""Plain 64-bit forms of the operators on a round's logits, and small random problems for them.

Everything here works on CPU tensors in float64, token by token from the definitions; nothing of the library is used.

Tolerances.  A rounding to type t is off by at most HALF[t] relative.
adjust: tokens that penalties or biases concern are computed in 64 bits from a bias that was added up in 64 bits and rounded to
fp32 once, then rounded to the output type: HALF[t] |y| + 2^-24 |bias|.  All others keep their bits.
distill: a term exp((s - m) / T) of a row's sum Z has an argument in units of log2 that is rounded twice (the factor log2(e) / T and the
fused multiply-add: 2 * 2^-24 |arg| ln 2 relative, and |arg| 2^-|arg| < 0.54 bounds what that adds to Z), an ex2 that is good to 2^-22, and at
most eight roundings of fp32 partial sums: 2^-22 + 9 * 2^-24 < Z_TOL = 2^-20, also of Z over the tokens that are not listed.  The loss adds S
log Z and p_rest (log Z' - log Z), so w (S + 2 p_rest) Z_TOL, and one rounding.  A gradient element g w / T (S q - p - p_rest q / q_rest) takes for
its q the same relative error, plus the argument's at its own distance from the largest logit, |s - m| / T * 2 * 2^-24, plus two fp32 products, and
one rounding to the output type; underflow of fp32 exponentials is below 2^-125 of the factors."""
import math
import random
from dataclasses import dataclass, field
from typing import Optional

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
Z_TOL = 2.0 ** -20


# ---------------------------------------------------------------------------------------------------------- adjust

@dataclass
class Adjust:
    """A problem of cadd_adjust_logits; arguments that are None are not passed."""
    logits: torch.Tensor
    n_nodes: Optional[torch.Tensor] = None
    token_ids: Optional[torch.Tensor] = None
    parent_idx: Optional[torch.Tensor] = None
    history: Optional[torch.Tensor] = None
    history_len: Optional[torch.Tensor] = None
    prompt_len: Optional[torch.Tensor] = None
    repetition: Optional[torch.Tensor] = None
    presence: Optional[torch.Tensor] = None
    frequency: Optional[torch.Tensor] = None
    bias_token: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    allowed: Optional[torch.Tensor] = None
    allowed_row: Optional[torch.Tensor] = None

    def args(self, dev):
        return {k: v.to(dev) for k, v in self.__dict__.items() if v is not None and k != "logits"}


def pack_bits(m):
    """bool [n, V] -> int32 [n, ceil(V/32)]."""
    n, V = m.shape
    w = (V + 31) // 32
    full = torch.zeros(n, w * 32, dtype=torch.int64)
    full[:, :V] = m
    x = (full.view(n, w, 32) << torch.arange(32)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).int()


def random_adjust(B, R, V, dtype, seed, tree=True, history=50, n_bias=7, masks=True, penalties=True, spread=None, dead=True):
    """Tokens are drawn from the first `spread` of the vocabulary, so that history, path, biases and masks meet."""
    g = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    spread = min(V, spread or max(4, V // 3))
    a = Adjust(logits=(3 * torch.randn(B, R, V, generator=g)).to(dtype))
    live = [rng.randint(0, R) if dead else R for _ in range(B)]
    live[-1] = R
    a.n_nodes = torch.tensor([n - 1 for n in live], dtype=torch.int32)
    tokens = lambda *s: torch.randint(0, spread, s, generator=g).int()
    if tree:
        a.token_ids, a.parent_idx = tokens(B, R), torch.full((B, R), -1, dtype=torch.int32)
        for b in range(B):
            for j in range(1, R):
                a.parent_idx[b, j] = rng.randint(max(0, j - 4), j - 1)
    if history:
        a.history = tokens(B, history)
        a.history_len = torch.tensor([rng.randint(0, history) for _ in range(B)], dtype=torch.int32)
        a.history_len[0] = history
        a.prompt_len = torch.tensor([rng.randint(0, int(n)) for n in a.history_len], dtype=torch.int32)
    if penalties:
        a.repetition, a.presence, a.frequency = 0.7 + torch.rand(B, generator=g), torch.randn(B, generator=g), 0.3 * torch.randn(B, generator=g)
    if n_bias:
        a.bias_token, a.bias = tokens(B, n_bias), 3 * torch.randn(B, n_bias, generator=g)
    if masks:
        n = max(1, B * R // 2)
        a.allowed = pack_bits(torch.rand(n, V, generator=g) < torch.rand(n, 1, generator=g))
        a.allowed_row = torch.randint(-1, n, (B, R), generator=g).int()
    return a


def plain_adjust(a: Adjust):
    """(result in float64, bool mask of the tokens that something concerned, sum of biases per token), rows above n_nodes as in the input."""
    x = a.logits.double().clone()
    B, R, V = x.shape
    touched = torch.zeros(B, R, V, dtype=torch.bool)
    added = torch.zeros(B, R, V, dtype=torch.float64)
    num = lambda t, b, default: float(t[b]) if t is not None else default
    penalised = a.repetition is not None or a.presence is not None or a.frequency is not None
    for b in range(B):
        live = R if a.n_nodes is None else max(0, min(R, int(a.n_nodes[b]) + 1))
        rep, pres, freq = num(a.repetition, b, 1.0), num(a.presence, b, 0.0), num(a.frequency, b, 0.0)
        prompt, said = [], []
        if a.history is not None:
            n = a.history.shape[1] if a.history_len is None else max(0, min(a.history.shape[1], int(a.history_len[b])))
            q = 0 if a.prompt_len is None else max(0, min(n, int(a.prompt_len[b])))
            h = a.history[b].tolist()
            prompt, said = h[:q], h[q:n]
        for j in range(live):
            path = []
            if a.token_ids is not None:
                at = j
                for _ in range(65):
                    path.append(int(a.token_ids[b, at]))
                    up = int(a.parent_idx[b, at])
                    if up < 0 or up >= at:
                        break
                    at = up
            out, every = {}, set()
            if penalised:
                for t in said + path:
                    if 0 <= t < V:
                        out[t] = out.get(t, 0) + 1
                every = set(out) | {t for t in prompt if 0 <= t < V}
            y = x[b, j]
            for t in every:
                v = float(y[t])
                v = v / rep if v > 0 else v * rep
                if out.get(t, 0) > 0:
                    v = v - freq * out[t] - pres
                y[t] = v
                touched[b, j, t] = True
            if a.bias is not None:
                for t, v in zip(a.bias_token[b].tolist(), a.bias[b].double().tolist()):
                    if 0 <= t < V:
                        added[b, j, t] += v
                        touched[b, j, t] = True
                y += added[b, j]
            if a.allowed is not None:
                m = int(a.allowed_row[b, j])
                if 0 <= m < a.allowed.shape[0]:
                    v = torch.arange(V)
                    bits = (a.allowed[m][v // 32] >> (v % 32).int()) & 1
                    y[bits == 0] = -math.inf
                    touched[b, j] |= bits == 0
    return x, touched, added


def check_adjust(got, a: Adjust, expected=None):
    want, touched, added = expected or plain_adjust(a)
    got, dtype = got.cpu(), a.logits.dtype
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    same = got.contiguous().view(bits) == a.logits.contiguous().view(bits)
    assert bool((same | touched).all()), "a token that nothing concerns has changed"
    g = got.double()
    assert torch.equal(torch.isnan(g), torch.isnan(want))
    # (rounding to nearest takes what is beyond the type's largest number by half a step to infinity)
    want = torch.where(torch.isinf(want.to(dtype)), want.to(dtype).double(), want)
    fine = torch.isfinite(want)
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(g[odd], want[odd])
    tol = HALF[dtype] * want.abs() + 2.0 ** -24 * added.abs() + 2.0 ** -126
    bad = fine & ~((g - want).abs() <= tol)
    assert not bool(bad.any()), (bad.nonzero()[:5], g[bad][:5], want[bad][:5])


# ---------------------------------------------------------------------------------------------------------- distill

@dataclass
class Distill:
    """A problem of cadd_distill_loss / cadd_distill_grad."""
    logits: torch.Tensor
    teacher_token: torch.Tensor
    teacher_logit: torch.Tensor
    teacher_lse: Optional[torch.Tensor] = None
    rest: bool = False
    temperature: float = 1.0
    path: Optional[torch.Tensor] = None
    path_len: Optional[torch.Tensor] = None
    n_rows: Optional[torch.Tensor] = None
    weight: Optional[torch.Tensor] = None
    grad_loss: Optional[torch.Tensor] = None

    def args(self, dev):
        put = lambda v: v.to(dev) if isinstance(v, torch.Tensor) else v
        return {k: put(v) for k, v in self.__dict__.items() if v is not None and k not in ("logits", "teacher_token", "teacher_logit")}


def random_distill(B, L, V, K, dtype, seed, rest=False, temperature=1.0, path=False, lse=False, twice=False, sharp=2.0, weight=True):
    g = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    R = 2 * L + 1 if path else L
    x = sharp * torch.randn(B, L, V, generator=g)
    tok = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(B * R)]).view(B, R, -1)
    if tok.shape[2] < K:                                                   # a vocabulary shorter than the list
        tok = torch.cat([tok, torch.full((B, R, K - tok.shape[2]), -1)], 2)
    if twice and K > 2:
        tok[:, :, K - 1] = tok[:, :, 0]
        tok[::2, :, K // 2] = tok[::2, :, 0]
    val = 2 * torch.randn(B, R, K, generator=g, dtype=torch.float64)
    if rest and not lse:
        val = torch.log_softmax(torch.where(tok >= 0, val, -math.inf), -1) + torch.log(0.3 + 0.69 * torch.rand(B, R, 1, generator=g, dtype=torch.float64))
    gone = torch.rand(B, R, K, generator=g) < 0.15
    gone[..., 0] = False
    tok = torch.where(gone, -1, tok)
    val = torch.where(tok < 0, -math.inf, val)
    d = Distill(x.to(dtype), tok.int(), val, rest=rest, temperature=temperature)
    if lse:
        d.teacher_lse = torch.logsumexp(torch.where(tok < 0, -math.inf, val) / temperature, -1) + torch.rand(B, R, generator=g, dtype=torch.float64)
    if path:
        n = [rng.randint(0, L - 1) for _ in range(B)]
        d.path = torch.full((B, L), -1, dtype=torch.int32)
        for b in range(B):
            d.path[b, :n[b]] = torch.tensor(sorted(rng.sample(range(1, R), n[b])), dtype=torch.int32)
        d.path_len = torch.tensor(n, dtype=torch.int32)
    else:
        d.n_rows = torch.tensor([rng.randint(0, L) for _ in range(B)], dtype=torch.int32)
        d.n_rows[0] = L
    if weight:
        d.weight = 0.1 + torch.rand(B, L, generator=g)
        d.grad_loss = torch.randn(B, L, generator=g)
    return d


def teacher_rows(d: Distill):
    """Row of the lists for each position, -1 for those left out by path, n_rows or weight."""
    B, L, _ = d.logits.shape
    R = d.teacher_token.shape[1]
    rows = torch.full((B, L), -1)
    for b in range(B):
        if d.path is not None:
            n = max(0, min(int(d.path_len[b]), L - 1, d.path.shape[1]))
            want = [0] + d.path[b, :n].tolist()
        else:
            n = L if d.n_rows is None else max(0, min(L, int(d.n_rows[b])))
            want = list(range(n))
        for i, r in enumerate(want):
            if 0 <= r < R and (d.weight is None or float(d.weight[b, i]) != 0.0):
                rows[b, i] = r
    return rows


def row_loss(s, tok, val, lse, rest, T):
    """Divergence of one row (float64 tensor s; autograd passes through), or None where the list leaves it out."""
    V = s.shape[0]
    keep = (tok >= 0) & (tok < V)
    tok, val = tok[keep].long(), val[keep]
    if len(tok) == 0 or (not rest and bool((val == -math.inf).all())):
        return None
    logq = torch.log_softmax(s / T, 0)
    logp = val / T - lse if rest else torch.log_softmax(val / T, 0)
    p = torch.exp(logp)
    has = p > 0
    loss = (p[has] * (logp[has] - logq[tok[has]])).sum()
    if rest:
        left = 1.0 - float(p.sum())
        others = torch.ones(V, dtype=torch.bool)
        others[tok] = False
        mass = bool(others.any()) and bool((s[others] > -math.inf).any())
        if left > 0 and (mass or left > 2.0 ** -20):
            if mass:
                loss = loss + left * (math.log(left) - torch.logsumexp(logq[others], 0))
            else:                                                          # log q_rest = -inf - log sum exp(s / T), whose gradient stays
                all_of_it = torch.logsumexp(s / T, 0)
                loss = loss + math.inf + left * (all_of_it - all_of_it.detach())
    return loss


def plain_distill(d: Distill):
    """loss, stats, gradient (of sum grad_loss * loss) and the gradient's error scale per element, all float64."""
    B, L, V = d.logits.shape
    T = d.temperature
    rows = teacher_rows(d)
    loss, stats = torch.zeros(B, L, dtype=torch.float64), torch.zeros(B, L, 4, dtype=torch.float64)
    grad, tol_loss = torch.zeros(B, L, V, dtype=torch.float64), torch.zeros(B, L, dtype=torch.float64)
    tol_grad = torch.zeros(B, L, V, dtype=torch.float64)
    for b in range(B):
        for i in range(L):
            r = int(rows[b, i])
            if r < 0:
                continue
            tok, val = d.teacher_token[b, r], d.teacher_logit[b, r]
            lse = float(d.teacher_lse[b, r]) if d.teacher_lse is not None else 0.0
            s = d.logits[b, i].double().requires_grad_(True)
            one = row_loss(s, tok, val, lse, d.rest, T)
            if one is None:
                continue
            w = float(d.weight[b, i]) if d.weight is not None else 1.0
            up = float(d.grad_loss[b, i]) if d.grad_loss is not None else 1.0
            loss[b, i] = w * float(one.detach())
            (ds,) = torch.autograd.grad(one, s)
            grad[b, i] = up * w * ds
            x = s.detach()
            keep = (tok >= 0) & (tok < V)
            ids, v = tok[keep].long(), val[keep]
            others = torch.ones(V, dtype=torch.bool)
            others[ids] = False
            q = torch.softmax(x / T, 0)
            for at, y in ((0, x), (2, x[others])):
                m = y.max() if len(y) else torch.tensor(-math.inf)
                stats[b, i, at] = m
                stats[b, i, at + 1] = torch.exp((y - m) / T).sum() if float(m) > -math.inf else 0.0
            p = torch.exp(v / T - lse) if d.rest else torch.softmax(v / T, 0)
            left = max(0.0, 1.0 - float(p.sum())) if d.rest else 0.0
            total = float(p.sum()) + left
            tol_loss[b, i] = abs(w) * (total + 2 * left) * Z_TOL + 2.0 ** -24 * abs(loss[b, i])
            share = torch.full((V,), total, dtype=torch.float64)
            if left > 0 and bool(others.any()):
                share[others] += left / max(float(q[others].sum()), 1e-300)
            far = torch.nan_to_num((x.max() - x) / T, posinf=0.0)
            tol_grad[b, i] = abs(up * w / T) * (q * share * (2 * Z_TOL + far * 2.0 ** -23) + 2.0 ** -120) + HALF[d.logits.dtype] * grad[b, i].abs()
            tol_grad[b, i][ids] += abs(up * w / T) * total * 2.0 ** -24          # a listed token's gradient is rounded to fp32 before
    return loss, stats, grad, tol_loss, tol_grad


def check_loss(got, stats, d: Distill, expected):
    loss, want, _, tol, _ = expected
    if got is not None:
        got = got.double()
        bad = ~(((got.cpu() - loss).abs() <= tol) | (got.cpu() == loss))      # (infinite ones are equal)
        assert not bool(bad.any()), (bad.nonzero()[:5], got.cpu()[bad][:5], loss[bad][:5], tol[bad][:5])
    if stats is not None:
        s = stats.double().cpu()
        assert torch.equal(s[..., 0], want[..., 0]) and torch.equal(s[..., 2], want[..., 2])
        for k in (1, 3):
            assert bool(((s[..., k] - want[..., k]).abs() <= Z_TOL * want[..., k]).all()), k


def check_grad(got, expected):
    _, _, grad, _, tol = expected
    g = got.double().cpu()
    bad = ~((g - grad).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:5], g[bad][:5], grad[bad][:5], tol[bad][:5])
