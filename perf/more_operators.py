"""Work of the logits operators, for timing and for checking them at real sizes.

Operators on the two kinds of logits of a decoding round, the target's at the nodes of the draft tree and the drafter's:

  adjust   penalties for tokens that were used before (in the history or on the node's own path), biases and grammar masks
  loss     distillation: divergence of the drafter's distribution from the target's top tokens, row by row
  grad     its gradient with respect to the drafter's logits, when the gradient of the losses is known
  step     both in one call, as a training step of the drafter takes them

`run` computes a case in plain torch operations (`own` false) or through the framework's entry points (`own` true)."""
import math
import random

import torch

own = False

TREE_DEPTH = 16                       # deepest node of a tree: the draft block of the benchmark configurations


# ---------------------------------------------------------------------------------------------------------- cases

def _case(name, op, **kw):
    c = dict(name=name, op=op, batch=1, rows=1, vocab=151936, bf16=True,
             tree=False, history=0, n_bias=0, masked=0.0, allow=0.5, penalties=True, in_place=False,
             k=16, rest=False, temperature=1.0, path=False)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one conversation, penalties over its thousand tokens and a few biases: the smallest call, where latency counts
        _case("adjust_token", "adjust", history=1000, n_bias=8),
        # one token each for a batch of conversations, half of them under a grammar
        _case("adjust_token_batch", "adjust", batch=64, history=8192, n_bias=16, masked=0.5),
        # the rows of draft trees of up to 64 nodes before verification: the ordinary round of a server
        _case("adjust_tree", "adjust", batch=32, rows=65, tree=True, history=4000, n_bias=8, masked=0.75),
        # trees at the node cap of 256 in fp32, an odd vocabulary, long histories
        _case("adjust_tree_fp32", "adjust", batch=8, rows=257, vocab=32001, bf16=False, tree=True, history=32768, masked=0.3),
        # a grammar alone, that leaves few tokens, on the logits in place
        _case("grammar_in_place", "adjust", batch=32, rows=65, tree=True, masked=1.0, allow=0.01, penalties=False, in_place=True),
        # how well the drafter meets the target on one request's block of 16: latency
        _case("loss_one", "loss", rows=16, k=8),
        # the same for a large batch over the accepted paths of a round
        _case("loss_batch", "loss", batch=256, rows=16, k=16, rest=True, path=True),
        # a small training step, odd vocabulary and odd block
        _case("step_odd", "step", batch=8, rows=15, vocab=50001, k=20),
        # an ordinary training step: 64 sequences, blocks of 32
        _case("step_rest", "step", batch=64, rows=32, k=32, rest=True),
        # a training step in fp32 with softened distributions and long lists
        _case("step_fp32", "step", batch=32, rows=16, vocab=100003, bf16=False, k=64, temperature=2.0),
        # the backward pass alone, over the accepted paths of a round
        _case("grad_path", "grad", batch=128, rows=16, k=16, rest=True, path=True),
        # the backward pass of a small odd batch
        _case("grad_odd", "grad", batch=6, rows=7, vocab=32001, k=5, temperature=0.7),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    cap = {}
    for c in listed():
        cap[c["op"]] = max(cap.get(c["op"], 0), work(c)["bytes"])
    op = rng.choice(["adjust", "adjust", "loss", "step", "grad"])
    while True:
        vocab = rng.choice([151936, _log_int(rng, 1000, 260000), _log_int(rng, 1000, 260000)])
        c = _case("", op, batch=_log_int(rng, 1, 256), vocab=vocab, bf16=rng.random() < 0.7)
        if op == "adjust":
            c["rows"] = rng.choice([1, _log_int(rng, 2, 1025)])
            c["tree"] = c["rows"] > 1 and rng.random() < 0.8
            c["history"] = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 1, 32768)])
            c["n_bias"] = rng.choice([0, _log_int(rng, 1, 300)])
            c["masked"] = rng.choice([0.0, round(rng.random(), 2), 1.0])
            c["allow"] = rng.choice([0.001, 0.01, 0.5, 0.99])
            if rng.random() < 0.2:
                c.update(in_place=True, penalties=False, history=0, n_bias=0, masked=1.0)
        else:
            c["rows"] = _log_int(rng, 1, 64)
            c["k"] = _log_int(rng, 1, 256)
            c["path"] = rng.random() < 0.3
            c["rest"] = rng.random() < 0.5
            c["temperature"] = 1.0 if c["rest"] else rng.choice([1.0, 0.5, 2.0, 4.0])
        if work(c)["bytes"] <= cap[op]:
            del c["name"]
            return c


def _live(case):
    """Rows in use of each request: nodes of its tree with the root, or rows that are learnt from."""
    rng = random.Random(case["batch"] * 7919 + case["rows"])
    if case["op"] == "adjust":
        n = [rng.randint(max(1, case["rows"] // 3), case["rows"]) for _ in range(case["batch"])]
        n[-1] = case["rows"]
        return n
    if case["path"]:
        return [min(rng.choice([0, 1, 2, 3, 4, 6, 8, 12, TREE_DEPTH]) + 1, case["rows"]) for _ in range(case["batch"])]
    return [case["rows"]] * case["batch"]


def _history_lens(case):
    rng = random.Random(case["batch"] * 1000003 + case["history"])
    n = [rng.randint(case["history"] // 4, case["history"]) for _ in range(case["batch"])]
    n[0] = case["history"]
    return n


def _mask_of_rows(case):
    """Number of the mask of every row, -1 for none: half of the masked rows share a mask with the row before."""
    rng = random.Random(case["batch"] * 104729 + case["rows"])
    out, n = [], 0
    for _ in range(case["batch"]):
        rows = []
        for j in range(case["rows"]):
            if rng.random() >= case["masked"]:
                rows.append(-1)
            elif n and rng.random() < 0.5:
                rows.append(n - 1)
            else:
                rows.append(n)
                n += 1
        out.append(rows)
    return out, n


def work(case):
    V, es, live = case["vocab"], 2 if case["bf16"] else 4, _live(case)
    if case["op"] == "adjust":
        words = (V + 31) // 32
        masks, n_masks = _mask_of_rows(case)
        if case["in_place"]:
            hit = sum(m >= 0 for b, r in zip(masks, live) for m in b[:r])
            return {"bytes": int(n_masks * words * 4 + hit * V * (1 - case["allow"]) * es), "flops": hit * V}
        n = sum(live)
        return {"bytes": n * V * 2 * es + n_masks * words * 4 + sum(_history_lens(case)) * 4 + case["batch"] * case["n_bias"] * 8 + n * 12, "flops": n * V}
    n = sum(live)
    read = n * (V * es + case["k"] * 12 + 4)
    if case["op"] == "loss":
        return {"bytes": read + case["batch"] * case["rows"] * 20, "flops": n * V * 4}
    return {"bytes": read + case["batch"] * case["rows"] * (V * es + 4), "flops": n * V * (8 if case["op"] == "step" else 4)}


# ---------------------------------------------------------------------------------------------------------- inputs

def _tree(rows, live, rng):
    """Parents of a random tree in the order in which best-first growth adds nodes."""
    parent, depth = [-1], [0]
    for j in range(1, rows):
        if j < live:
            p = rng.randint(max(0, j - 1 - j // 2), j - 1)
            while depth[p] >= TREE_DEPTH:
                p = parent[p]
            parent.append(p)
            depth.append(depth[p] + 1)
        else:
            parent.append(-1)
            depth.append(0)
    return parent


def _prepare_adjust(case, st, g, rng, dev):
    B, R, V = case["batch"], case["rows"], case["vocab"]
    live, lens = st["live"], _history_lens(case)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    st["n_nodes"] = i32([n - 1 for n in live])
    # tokens as in text: a few are frequent, and those come back in the tree
    tokens = lambda *s: (torch.rand(*s, generator=g, device=dev).pow_(3) * V).int().clamp_(max=V - 1)
    if case["tree"]:
        st["parent_idx"] = i32([_tree(R, n, rng) for n in live])
        used = torch.arange(R, device=dev)[None] <= st["n_nodes"][:, None]
        st["token_ids"] = torch.where(used, tokens(B, R), -1)
    if case["history"]:
        st["history"] = tokens(B, case["history"])
        st["history_len"], st["prompt_len"] = i32(lens), i32([n // 3 for n in lens])
    if case["penalties"]:
        st["repetition"] = 1.0 + 0.5 * torch.rand(B, generator=g, device=dev)
        st["presence"] = torch.rand(B, generator=g, device=dev)
        st["frequency"] = 0.2 * torch.rand(B, generator=g, device=dev)
    if case["n_bias"]:
        st["bias_token"] = torch.stack([torch.randperm(V, generator=g, device=dev)[:case["n_bias"]] for _ in range(B)]).int()
        st["bias"] = 4.0 * torch.randn(B, case["n_bias"], generator=g, device=dev)
    masks, n_masks = _mask_of_rows(case)
    if n_masks:
        words = (V + 31) // 32
        bits = torch.zeros(n_masks, words, dtype=torch.int32, device=dev)
        for a in range(0, n_masks, 64):
            m = torch.rand(min(64, n_masks - a), words * 32, generator=g, device=dev) < case["allow"]
            w = (m.view(-1, words, 32).long() << torch.arange(32, device=dev)).sum(-1)
            bits[a:a + 64] = torch.where(w >= 1 << 31, w - (1 << 32), w).int()
        st["allowed"], st["allowed_row"] = bits, i32(masks)
    if not case["in_place"]:
        st["out"] = torch.zeros_like(st["logits"])


def _prepare_distill(case, st, g, rng, dev):
    B, L, V, K = case["batch"], case["rows"], case["vocab"], min(case["k"], case["vocab"])
    live = st["live"]
    R = 4 * L + 1 if case["path"] else L
    # distinct tokens; a position has fewer than K now and then
    token = (torch.rand(B, R, K, generator=g, device=dev) * (V // K)).long() + torch.arange(K, device=dev) * (V // K)
    token = torch.gather(token, 2, torch.rand(B, R, K, generator=g, device=dev).argsort(-1))
    value = torch.sort(3.0 * torch.randn(B, R, K, generator=g, device=dev), -1, descending=True).values.double()
    value = torch.log_softmax(value, -1) + torch.log(0.4 + 0.599 * torch.rand(B, R, 1, generator=g, device=dev, dtype=torch.float64))
    short = (torch.rand(B, R, 1, generator=g, device=dev) < 0.1) & (torch.arange(K, device=dev) >= max(1, K // 2))
    st["teacher_token"] = torch.where(short, -1, token).int()
    st["teacher_logprob"] = torch.where(short, -math.inf, value)
    if case["path"]:
        path = torch.full((B, L), -1, dtype=torch.int32)
        for b in range(B):
            path[b, :live[b] - 1] = torch.tensor(sorted(rng.sample(range(1, R), live[b] - 1)), dtype=torch.int32)
        st["path"], st["path_len"] = path.to(dev), torch.tensor([n - 1 for n in live], dtype=torch.int32, device=dev)
        st["rows_of"] = [[0] + path[b, :live[b] - 1].tolist() for b in range(B)]
    else:
        st["rows_of"] = [list(range(L)) for _ in range(B)]
    st["weight"] = (0.9 ** torch.arange(L, device=dev)).expand(B, L).contiguous()
    # the drafter knows something: the target's tokens stand out in its logits
    for b in range(B):
        rows = torch.tensor(st["rows_of"][b], device=dev)
        t = st["teacher_token"][b, rows].long()
        x = st["logits"][b, :len(rows)]
        up = torch.where(t >= 0, 4.0 + st["teacher_logprob"][b, rows].clamp(min=-8.0), 0.0).float()
        x.scatter_add_(1, t.clamp(min=0), up.to(x.dtype))
    if case["op"] != "grad":
        st["loss"] = torch.zeros(B, L, device=dev)
    if case["op"] != "step":
        st["stats"] = torch.zeros(B, L, 4, device=dev)
    if case["op"] == "grad":                                                 # what the forward pass left, and the gradient of its losses
        st["grad_loss"] = torch.randn(B, L, generator=g, device=dev)
        for b in range(B):
            rows = st["rows_of"][b]
            st["stats"][b, :len(rows)] = _stats(st["logits"][b, :len(rows)].double(), st["teacher_token"][b, rows].long(), case["temperature"]).float()
    if case["op"] != "loss":
        st["grad"] = torch.zeros_like(st["logits"])


def _rest_only(x, t):
    """x with -inf at the listed tokens (t, -1 where none)."""
    listed = torch.zeros(x.shape[0], x.shape[1] + 1, dtype=torch.bool, device=x.device)
    listed.scatter_(1, torch.where(t >= 0, t, x.shape[1]), True)
    return x.masked_fill(listed[:, :-1], -math.inf)


def _stats(x, t, temperature):
    """Largest logit and the sum of exp((logit - largest) / temperature), of all tokens and of those that are not listed: [rows, 4]."""
    out = []
    for y in (x, _rest_only(x, t)):
        m = y.amax(-1)
        out += [m, torch.where(m[:, None] > -math.inf, torch.exp((y - m[:, None]) / temperature), 0.0).sum(-1)]
    return torch.stack(out, -1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    B, R, V = case["batch"], case["rows"], case["vocab"]
    st = dict(case=case, live=_live(case))
    st["logits"] = torch.empty(B, R, V, dtype=torch.bfloat16 if case["bf16"] else torch.float32, device=dev)
    step = max(1, (1 << 28) // (R * V))
    for a in range(0, B, step):
        st["logits"][a:a + step] = 2.5 * torch.randn(min(step, B - a), R, V, generator=g, device=dev)
    if case["op"] == "adjust":
        _prepare_adjust(case, st, g, rng, dev)
    else:
        _prepare_distill(case, st, g, rng, dev)
    if own and case["op"] != "adjust":
        from paper_2606_01813_b200 import binding as A
        st["result"] = A.Distilled(loss=st.get("loss"), stats=st.get("stats"), grad=st.get("grad"))
    return st


# ---------------------------------------------------------------------------------------------------------- plain forms

def _plain_adjust(st):
    c = st["case"]
    V, dev = c["vocab"], st["logits"].device
    out = st["logits"] if c["in_place"] else st["out"]
    for b in range(c["batch"]):
        r = st["live"][b]
        for a in range(0, r, 64):                                             # some rows at a time: counts are as large as the logits
            rows = torch.arange(a, min(r, a + 64), device=dev)
            x = st["logits"][b, rows].float()
            if c["penalties"]:
                used = torch.zeros(len(rows), V, device=dev)                  # times that a token was put out
                seen = torch.zeros(V, dtype=torch.bool, device=dev)
                if c["history"]:
                    n = st["history_len"][b]
                    i = torch.arange(c["history"], device=dev)
                    h = st["history"][b].long()
                    used += torch.zeros(V, device=dev).scatter_add_(0, h, ((i < n) & (i >= st["prompt_len"][b])).float())
                    seen = torch.zeros(V, device=dev).scatter_add_(0, h, (i < n).float()) > 0
                if c["tree"]:
                    at = rows
                    for _ in range(TREE_DEPTH + 1):
                        t = st["token_ids"][b, at.clamp(min=0)].long()
                        used.scatter_add_(1, t.clamp(min=0)[:, None], ((at >= 0) & (t >= 0)).float()[:, None])
                        at = torch.where(at >= 0, st["parent_idx"][b, at.clamp(min=0)].long(), -1)
                any_use = seen[None] | (used > 0)
                x = torch.where(any_use, torch.where(x > 0, x / st["repetition"][b], x * st["repetition"][b]), x)
                x = x - st["frequency"][b] * used - st["presence"][b] * (used > 0)
            if c["n_bias"]:
                x[:, st["bias_token"][b].long()] += st["bias"][b]
            if "allowed" in st:
                m = st["allowed_row"][b, rows].long()
                bits = (st["allowed"][m.clamp(min=0)][:, :, None] >> torch.arange(32, dtype=torch.int32, device=dev) & 1).flatten(1)[:, :V].bool()
                x = torch.where(bits | (m < 0)[:, None], x, -math.inf)
            out[b, rows] = x.to(out.dtype)
    return [out]


def _plain_distill(st, want_loss, want_grad):
    c = st["case"]
    for name in ("loss", "stats", "grad"):
        if name in st and not (name == "stats" and c["op"] == "grad"):
            st[name].zero_()
    for b in range(c["batch"]):
        rows = st["rows_of"][b]
        n, T = len(rows), c["temperature"]
        x = st["logits"][b, :n].float()
        t = st["teacher_token"][b, rows].long()
        at, have = t.clamp(min=0), t >= 0
        v = st["teacher_logprob"][b, rows].float()
        w = st["weight"][b, :n]
        if c["op"] == "grad":
            stats = st["stats"][b, :n]
        else:
            stats = _stats(x, t, T)
            if "stats" in st:
                st["stats"][b, :n] = stats
        m, z, m_rest, z_rest = stats.unsqueeze(1).unbind(-1)
        if c["rest"]:
            p = torch.where(have, torch.exp(v), 0.0)
            left = (1.0 - torch.exp(st["teacher_logprob"][b, rows]).sum(-1, keepdim=True)).clamp(min=0.0).float()
        else:
            p = torch.softmax(torch.where(have, v / T, -math.inf), -1)
            left = torch.zeros_like(z)
        if want_loss:
            q = (torch.gather(x, 1, at) - m) / T - torch.log(z)
            loss = torch.where(p > 0, p * (torch.log(p) - q), 0.0).sum(-1)
            q = (m_rest - m) / T + torch.log(z_rest) - torch.log(z)
            loss = loss + torch.where(left > 0, left * (torch.log(left) - q), 0.0).squeeze(-1)
            st["loss"][b, :n] = w * loss
        if want_grad:
            if c["op"] == "grad":
                w = w * st["grad_loss"][b, :n]
            total = p.sum(-1, keepdim=True) + left
            q = torch.exp((x - m) / T) / z
            d = q * total - torch.where(left > 0, left * torch.exp((x - m_rest) / T) / z_rest, 0.0)
            listed = torch.gather(q, 1, at) * total
            d.scatter_(1, torch.where(have, at, at[:, :1]), torch.where(have, listed, listed[:, :1]))
            d.scatter_add_(1, at, -p)
            st["grad"][b, :n] = (d * (w / T)[:, None]).to(st["grad"].dtype)
    return {"loss": [st.get("loss"), st.get("stats")], "grad": [st.get("grad")], "step": [st.get("loss"), st.get("grad")]}[c["op"]]


def run(st):
    c = st["case"]
    if not own:
        if c["op"] == "adjust":
            return _plain_adjust(st)
        return _plain_distill(st, c["op"] != "grad", c["op"] != "loss")
    from paper_2606_01813_b200 import binding as A
    if c["op"] == "adjust":
        out = A.cadd_adjust_logits(st["logits"], n_nodes=st["n_nodes"], token_ids=st.get("token_ids"), parent_idx=st.get("parent_idx"),
                                   history=st.get("history"), history_len=st.get("history_len"), prompt_len=st.get("prompt_len"),
                                   repetition=st.get("repetition"), presence=st.get("presence"), frequency=st.get("frequency"),
                                   bias_token=st.get("bias_token"), bias=st.get("bias"), allowed=st.get("allowed"),
                                   allowed_row=st.get("allowed_row"), out=st.get("out"))
        return [out]
    kw = dict(rest=c["rest"], temperature=c["temperature"], path=st.get("path"), path_len=st.get("path_len"), weight=st["weight"])
    if c["op"] == "grad":
        return [A.cadd_distill_grad(st["logits"], st["teacher_token"], st["teacher_logprob"], st["stats"], grad_loss=st["grad_loss"], grad=st["grad"], **kw)]
    r = A.cadd_distill_loss(st["logits"], st["teacher_token"], st["teacher_logprob"], out=st["result"], **kw)
    return [r.loss, r.stats] if c["op"] == "loss" else [r.loss, r.grad]


# ---------------------------------------------------------------------------------------------------------- 64 bits

def _exact_adjust(case, st):
    B, V = case["batch"], case["vocab"]
    if B * case["rows"] > 3000:
        return None
    dev = st["logits"].device
    out = st["logits"].double() if case["in_place"] else torch.zeros(st["logits"].shape, dtype=torch.float64, device=dev)
    token = st["token_ids"].tolist() if case["tree"] else None
    parent = st["parent_idx"].tolist() if case["tree"] else None
    number = lambda name, b, default: float(st[name][b]) if case["penalties"] else default
    for b in range(B):
        rep, pres, freq = number("repetition", b, 1.0), number("presence", b, 0.0), number("frequency", b, 0.0)
        prompt, said = [], []
        if case["history"]:
            n, q = int(st["history_len"][b]), int(st["prompt_len"][b])
            h = st["history"][b, :n].tolist()
            prompt, said = h[:q], h[q:]
        count = {}
        for t in prompt:
            count.setdefault(t, 0)
        for t in said:
            count[t] = count.get(t, 0) + 1
        biases = dict(zip(st["bias_token"][b].tolist(), st["bias"][b].double().tolist())) if case["n_bias"] else {}
        common = set(count) | set(biases) if case["penalties"] else set(biases)
        ids = torch.tensor(sorted(common), dtype=torch.long, device=dev)
        times = torch.tensor([count.get(t, 0) for t in sorted(common)], dtype=torch.float64, device=dev)
        known = torch.tensor([t in count for t in sorted(common)], dtype=torch.bool, device=dev)
        plus = torch.tensor([biases.get(t, 0.0) for t in sorted(common)], dtype=torch.float64, device=dev)
        for j in range(st["live"][b]):
            y = st["logits"][b, j].double()
            path = []
            if case["tree"] and case["penalties"]:
                a = j
                while a >= 0:
                    path.append(token[b][a])
                    a = parent[b][a]
            fix = [(ids, times, known, plus)]
            if path:
                own_ids = sorted(set(path))
                fix.append((torch.tensor(own_ids, device=dev), torch.tensor([count.get(t, 0) + path.count(t) for t in own_ids], dtype=torch.float64, device=dev),
                            torch.ones(len(own_ids), dtype=torch.bool, device=dev), torch.tensor([biases.get(t, 0.0) for t in own_ids], dtype=torch.float64, device=dev)))
            new = y.clone()
            for i, k, s, p in fix:                                            # the path's own entries come last and replace the common ones
                z = y[i]
                z = torch.where(s, torch.where(z > 0, z / rep, z * rep), z) - freq * k - pres * (k > 0).double() + p
                new[i] = z
            m = int(st["allowed_row"][b, j]) if "allowed" in st else -1
            if m >= 0:
                v = torch.arange(V, device=dev)
                new[(st["allowed"][m][v // 32] >> (v % 32).int()) & 1 == 0] = -math.inf
            out[b, j] = new
    return [out]


def _exact_distill(case, st):
    B, L, T = case["batch"], case["rows"], case["temperature"]
    loss = torch.zeros(B, L, dtype=torch.float64, device=st["logits"].device)
    stats = torch.zeros(B, L, 4, dtype=torch.float64, device=loss.device)
    grad = torch.zeros(st["logits"].shape, dtype=torch.float64, device=loss.device) if case["op"] != "loss" else None
    for b in range(B):
        for i, r in enumerate(st["rows_of"][b]):
            t = st["teacher_token"][b, r].long()
            v = st["teacher_logprob"][b, r][t >= 0]
            t = t[t >= 0]
            x = st["logits"][b, i].double()
            rest = torch.ones(case["vocab"], dtype=torch.bool, device=x.device)
            rest[t] = False
            stats[b, i, 0], stats[b, i, 2] = x.max(), x[rest].max()
            stats[b, i, 1], stats[b, i, 3] = torch.exp((x - x.max()) / T).sum(), torch.exp((x[rest] - x[rest].max()) / T).sum()
            logq = torch.log_softmax(x / T, 0)
            weight = float(st["weight"][b, i]) * (float(st["grad_loss"][b, i]) if case["op"] == "grad" else 1.0)
            logp = v if case["rest"] else torch.log_softmax(v / T, 0)
            p = logp.exp()
            loss[b, i] = weight * (p * (logp - logq[t])).sum()
            q = logq.exp()
            d = q * p.sum()
            d[t] -= p
            if case["rest"]:
                rest = max(0.0, 1.0 - float(p.sum()))
                others = logq.clone()
                others[t] = -math.inf
                log_rest = torch.logsumexp(others, 0)
                if rest > 0:
                    loss[b, i] += weight * rest * (math.log(rest) - log_rest)
                d += rest * (q - torch.exp(others - log_rest))
            if grad is not None:
                grad[b, i] = d * weight / T
    return {"loss": [loss, stats], "grad": [grad], "step": [loss, grad]}[case["op"]]


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_adjust(case, st) if case["op"] == "adjust" else _exact_distill(case, st)
