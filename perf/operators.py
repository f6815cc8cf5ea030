"""Work of the cache and tree-attention operators, for timing and for checking them at real sizes.

Four operators of one decoding round around the draft tree, all over a paged key/value cache that is held in bf16 or in
4 bits (e2m1 codes, one e4m3 scale for 16 of them):

  attention   the rows of a draft tree (or one decoded token, or the rows of a prompt chunk) over the cache and the tree
  append      rows written to the cache (a prompt, or the root and the accepted path), and read back as what they stand for
  weights     attention weight that the accepted rows spend on each cached position, added up
  evict       the positions with the largest weight kept, the others dropped

`run` computes a case in plain torch operations (`own` false) or through the framework's entry points (`own` true)."""
import math
import random

import torch

own = False

FP4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TREE_DEPTH = 16                       # deepest node of a tree: the draft block of the benchmark configurations


# ---------------------------------------------------------------------------------------------------------- cases

def _case(name, op, **kw):
    c = dict(name=name, op=op, batch=1, rows=1, causal=False, heads=8, group=4, dim=128, fp4=True, page=64,
             len_max=1024, window=0, sinks=0, budget=0, recent=0)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one conversation of ordinary length: the smallest call, where latency counts
        _case("token_fp4", "attention", len_max=1000, page=16),
        # one token each for a batch of conversations of very different lengths, small pages
        _case("token_batch_bf16", "attention", batch=64, len_max=8191, page=16, fp4=False),
        # trees of up to 64 nodes for a batch with long contexts: the ordinary round of a speculating server
        _case("tree_batch_fp4", "attention", batch=32, rows=65, len_max=32768),
        # trees at the node cap of 256 over a sliding window with sinks, eight query heads to a key head
        _case("tree_window_bf16", "attention", batch=16, rows=257, len_max=20011, heads=4, group=8, window=4096, sinks=4, fp4=False, page=32),
        # trees of a thousand nodes: arithmetic, not memory
        _case("tree_thousand_fp4", "attention", batch=4, rows=1025, len_max=16384, page=128),
        # a prompt chunk behind an earlier part of the prompt, head dimension 64, no grouping
        _case("chunk_bf16", "attention", batch=2, rows=2000, causal=True, heads=12, group=1, dim=64, len_max=6001, fp4=False, page=16),
        # commit of a round: the root and the accepted path of each request of a large batch
        _case("commit_fp4", "append", batch=256, rows=385, len_max=4096, page=32),
        # prompts written to the cache
        _case("prompt_fp4", "append", batch=6, rows=8000, causal=True, len_max=0),
        # the accepted rows' weights: one request, and a batch with long contexts
        _case("weights_bf16", "weights", batch=2, rows=33, len_max=5000, fp4=False, page=16),
        _case("weights_fp4", "weights", batch=32, rows=65, len_max=32768),
        # eviction: one conversation just over its budget, and a batch cut to a quarter
        _case("evict_bf16", "evict", batch=1, len_max=1100, budget=1024, sinks=4, recent=64, fp4=False, page=16),
        _case("evict_fp4", "evict", batch=24, len_max=32000, budget=8192, sinks=4, recent=256),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    cap = {}
    for c in listed():
        w = work(c)
        o = cap.setdefault(c["op"], [0, 0])
        o[0], o[1] = max(o[0], w["bytes"]), max(o[1], w["flops"])
    op = rng.choice(["attention", "attention", "append", "weights", "evict"])
    while True:
        dim, group = rng.choice([64, 128]), rng.choice([1, 2, 3, 4, 5, 7, 8])
        c = _case("", op, batch=_log_int(rng, 1, 64), heads=rng.choice([1, 2, 4, 8]), group=group, dim=dim, fp4=rng.random() < 0.5,
                  page=rng.choice([16, 32, 64, 128, 256]), len_max=_log_int(rng, 30, 32768))
        if op == "attention":
            c["rows"] = rng.choice([1, _log_int(rng, 2, 1025)])
            c["causal"] = rng.random() < 0.25
            if rng.random() < 0.4:
                c["window"], c["sinks"] = _log_int(rng, 8, 8192), rng.choice([0, 1, 4, 129])
        elif op == "append":
            c["rows"] = _log_int(rng, 1, 8000 if dim == 64 else 4000)
            c["causal"] = rng.random() < 0.5
        elif op == "weights":
            c["rows"] = _log_int(rng, 1, 257)
            if rng.random() < 0.3:
                c["window"], c["sinks"] = _log_int(rng, 8, 8192), rng.choice([0, 1, 4, 129])
        else:
            c["budget"] = _log_int(rng, 16, 16384)
            c["sinks"], c["recent"] = rng.choice([0, 1, 4, 8]), rng.choice([0, 1, 8])
        w = work(c)
        if w["bytes"] <= cap[op][0] and w["flops"] <= cap[op][1]:
            del c["name"]
            return c


def _lengths(case):
    """Cached tokens of each request: ragged, the longest is len_max, in a large batch one is empty."""
    rng = random.Random(case["batch"] * 1000003 + case["len_max"])
    n = [rng.randint(case["len_max"] // 4, case["len_max"]) for _ in range(case["batch"])]
    n[0] = case["len_max"]
    if case["batch"] > 8:
        n[5] = 0
    return n


def _live(case):
    """Rows in use of each request (the root among them)."""
    rng = random.Random(case["batch"] * 7919 + case["rows"])
    n = [rng.randint(max(1, case["rows"] // 3), case["rows"]) for _ in range(case["batch"])]
    n[-1] = case["rows"]
    return n


def _path_lens(case):
    """Accepted nodes of each request's path, root not counted."""
    rng = random.Random(case["batch"] * 104729 + case["rows"])
    return [min(rng.choice([0, 1, 2, 3, 4, 6, 8, 12]), n - 1) for n in _live(case)]


def _row_bytes(case):
    """Bytes of one cached key (or value) row of one head."""
    return case["dim"] // 2 + case["dim"] // 16 if case["fp4"] else case["dim"] * 2


def _visible(case, n):
    return min(n, case["window"] + case["sinks"]) if case["window"] else n


def work(case):
    h, d, hq = case["heads"], case["dim"], case["heads"] * case["group"]
    lens, row = _lengths(case), _row_bytes(case)
    if case["op"] == "attention":
        live = _live(case)
        nbytes = flops = 0
        for n, r in zip(lens, live):
            seen = _visible(case, n)
            pairs = r * (r + 1) // 2 if case["causal"] else r * min(r, TREE_DEPTH)
            nbytes += seen * h * 2 * row + r * (2 * hq + 2 * h) * d * 2 + r * hq * 4 + (n + case["page"] - 1) // case["page"] * 4
            flops += 4 * d * hq * (r * seen + pairs)
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "append":
        rows = sum(_live(case)) if case["causal"] else sum(p + 1 for p in _path_lens(case))
        return {"bytes": rows * h * 2 * (2 * d * 2 + 2 * row), "flops": rows * h * 2 * d * 4}
    if case["op"] == "weights":
        nbytes = flops = 0
        for n, p in zip(lens, _path_lens(case)):
            seen = _visible(case, n) + p + 1
            nbytes += seen * h * row + (n + p + 1) * h * 8 + (p + 1) * hq * (d * 2 + 4)
            flops += 2 * d * hq * (p + 1) * seen
        return {"bytes": nbytes, "flops": flops}
    kept = sum(min(n, case["budget"]) for n in lens)
    return {"bytes": sum(lens) * h * 4 + kept * h * (4 * row + 8), "flops": sum(lens) * h * 4}


# ---------------------------------------------------------------------------------------------------------- inputs

def _quantize(x):
    """fp32 [..., D] -> codes uint8 [..., D/2] (the even element in the low four bits), scales e4m3 as uint8 [..., D/16]."""
    b = x.unflatten(-1, (-1, 16))
    s = (b.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    sf = s.float().unsqueeze(-1)
    y = torch.where(sf > 0, b / torch.where(sf > 0, sf, 1.0), 0.0)
    a = y.abs()
    # nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a value half way goes to the even code
    c = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
         + (a > 5.0).byte())
    c = (c | ((y < 0) & (c > 0)).byte() * 8).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s.view(torch.uint8)


def _values(codes, scales, dtype):
    """The numbers that codes and scales stand for."""
    table = torch.tensor(FP4_VALUES + tuple(-v for v in FP4_VALUES), dtype=dtype, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    s = scales.view(torch.float8_e4m3fn).to(dtype).unsqueeze(-1)
    return (table[c.int()].unflatten(-1, (-1, 16)) * s).flatten(-2)


def _tree(rows, live, rng):
    """Parents of a random tree in the order in which best-first growth adds nodes, and depths."""
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
    return parent, depth


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    B, R, H, G, D, P = case["batch"], case["rows"], case["heads"], case["group"], case["dim"], case["page"]
    lens = _lengths(case)
    live = _live(case)
    st = dict(case=case, lens=lens, live=live, scale=1.0 / math.sqrt(D))
    grow = R if case["op"] in ("append", "weights") else 0
    if case["op"] in ("append", "weights") and not case["causal"]:
        grow = TREE_DEPTH + 1
    pages = [(n + grow + P - 1) // P for n in lens]
    total = sum(pages)
    new_pages = [(min(n, case["budget"]) + P - 1) // P for n in lens] if case["op"] == "evict" else [0] * B
    n_pages = total + sum(new_pages)
    # pages of the requests in shuffled order, as an allocator leaves them
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.zeros(B, max(max(pages), 1), dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = torch.tensor(order[at:at + pages[b]], dtype=torch.int32)
        at += pages[b]
    st["block_table"], st["pages"] = table.to(dev), pages
    st["length"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    channel = 0.5 + torch.rand(2, H, 1, D, generator=g, device=dev)           # some channels are larger than others
    st["pool"] = []
    for i in range(2):
        if case["fp4"]:
            codes = torch.zeros(n_pages, H, P, D // 2, dtype=torch.uint8, device=dev)
            scales = torch.zeros(n_pages, H, P, D // 16, dtype=torch.uint8, device=dev)
            step = max(1, (1 << 26) // (H * P * D))
            for a in range(0, total, step):
                e = min(total, a + step)
                x = torch.randn(e - a, H, P, D, generator=g, device=dev) * channel[i]
                codes[a:e], scales[a:e] = _quantize(x)
            st["pool"].append((codes, scales))
        else:
            x = torch.zeros(n_pages, H, P, D, dtype=torch.bfloat16, device=dev)
            step = max(1, (1 << 26) // (H * P * D))
            for a in range(0, total, step):
                e = min(total, a + step)
                x[a:e] = torch.randn(e - a, H, P, D, generator=g, device=dev) * channel[i]
            st["pool"].append((x, None))
    if case["op"] != "evict":
        st["q"] = (2.0 * torch.randn(B, R, H * G, D, generator=g, device=dev)).bfloat16() if case["op"] != "append" else None
        st["k"] = (torch.randn(B, R, H, D, generator=g, device=dev) * channel[0, :, 0]).bfloat16()
        st["v"] = (torch.randn(B, R, H, D, generator=g, device=dev) * channel[1, :, 0]).bfloat16()
        st["n_nodes"] = torch.tensor([n - 1 for n in live], dtype=torch.int32, device=dev)
        st["n_rows"] = torch.tensor(live, dtype=torch.int32, device=dev)
    if case["op"] == "attention" and not case["causal"]:
        W = (R + 31) // 32
        dense = torch.zeros(B, R, W * 32, dtype=torch.uint8)
        depth = torch.zeros(B, R, dtype=torch.int32)
        for b in range(B):
            parent, dep = _tree(R, live[b], rng)
            m = dense[b].numpy()
            m[0, 0] = 1
            for j in range(1, live[b]):
                m[j] = m[parent[j]]
                m[j, j] = 1
            depth[b] = torch.tensor(dep, dtype=torch.int32)
        st["mask"] = dense[:, :, :R].bool().to(dev)
        bits = dense.view(B, R, W, 32).to(dev).long() << torch.arange(32, device=dev)
        bits = bits.sum(-1)
        st["mask_bits"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
        st["depth"] = depth.to(dev)
    if case["op"] == "attention":
        st["out"] = torch.zeros(B, R, H * G, D, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.zeros(B, R, H * G, dtype=torch.float32, device=dev)
    if case["op"] in ("append", "weights") and not case["causal"]:
        plen = _path_lens(case)
        path = torch.full((B, TREE_DEPTH), -1, dtype=torch.int32)
        for b in range(B):
            path[b, :plen[b]] = torch.tensor(sorted(rng.sample(range(1, live[b]), plen[b])), dtype=torch.int32)
        st["path"], st["path_len"] = path.to(dev), torch.tensor(plen, dtype=torch.int32, device=dev)
        st["path_rows"] = [[0] + path[b, :plen[b]].tolist() for b in range(B)]
    elif case["op"] == "append":
        st["path_rows"] = [list(range(live[b])) for b in range(B)]
    if case["op"] == "append":
        n_max = R if case["causal"] else TREE_DEPTH + 1
        st["n_max"] = n_max
        st["count"] = torch.tensor([len(r) for r in st["path_rows"]], dtype=torch.int32, device=dev)
        st["out_k"] = torch.zeros(B, n_max, H, D, dtype=torch.bfloat16, device=dev)
        st["out_v"] = torch.zeros(B, n_max, H, D, dtype=torch.bfloat16, device=dev)
        st["new_length"] = torch.zeros(B, dtype=torch.int32, device=dev)
    if case["op"] == "weights":
        st["base"] = st["length"]
        st["length"] = st["base"] + st["path_len"] + 1                       # the accepted rows have been appended
        cap = table.shape[1] * P
        st["weights"] = torch.rand(B, H, cap, generator=g, device=dev) * 0.5
        st["weights_out"] = torch.zeros(B, H, cap, device=dev)
        st["lse"] = torch.zeros(B, R, H * G, device=dev)
        for b in range(B):                                                   # what the attention of the round left
            s = _path_scores(st, b, torch.float32)
            st["lse"][b, st["path_rows"][b]] = torch.logsumexp(s, -1).permute(1, 0, 2).flatten(1)
    if case["op"] == "evict":
        table2 = torch.zeros(B, max(max(new_pages), 1), dtype=torch.int32)
        at = total
        for b in range(B):
            table2[b, :new_pages[b]] = torch.arange(at, at + new_pages[b], dtype=torch.int32)
            at += new_pages[b]
        st["new_table"], st["first_new"] = table2.to(dev), total
        cap = table.shape[1] * P
        # a few heavy positions over a long light tail, among them equal ones and ones that never got any weight
        w = torch.rand(B, H, cap, generator=g, device=dev).pow_(8.0)
        w = torch.where(w < 1e-4, 0.0, w)
        st["weights"] = torch.where(torch.rand(B, H, cap, generator=g, device=dev) < 0.2, (w * 64).round() / 64, w)
        st["out"] = dict(new_length=torch.zeros(B, dtype=torch.int32, device=dev),
                         weights=torch.zeros(B, H, case["budget"], device=dev),
                         kept=torch.zeros(B, H, case["budget"], dtype=torch.int32, device=dev))
    if own:
        from paper_2606_01813_b200 import binding as A
        (k, ks), (v, vs) = st["pool"]
        st["cache"] = A.KvCache(k=k, v=v, block_table=st["block_table"], length=st["length"], k_scale=ks, v_scale=vs)
        if case["op"] == "attention":
            n = A.cadd_tree_attention_workspace_bytes(B, R, H * G, st["cache"])
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device=dev)
            st["result"] = A.Attention(out=st["out"], lse=st["lse"], status=torch.zeros(B, dtype=torch.int32, device=dev))
        if case["op"] == "evict":
            st["result"] = A.Evicted(status=torch.zeros(B, dtype=torch.int32, device=dev), **st["out"])
    return st


# ---------------------------------------------------------------------------------------------------------- plain forms

def _cached(st, which, b, n, dtype=torch.float32):
    """Rows 0..n-1 of request b's cached keys (0) or values (1): [heads, n, D]."""
    data, scales = st["pool"][which]
    P = st["case"]["page"]
    pages = st["block_table"][b, :(n + P - 1) // P].long()
    x = _values(data[pages], scales[pages], dtype) if scales is not None else data[pages].to(dtype)
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def _path_scores(st, b, dtype):
    """Scores of the accepted rows: [heads, rows, group, positions], -inf where a row does not see a position."""
    c = st["case"]
    rows, base = st["path_rows"][b], st["lens"][b]
    n = base + len(rows)
    q = st["q"][b, rows].to(dtype).unflatten(1, (c["heads"], c["group"])).permute(1, 0, 2, 3)
    s = torch.matmul(q.flatten(1, 2), _cached(st, 0, b, n, dtype).transpose(1, 2)).unflatten(1, (len(rows), c["group"])) * st["scale"]
    p = torch.arange(n, device=s.device)
    me = base + torch.arange(len(rows), device=s.device)
    see = p[None, :] <= me[:, None]
    if c["window"]:
        see = see & ((p[None, :] > me[:, None] - c["window"]) | (p[None, :] < c["sinks"]))
    return s.masked_fill(~see[None, :, None, :], -math.inf)


def _plain_attention(st):
    c = st["case"]
    for b in range(c["batch"]):
        n, r = st["lens"][b], st["live"][b]
        k = torch.cat([_cached(st, 0, b, n), st["k"][b, :r].float().transpose(0, 1)], 1)
        v = torch.cat([_cached(st, 1, b, n), st["v"][b, :r].float().transpose(0, 1)], 1)
        q = st["q"][b, :r].float().unflatten(1, (c["heads"], c["group"])).permute(1, 0, 2, 3)
        i = torch.arange(r, device=k.device)
        depth = i if c["causal"] else st["depth"][b, :r]
        tree = i[None, :] <= i[:, None] if c["causal"] else st["mask"][b, :r, :r]
        p = torch.arange(n, device=k.device)
        ctx = torch.ones(r, n, dtype=torch.bool, device=k.device)
        if c["window"]:
            ctx = (p[None, :] > (n + depth - c["window"])[:, None]) | (p[None, :] < c["sinks"])
            tree = tree & ((depth[:, None] - depth[None, :] < c["window"]) | ((n + depth)[None, :] < c["sinks"]))
        see = torch.cat([ctx, tree], 1)
        for h in range(c["heads"]):                                           # a head at a time: the scores of a large tree are large
            s = (torch.matmul(q[h].flatten(0, 1), k[h].t()) * st["scale"]).unflatten(0, (r, c["group"]))
            s = s.masked_fill(~see[:, None, :], -math.inf)
            m = s.amax(-1, keepdim=True)
            e = torch.exp(s - m)
            z = e.sum(-1, keepdim=True)
            o = torch.matmul(e.flatten(0, 1), v[h]).unflatten(0, (r, c["group"])) / z
            cols = slice(h * c["group"], (h + 1) * c["group"])
            st["out"][b, :r, cols] = o.bfloat16()
            st["lse"][b, :r, cols] = (m + torch.log(z)).squeeze(-1)
    return [st["out"], st["lse"]]


def _plain_append(st):
    c, P = st["case"], st["case"]["page"]
    for b in range(c["batch"]):
        rows = torch.tensor(st["path_rows"][b], device=st["k"].device)
        pos = st["lens"][b] + torch.arange(len(rows), device=rows.device)
        page, slot = st["block_table"][b, pos // P].long(), pos % P
        for which, name, out in ((0, "k", st["out_k"]), (1, "v", st["out_v"])):
            data, scales = st["pool"][which]
            x = st[name][b, rows]
            if scales is None:
                data[page, :, slot] = x
                out[b, :len(rows)] = data[page, :, slot]
            else:
                data[page, :, slot], scales[page, :, slot] = _quantize(x.float())
                out[b, :len(rows)] = _values(data[page, :, slot], scales[page, :, slot], torch.float32).bfloat16()
    torch.add(st["length"], st["count"], out=st["new_length"])
    return [st["out_k"], st["out_v"], st["new_length"]]


def _plain_weights(st):
    st["weights_out"].copy_(st["weights"])
    c = st["case"]
    for b in range(c["batch"]):
        rows, n = st["path_rows"][b], st["lens"][b]
        lse = st["lse"][b, rows].unflatten(1, (c["heads"], c["group"])).permute(1, 0, 2).unsqueeze(-1)
        w = torch.exp(_path_scores(st, b, torch.float32) - lse).sum((1, 2))
        st["weights_out"][b, :, :n] += w[:, :n]
        st["weights_out"][b, :, n:n + len(rows)] = w[:, n:]
    return [st["weights_out"]]


def _plain_evict(st):
    c, P, o = st["case"], st["case"]["page"], st["out"]
    for b in range(c["batch"]):
        n = st["lens"][b]
        keep = min(n, c["budget"])
        o["new_length"][b] = keep
        o["kept"][b] = -1
        if keep == 0:
            continue
        w = st["weights"][b, :, :n]
        key = w.clone()
        if n > c["budget"]:
            key[:, :c["sinks"]] = math.inf
            key[:, n - c["recent"]:] = math.inf
        kept = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :keep].sort(1).values
        o["kept"][b, :, :keep] = kept
        o["weights"][b, :, :keep] = torch.gather(w, 1, kept)
        page, slot = st["block_table"][b, kept // P].long(), kept % P
        to = torch.arange(keep, device=w.device)
        to_page, to_slot = st["new_table"][b, to // P].long()[None], (to % P)[None]
        h = torch.arange(c["heads"], device=w.device)[:, None]
        for data, scales in st["pool"]:
            for t in (data, scales):
                if t is not None:
                    t[to_page, h, to_slot] = t[page, h, slot]
    return _evicted(st)


def _evicted(st):
    o = st["out"]
    return [o["new_length"], o["kept"], o["weights"]] + [t[st["first_new"]:] for pair in st["pool"] for t in pair if t is not None]


def run(st):
    c = st["case"]
    if not own:
        return {"attention": _plain_attention, "append": _plain_append, "weights": _plain_weights, "evict": _plain_evict}[c["op"]](st)
    from paper_2606_01813_b200 import binding as A
    cache = st["cache"]
    if c["op"] == "attention":
        A.cadd_tree_attention(st["q"], st["k"], st["v"], cache, mask_bits=st.get("mask_bits"), n_nodes=st["n_nodes"],
                              depth=st.get("depth"), scale=st["scale"], window=c["window"], n_sinks=c["sinks"], out=st["result"],
                              workspace=st["workspace"])
        return [st["out"], st["lse"]]
    if c["op"] == "append":
        if c["causal"]:
            A.cadd_cache_append(cache, st["k"], st["v"], n_rows=st["n_rows"], new_length=st["new_length"])
        else:
            A.cadd_cache_append(cache, st["k"], st["v"], path=st["path"], path_len=st["path_len"], new_length=st["new_length"])
        after = A.KvCache(k=cache.k, v=cache.v, block_table=cache.block_table, length=st["new_length"], k_scale=cache.k_scale,
                          v_scale=cache.v_scale)
        A.cadd_cache_read(after, st["n_max"], start=st["length"], out=(st["out_k"], st["out_v"]))
        return [st["out_k"], st["out_v"], st["new_length"]]
    if c["op"] == "weights":
        A.cadd_cache_weights(st["q"], st["lse"], cache, st["base"], st["weights"], path=st["path"], path_len=st["path_len"],
                             scale=st["scale"], window=c["window"], n_sinks=c["sinks"], out=st["weights_out"])
        return [st["weights_out"]]
    A.cadd_cache_evict(cache, st["weights"], st["new_table"], c["budget"], n_sinks=c["sinks"], n_recent=c["recent"], out=st["result"])
    return _evicted(st)


# ---------------------------------------------------------------------------------------------------------- 64 bits

def _rows64(st, which, b, n):
    """Request b's first n cached rows in 64 bits, token by token from the pages: [n, heads, D]."""
    data, scales = st["pool"][which]
    P = st["case"]["page"]
    pos = torch.arange(n, device=data.device)
    page, slot = st["block_table"][b].long()[pos // P], pos % P
    x = data[page, :, slot]
    if scales is None:
        return x.double()
    grid = torch.tensor(FP4_VALUES, dtype=torch.float64, device=x.device)
    lo, hi = (x & 15).long(), (x >> 4).long()
    val = torch.empty(*x.shape[:-1], 2 * x.shape[-1], dtype=torch.float64, device=x.device)
    for at, code in ((0, lo), (1, hi)):
        val[..., at::2] = grid[code & 7] * (1 - 2 * (code >> 3)).double()
    s = scales[page, :, slot].view(torch.float8_e4m3fn).double()
    return val * s.repeat_interleave(16, -1)


def exact(case, seed):
    st = prepare(case, seed)
    B, H, G, D, P = case["batch"], case["heads"], case["group"], case["dim"], case["page"]
    dev = st["length"].device
    if case["op"] == "attention":
        out = torch.zeros(B, case["rows"], H * G, D, dtype=torch.float64, device=dev)
        lse = torch.zeros(B, case["rows"], H * G, dtype=torch.float64, device=dev)
        for b in range(B):
            n, r = st["lens"][b], st["live"][b]
            k = torch.cat([_rows64(st, 0, b, n), st["k"][b, :r].double()])
            v = torch.cat([_rows64(st, 1, b, n), st["v"][b, :r].double()])
            row = torch.arange(r, device=dev)
            dep = row if case["causal"] else st["depth"][b, :r].long()
            # place of every key in the sequence, and whether a row sees it
            place = torch.cat([torch.arange(n, device=dev), n + dep])
            hidden = torch.zeros(r, n + r, dtype=torch.bool, device=dev)
            hidden[:, n:] = row[None] > row[:, None] if case["causal"] else ~st["mask"][b, :r, :r]
            if case["window"]:
                hidden |= ((n + dep)[:, None] - place[None] >= case["window"]) & (place[None] >= case["sinks"])
            for hq in range(H * G):
                x = st["q"][b, :r, hq].double() @ k[:, hq // G].t() * st["scale"]
                x[hidden] = -math.inf
                lse[b, :r, hq] = torch.logsumexp(x, 1)
                out[b, :r, hq] = torch.softmax(x, 1) @ v[:, hq // G]
        return [out, lse]
    if case["op"] == "append":
        res = [torch.zeros(B, st["n_max"], H, D, dtype=torch.float64, device=dev) for _ in range(2)]
        grid = torch.tensor(FP4_VALUES, dtype=torch.float64, device=dev)
        for b in range(B):
            rows = torch.tensor(st["path_rows"][b], device=dev)
            for o, x in zip(res, (st["k"], st["v"])):
                x = x[b, rows].double()
                if case["fp4"]:
                    x = x.unflatten(-1, (-1, 16))
                    s = (x.abs().amax(-1, keepdim=True) / 6).clamp(max=448)
                    # e4m3 in 64 bits: three bits behind the leading one, steps of 2^-9 below 2^-6
                    step = torch.exp2(torch.floor(torch.log2(s.clamp(min=2.0 ** -6))) - 3)
                    s = torch.round(s / step) * step
                    y = torch.where(s > 0, x / s.clamp(min=2.0 ** -9), 0.0)
                    mag = y.abs().clamp(max=6)
                    low = (torch.searchsorted(grid, mag, right=True) - 1).clamp(max=6)
                    up, down = grid[low + 1] - mag, mag - grid[low]
                    code = torch.where((up < down) | ((up == down) & (low % 2 == 1)), low + 1, low)
                    x = (grid[code] * y.sign() * s).flatten(-2)
                o[b, :len(rows)] = x
        return res + [(st["length"] + st["count"])]
    if case["op"] == "weights":
        w = st["weights"].double()
        for b in range(B):
            rows, n = st["path_rows"][b], st["lens"][b]
            k = _rows64(st, 0, b, n + len(rows))
            w[b, :, n:n + len(rows)] = 0
            for i, r in enumerate(rows):
                place = torch.arange(n + i + 1, device=dev)
                seen = place[(place > n + i - case["window"]) | (place < case["sinks"])] if case["window"] else place
                for h in range(H):
                    q = st["q"][b, r, h * G:(h + 1) * G].double()
                    x = k[seen, h] @ q.t() * st["scale"] - st["lse"][b, r, h * G:(h + 1) * G].double()
                    w[b, h, seen] += torch.exp(x).sum(1)
        return [w]
    # eviction moves numbers as they are: positions by weight, then by place
    pools = [t.clone()[st["first_new"]:] for pair in st["pool"] for t in pair if t is not None]
    source = [t for pair in st["pool"] for t in pair if t is not None]
    length = torch.zeros(B, dtype=torch.int32, device=dev)
    kept = torch.full((B, H, case["budget"]), -1, dtype=torch.int32, device=dev)
    weights = torch.zeros(B, H, case["budget"], device=dev)
    for b in range(B):
        n = st["lens"][b]
        keep = min(n, case["budget"])
        length[b] = keep
        for h in range(H):
            w = st["weights"][b, h, :n].double()
            if n > keep:
                inner = torch.arange(case["sinks"], n - case["recent"], device=dev)
                left = keep - case["sinks"] - case["recent"]
                by_weight = inner[torch.argsort(-w[inner], stable=True)[:left]]
                pos = torch.cat([torch.arange(case["sinks"], device=dev), by_weight, torch.arange(n - case["recent"], n, device=dev)]).sort().values
            else:
                pos = torch.arange(n, device=dev)
            kept[b, h, :keep] = pos.int()
            weights[b, h, :keep] = w[pos].float()
            i = torch.arange(keep, device=dev)
            for dst, src in zip(pools, source):
                dst[st["new_table"][b].long()[i // P] - st["first_new"], h, i % P] = src[st["block_table"][b].long()[pos // P], h, pos % P]
    return [length, kept, weights] + pools
