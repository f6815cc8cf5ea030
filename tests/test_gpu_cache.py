"""The cache calls against their definitions in 64 bits: rows written and read back in both forms, weights added up, eviction;
and the calls of a whole round one after the other."""
import math

import pytest
import torch

from paper_2606_01813_b200 import binding as G
from cache_util import Problem, decode, encode

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def problem(**kw):
    d = dict(batch=2, heads=2, group=2, dim=128, page=16, fp4=False, lens=[70, 33], R=5, live=[5, 3], causal=False, seed=1, extra_places=64)
    d.update(kw)
    return Problem(**d)


def stored(x, fp4, exp=0):
    """What the cache stands for after rows x (bf16) have been written."""
    return decode(*encode(x.double(), exp), exp) if fp4 else x.double()


def read_all(cache, n_max):
    k, v = G.cadd_cache_read(cache, n_max)
    return k.cpu().double(), v.cpu().double()


def at_length(c, length):
    return G.KvCache(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, block_table=c.block_table, length=length, k_exp=c.k_exp, v_exp=c.v_exp)


# ---- append and read ----

@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [1, 4, 16, 64, 256])
@pytest.mark.parametrize("token_major", [False, True])
def test_read_gives_what_the_cache_stands_for(fp4, dim, page, token_major):
    p = problem(fp4=fp4, dim=dim, page=page, lens=[70, 0, 1, 129], batch=4, live=[1] * 4, heads=3, token_major=token_major)
    c = p.cache(G)
    k, v = read_all(c, 140)
    for b, n in enumerate(p.lens):
        assert torch.equal(k[b, :n], p.K[b]) and torch.equal(v[b, :n], p.V[b])
        assert bool((k[b, n:] == 0).all())
    out = tuple(torch.full((4, 9, 3, dim), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    status = i32([9] * 4)
    G.cadd_cache_read(c, 9, start=i32([66, 0, 0, 120]), count=i32([3, 2, 1, 50]), out=out, status=status)
    assert status.tolist() == [0, G.STATUS_BAD_LENGTH, 0, 0]
    for b, (s, n) in enumerate(((66, 3), (0, 0), (0, 1), (120, 9))):
        assert torch.equal(out[0][b, :n].cpu().double(), p.K[b][s:s + n]) and torch.equal(out[1][b, :n].cpu().double(), p.V[b][s:s + n])
        assert bool((out[0][b, n:] == 5.0).all()) and bool((out[1][b, n:] == 5.0).all())


def awkward_rows(n, H, D, g):
    """Rows whose blocks are zero, tiny, huge, half way between codes, with NaN and infinities among them."""
    x = torch.randn(n, H, D, generator=g, dtype=torch.float64)
    x[0] = 0.0
    x[1] *= 2.0 ** -14
    x[2] *= 2.0 ** 14
    x[3] = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 5.5, 6], dtype=torch.float64).repeat(D // 16) * 2.0 ** -3
    x[4] = -x[3] * 7
    x[5, :, 3] = math.nan
    x[6, :, 20] = math.inf
    x[7, :, 5] = -math.inf
    x[8] = math.nan
    x[9] = x[9].sign() * 2.0 ** -10
    return x.bfloat16()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("exps", [(0, 0), (4, -3), (-16, 16)])
def test_append_stores_the_nearest_codes(fp4, dim, exps):
    if not fp4 and exps != (0, 0):
        exps = (0, 0)
    p = problem(fp4=fp4, dim=dim, lens=[5, 0], R=40, live=[40, 40], k_exp=exps[0], v_exp=exps[1], page=8)
    for b in range(2):
        p.k[b, :10], p.v[b, 3:13] = awkward_rows(10, 2, dim, p.g), awkward_rows(10, 2, dim, p.g)
    c = p.cache(G)
    before = [t.clone() for t in ((c.k, c.v, c.k_scale, c.v_scale) if fp4 else (c.k, c.v))]
    status = i32([7, 7])
    n = G.cadd_cache_append(c, p.k.to(DEV), p.v.to(DEV), n_rows=i32([40, 23]), status=status)
    assert n.tolist() == [45, 23] and status.tolist() == [0, 0] and c.length.tolist() == [5, 0]
    k, v = read_all(at_length(c, n), 50)
    for b, (s, m) in enumerate(((5, 40), (0, 23))):
        for got, src, old, exp in ((k, p.k, p.K, exps[0]), (v, p.v, p.V, exps[1])):
            want = stored(src[b, :m], fp4, exp)
            assert torch.equal(torch.nan_to_num(got[b, s:s + m], nan=123.0), torch.nan_to_num(want, nan=123.0))
            assert torch.equal(got[b, :s], old[b])
    # nothing else in the pools has changed
    for t, old in zip((c.k, c.v, c.k_scale, c.v_scale), before):
        changed = (t.cpu().view(torch.uint8) != old.cpu().view(torch.uint8)).flatten(3).any(-1)             # [page, head, slot]
        allowed = torch.zeros_like(changed)
        for b, (s, m) in enumerate(((5, 40), (0, 23))):
            for pos in range(s, s + m):
                allowed[int(p.block_table[b, pos // 8]), :, pos % 8] = True
        assert not bool((changed & ~allowed).any())


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_an_accepted_path(fp4, in_place):
    p = problem(fp4=fp4, batch=4, lens=[10, 31, 0, 64], R=30, live=[30] * 4, heads=1, page=16)
    path = torch.full((4, 6), -1, dtype=torch.int32)
    path[1, :3] = torch.tensor([4, 9, 29])
    path[2, :6] = torch.tensor([1, 2, 3, 5, 8, 13])
    path[3, :2] = torch.tensor([7, 7])                                     # the same row twice
    lens = [0, 3, 6, 2]
    c = p.cache(G)
    n = G.cadd_cache_append(c, p.k.to(DEV), p.v.to(DEV), path=path.to(DEV), path_len=i32(lens), new_length=c.length if in_place else None)
    assert n.tolist() == [11, 35, 7, 67]
    assert c.length.tolist() == (n.tolist() if in_place else p.lens)
    k, v = read_all(at_length(c, n), 70)
    for b in range(4):
        rows = [0] + path[b, :lens[b]].tolist()
        s = p.lens[b]
        assert torch.equal(k[b, s:s + len(rows)], stored(p.k[b, rows], fp4)) and torch.equal(v[b, s:s + len(rows)], stored(p.v[b, rows], fp4))
        assert torch.equal(k[b, :s], p.K[b])


def test_append_flags_what_it_cannot_store():
    p = problem(batch=5, lens=[10] * 5, R=8, live=[8] * 5, extra_places=0, page=4)      # capacity 12
    table = p.block_table.clone()
    table[1, 2] = p.n_pages
    c0 = p.cache(G)
    c = G.KvCache(k=c0.k, v=c0.v, block_table=table.to(DEV), length=i32([10, 10, 10, 900, -4]))
    path = torch.zeros(5, 3, dtype=torch.int32)
    path[2, 0] = 8
    path[4, 1] = -2
    before = c.k.clone()
    status = i32([0] * 5)
    n = G.cadd_cache_append(c, p.k.to(DEV), p.v.to(DEV), path=path.to(DEV), path_len=i32([3, 1, 1, 0, 2]), status=status)
    assert n.tolist() == [12, 12, 12, 12, 3]
    assert status.tolist() == [G.STATUS_CACHE_FULL, G.STATUS_BAD_PAGE, G.STATUS_BAD_PATH, G.STATUS_CACHE_FULL | G.STATUS_BAD_LENGTH,
                               G.STATUS_BAD_PATH | G.STATUS_BAD_LENGTH]
    changed = (c.k.view(torch.int16) != before.view(torch.int16)).flatten(3).any(-1).cpu()
    want = torch.zeros_like(changed)
    for b, pos in ((0, 10), (0, 11), (2, 10), (4, 0), (4, 1)):             # entry 2 of request 4 is the bad row
        want[int(p.block_table[b, pos // 4]), :, pos % 4] = True
    assert torch.equal(changed, want)
    status2 = i32([0] * 5)
    G.cadd_cache_append(c, p.k.to(DEV), p.v.to(DEV), n_rows=i32([-1, 0, 9, 0, 0]), status=status2)
    assert status2.tolist() == [G.STATUS_BAD_LENGTH, 0, G.STATUS_BAD_LENGTH | G.STATUS_CACHE_FULL, G.STATUS_BAD_LENGTH, G.STATUS_BAD_LENGTH]


# ---- weights ----

def weights_wanted(p, base, rows, lse, w, window=0, sinks=0):
    """Running totals after the rows' weights, and how far fp32 may be off: lists over requests of [heads, length]."""
    res, tol = [], []
    for b in range(p.batch):
        n = base[b] + len(rows[b])
        total = torch.zeros(p.heads, n, dtype=torch.float64)
        total[:, :base[b]] = w[b, :, :base[b]].double()
        slack = total.abs() * 2.0 ** -24 * (len(rows[b]) * p.group + 1)
        for i, r in enumerate(rows[b]):
            place, me = torch.arange(n), base[b] + i
            see = place <= me
            if window:
                see &= (me - place < window) | (place < sinks)
            for h in range(p.heads * p.group):
                e = float(lse[b, r, h])
                if math.isinf(e):
                    continue
                q, k = p.q[b, r, h].double(), p.K[b][:, h // p.group]
                x = torch.where(see, torch.exp(k @ q * p.scale - e), 0.0)
                total[h // p.group] += x
                # a score is off by scale sum|q k| (dim + 4) 2^-24, its difference to lse by 2^-24 (|s| + |lse|) log2(e) twice, exp2 by 2^-20
                ds = p.scale * (k.abs() @ q.abs()) * (p.dim + 4) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * ((k @ q * p.scale).abs() + abs(e))
                slack[h // p.group] += x * (ds * 1.01 + 2.0 ** -24 * (len(rows[b]) * p.group + 1))
        res.append(total)
        tol.append(slack + 1e-37)
    return res, tol


def weights_case(**kw):
    """A round's end: the accepted rows have been appended; lse as the attention over the places they see gives it."""
    window, sinks = kw.pop("window", 0), kw.pop("sinks", 0)
    path_lens = kw.pop("path_lens")
    base = kw.pop("base")
    p = problem(batch=len(base), lens=[n + m + 1 for n, m in zip(base, path_lens)], live=[kw["R"]] * len(base), extra_places=3, **kw)
    path = torch.full((p.batch, max(1, max(path_lens))), -1, dtype=torch.int32)
    rows = []
    for b, m in enumerate(path_lens):
        path[b, :m] = 1 + torch.randperm(p.R - 1, generator=p.g)[:m].int()
        rows.append([0] + path[b, :m].tolist())
    lse = torch.zeros(p.batch, p.R, p.heads * p.group)
    for b in range(p.batch):
        for i, r in enumerate(rows[b]):
            for h in range(p.heads * p.group):
                lse[b, r, h] = torch.logsumexp(p.K[b][:base[b] + i + 1, h // p.group] @ p.q[b, r, h].double() * p.scale, 0)
    w = torch.rand(p.batch, p.heads, p.max_pages * p.page, generator=p.g)
    return p, path, path_lens, base, rows, lse, w, window, sinks


def check_weights(case, in_place=False):
    p, path, path_lens, base, rows, lse, w, window, sinks = case
    wd = w.to(DEV)
    out = wd if in_place else torch.full_like(wd, -1.0)
    status = i32([5] * p.batch)
    G.cadd_cache_weights(p.q.to(DEV), lse.to(DEV), p.cache(G), i32(base), wd, path=path.to(DEV), path_len=i32(path_lens), scale=p.scale,
                         window=window, n_sinks=sinks, out=out, status=status)
    assert status.tolist() == [0] * p.batch
    want, tol = weights_wanted(p, base, rows, lse, w, window, sinks)
    got = out.cpu().double()
    for b in range(p.batch):
        n = p.lens[b]
        err = (got[b, :, :n] - want[b]).abs()
        assert bool((err <= tol[b]).all()), (b, float((err / tol[b]).max()))
        rest = got[b, :, n:]
        assert torch.equal(rest, w[b, :, n:].double())
    return out


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8])
def test_weights_of_paths(fp4, dim, group):
    check_weights(weights_case(fp4=fp4, dim=dim, group=group, R=20, base=[70, 0, 31, 300], path_lens=[4, 0, 16, 1]))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("base", [0, 1, 30, 31, 32, 33, 63, 64, 127, 128, 129, 500])
def test_weights_at_every_kind_of_length(fp4, base):
    check_weights(weights_case(fp4=fp4, group=4, R=9, base=[base, 3], path_lens=[2, 0], page=8, token_major=True), in_place=True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 2), (64, 1), (100, 129), (4000, 0)])
def test_weights_under_a_window(window, sinks):
    check_weights(weights_case(fp4=True, group=3, R=12, base=[250, 20], path_lens=[6, 11], window=window, sinks=sinks))


def test_many_rows_of_a_prompt_and_rows_without_a_sum():
    p, path, path_lens, base, rows, lse, w, *_ = weights_case(fp4=False, group=4, R=90, base=[40, 0], path_lens=[88, 50])
    lse[0, 0], lse[1, rows[1][3], 2] = -math.inf, math.inf
    check_weights((p, path, path_lens, base, rows, lse, w, 0, 0))
    n_rows = [89, 51]
    rows = [list(range(n)) for n in n_rows]
    lse = torch.randn(lse.shape, generator=p.g) + 12
    out = torch.zeros_like(w, device=DEV)
    G.cadd_cache_weights(p.q.to(DEV), lse.to(DEV), p.cache(G), i32(base), w.to(DEV), n_rows=i32(n_rows), scale=p.scale, out=out)
    want, tol = weights_wanted(p, base, rows, lse, w)
    for b in range(2):
        assert bool(((out[b, :, :p.lens[b]].cpu().double() - want[b]).abs() <= tol[b]).all())


@pytest.mark.parametrize("fp4", [False, True])
def test_rows_without_a_sum_add_nothing_whatever_they_hold(fp4):
    p, path, path_lens, base, rows, lse, w, *_ = weights_case(fp4=fp4, group=2, R=9, base=[70, 200], path_lens=[5, 3])
    for b, r, h, x, e in ((0, 0, 0, math.inf, math.inf), (0, rows[0][2], 3, math.nan, -math.inf), (1, rows[1][3], 1, -math.inf, math.inf)):
        p.q[b, r, h] = x
        lse[b, r, h] = e
    check_weights((p, path, path_lens, base, rows, lse, w, 0, 0))


def test_weights_flag_bad_paths_pages_and_lengths():
    p, path, path_lens, base, rows, lse, w, *_ = weights_case(fp4=False, R=9, base=[70, 20, 33], path_lens=[3, 2, 1])
    path[1, 1] = 9
    table = p.block_table.clone()
    table[0, 1] = -3
    c0 = p.cache(G)
    c = G.KvCache(k=c0.k, v=c0.v, block_table=table.to(DEV), length=c0.length)
    status = i32([0] * 3)
    out = torch.zeros_like(w, device=DEV)
    G.cadd_cache_weights(p.q.to(DEV), lse.to(DEV), c, i32([70, 20, 900]), w.to(DEV), path=path.to(DEV), path_len=i32(path_lens), scale=p.scale,
                         out=out, status=status)
    assert status.tolist() == [G.STATUS_BAD_PAGE, G.STATUS_BAD_PATH, G.STATUS_BAD_LENGTH]
    assert torch.equal(out[0, :, 16:32].cpu(), w[0, :, 16:32])             # places on no page get nothing
    assert torch.equal(out[2, :, :p.lens[2]].cpu(), w[2, :, :p.lens[2]])   # base clamped to the length: no row is in the cache
    rows[1] = rows[1][:2]
    base = [70, 20, 33]
    p.K[1] = p.K[1][:-1]
    want, tol = weights_wanted(p, base, rows, lse, w)
    assert bool(((out[1, :, :22].cpu().double() - want[1]).abs() <= tol[1]).all())


def test_the_same_weights_call_gives_the_same_bits():
    case = weights_case(fp4=True, group=4, R=20, base=[3000, 1700], path_lens=[13, 5], page=64)
    a = check_weights(case).clone()
    assert torch.equal(a, check_weights(case))


# ---- eviction ----

def evict_wanted(p, b, w, budget, sinks, recent):
    """Kept places of every head, by the definition."""
    n = p.lens[b]
    res = []
    for h in range(p.heads):
        if n <= budget:
            res.append(list(range(n)))
            continue
        inner = range(sinks, n - recent)
        key = lambda i: (-(-math.inf if math.isnan(float(w[b, h, i])) else float(w[b, h, i])), i)
        best = sorted(inner, key=key)[:budget - sinks - recent]
        res.append(sorted(list(range(sinks)) + best + list(range(n - recent, n))))
    return res


def check_evict(p, w, budget, sinks, recent, new_page_order=None):
    """Runs an eviction into pages behind the pool's and checks places, weights, rows and what must not change."""
    c0 = p.cache(G)
    per = max(1, (min(budget, max(max(p.lens), 1)) + p.page - 1) // p.page)
    per = max(per, (budget + p.page - 1) // p.page)
    extra = p.batch * per
    grow = lambda t: torch.cat([t, torch.full((extra, *t.shape[1:]), 0 if t.dtype == torch.uint8 else 0.0, dtype=t.dtype, device=DEV)])
    pools = [grow(t) for t in ((c0.k, c0.v, c0.k_scale, c0.v_scale) if p.fp4 else (c0.k, c0.v))]
    before = [t.clone() for t in pools]
    c = G.KvCache(k=pools[0], v=pools[1], k_scale=pools[2] if p.fp4 else None, v_scale=pools[3] if p.fp4 else None,
                  block_table=c0.block_table, length=c0.length)
    table = (p.n_pages + torch.randperm(extra, generator=p.g)).int().reshape(p.batch, per)
    got = G.cadd_cache_evict(c, w.to(DEV), table.to(DEV), budget, n_sinks=sinks, n_recent=recent)
    assert got.status.tolist() == [0] * p.batch
    assert got.new_length.tolist() == [min(n, budget) for n in p.lens]
    after = G.KvCache(k=pools[0], v=pools[1], k_scale=c.k_scale, v_scale=c.v_scale, block_table=table.to(DEV), length=got.new_length)
    k, v = read_all(after, budget)
    for b in range(p.batch):
        for h, places in enumerate(evict_wanted(p, b, w, budget, sinks, recent)):
            m = len(places)
            assert got.kept[b, h].tolist() == places + [-1] * (budget - m), (b, h)
            assert torch.equal(got.weights[b, h, :m].cpu().view(torch.int32), w[b, h, places].view(torch.int32))
            assert torch.equal(k[b, :m, h], p.K[b][places, h]) and torch.equal(v[b, :m, h], p.V[b][places, h])
    for t, old in zip(pools, before):
        assert torch.equal(t[:p.n_pages].view(torch.uint8), old[:p.n_pages].view(torch.uint8))
    return c, table, got


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (40, 4, 8), (64, 0, 0), (64, 30, 34), (128, 5, 0), (300, 2, 3)])
def test_eviction_keeps_the_heaviest(fp4, dim, budget, sinks, recent):
    p = problem(fp4=fp4, dim=dim, batch=4, lens=[70, 0, 131, 64], live=[1] * 4, heads=3)
    w = torch.rand(4, 3, p.max_pages * p.page, generator=p.g)
    check_evict(p, w, budget, sinks, recent)


@pytest.mark.parametrize("kind", ["equal", "few", "zero", "signs", "close", "special"])
@pytest.mark.parametrize("page", [1, 16, 128])
def test_eviction_with_ties_and_odd_weights(kind, page):
    p = problem(batch=2, lens=[2500, 1033], live=[1] * 2, heads=2, page=page, dim=64)
    shape = (2, 2, p.max_pages * p.page)
    w = {"equal": lambda: torch.full(shape, 0.25), "few": lambda: torch.randint(0, 4, shape, generator=p.g).float(),
         "zero": lambda: torch.where(torch.rand(shape, generator=p.g) < 0.9, 0.0, torch.rand(shape, generator=p.g)),
         "signs": lambda: torch.where(torch.rand(shape, generator=p.g) < 0.5, 0.0, -0.0) * torch.randint(0, 2, shape, generator=p.g),
         "close": lambda: 1.0 + torch.randint(0, 300, shape, generator=p.g) * 2.0 ** -23,
         "special": lambda: torch.tensor([math.nan, math.inf, -math.inf, -1.0, 3e38, 1e-45, 0.0])[torch.randint(0, 7, shape, generator=p.g)]}[kind]()
    check_evict(p, w, 700, 3, 40)


def test_a_budget_above_what_the_new_pages_hold_means_what_they_hold():
    p = problem(batch=2, lens=[90, 20], live=[1] * 2, extra_places=0)
    c = p.cache(G)
    new = torch.stack([p.spare[:2], torch.tensor([int(p.spare[2]), int(p.block_table[1, 5])])]).int()
    w = torch.rand(2, 2, p.max_pages * 16, generator=p.g)
    got = G.cadd_cache_evict(c, w.to(DEV), new.to(DEV), 1000, n_sinks=3, n_recent=5)
    assert got.new_length.tolist() == [32, 20] and got.status.tolist() == [0, 0]
    k, v = read_all(at_length(G.KvCache(k=c.k, v=c.v, block_table=new.to(DEV), length=c.length), got.new_length), 32)
    for b in range(2):
        for h, places in enumerate(evict_wanted(p, b, w, 32, 3, 5)):
            assert got.kept[b, h].tolist() == places + [-1] * (1000 - len(places))
            assert torch.equal(k[b, :len(places), h], p.K[b][places, h]) and torch.equal(v[b, :len(places), h], p.V[b][places, h])


@pytest.mark.parametrize("n", [49000, 57000, 140000])
def test_eviction_from_long_caches(n):
    """Lengths on both sides of what a kernel could hold on chip."""
    H, P = 2, 256
    dev = DEV
    g = torch.Generator(device=dev).manual_seed(n)
    pages = (n + P - 1) // P
    budget = n // 5
    extra = (budget + P - 1) // P
    k = torch.randint(0, 255, (pages + extra, H, P, 32), dtype=torch.uint8, device=dev, generator=g)
    ks = torch.randint(0, 127, (pages + extra, H, P, 4), dtype=torch.uint8, device=dev, generator=g)
    w = torch.rand(1, H, pages * P, device=dev, generator=g).mul(1000).round()
    c = G.KvCache(k=k, v=k.clone(), k_scale=ks, v_scale=ks.clone(), block_table=torch.arange(pages, dtype=torch.int32, device=dev)[None], length=i32([n]))
    table = torch.arange(pages, pages + extra, dtype=torch.int32, device=dev)[None]
    got = G.cadd_cache_evict(c, w, table, budget, n_sinks=4, n_recent=100)
    key = w[0, :, :n].clone()
    key[:, :4] = math.inf
    key[:, n - 100:] = math.inf
    want = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :budget].sort(1).values
    assert torch.equal(got.kept[0].long(), want)
    flat = lambda t: t.transpose(0, 1).flatten(1, 2)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        src, dst = flat(t[:pages]), flat(t[pages:])[:, :budget]
        assert torch.equal(dst, torch.stack([src[h, want[h]] for h in range(H)]))


def test_eviction_flags_bad_pages_and_lengths_and_writes_nothing_astray():
    p = problem(batch=3, lens=[100, 100, 100], live=[1] * 3, extra_places=0)
    c0 = p.cache(G)
    table = p.block_table.clone()
    table[1, 3] = p.n_pages + 5
    c = G.KvCache(k=c0.k, v=c0.v, block_table=table.to(DEV), length=i32([100, 100, 4000]))
    before = c.k.clone()
    new = torch.full((3, 2), -1, dtype=torch.int32)
    new[1, 0], new[1, 1], new[2, 0] = int(p.spare[0]), int(p.spare[1]), int(p.spare[2])
    w = torch.rand(3, 2, p.max_pages * 16, generator=p.g)
    got = G.cadd_cache_evict(c, w.to(DEV), new.to(DEV), 20, n_sinks=2, n_recent=3)
    assert got.status.tolist() == [G.STATUS_BAD_PAGE, G.STATUS_BAD_PAGE, G.STATUS_BAD_PAGE | G.STATUS_BAD_LENGTH]
    changed = (c.k.view(torch.int16) != before.view(torch.int16)).flatten(1).any(1).cpu()
    assert set(changed.nonzero().flatten().tolist()) <= set(p.spare.tolist())


def test_eviction_in_place_of_the_length_and_without_optional_outputs():
    p = problem(batch=2, lens=[90, 10], live=[1] * 2, extra_places=0)
    c = p.cache(G)
    new = torch.stack([p.spare[:2], torch.tensor([int(p.spare[2]), int(p.block_table[1, 5])])]).int()     # a page behind request 1's length
    w = torch.rand(2, 2, p.max_pages * 16, generator=p.g)
    out = G.Evicted(new_length=c.length, kept=torch.zeros(2, 2, 30, dtype=torch.int32, device=DEV))
    G.cadd_cache_evict(c, w.to(DEV), new.to(DEV), 30, out=out)
    assert c.length.tolist() == [30, 10]
    for b in range(2):
        for h, places in enumerate(evict_wanted(p, b, w, 30, 0, 0)):
            assert out.kept[b, h].tolist() == places + [-1] * (30 - len(places))


# ---- rounds ----

@pytest.mark.parametrize("fp4", [False, True])
def test_rounds_of_building_attending_verifying_committing_and_evicting(fp4):
    """The framework's own trees: built from draft logits, attended over the cache, verified, the accepted path committed and
    weighed, the cache cut to its budget: three rounds, each checked against the 64-bit forms on what the round before left."""
    g = torch.Generator().manual_seed(5)
    B, L, K, B_max, V, H, GR, D, P, budget = 3, 5, 4, 24, 400, 2, 4, 128, 16, 60
    R, HQ, per = B_max + 1, H * GR, 8
    shape = (B * per * 4, H, P)
    if fp4:
        pools = [torch.zeros(*shape, n, dtype=torch.uint8, device=DEV) for n in (D // 2, D // 2, D // 16, D // 16)]
    else:
        pools = [torch.zeros(*shape, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    make = lambda table, length: G.KvCache(k=pools[0], v=pools[1], k_scale=pools[2] if fp4 else None, v_scale=pools[3] if fp4 else None,
                                           block_table=table, length=length)
    tables = [torch.arange(i * B * per, (i + 1) * B * per, dtype=torch.int32, device=DEV).reshape(B, per) for i in range(4)]
    prompt = torch.randn(2, B, 70, H, D, generator=g).bfloat16()
    cache = make(tables[0], i32([0] * B))
    G.cadd_cache_append(cache, prompt[0].to(DEV), prompt[1].to(DEV), n_rows=i32([70, 12, 41]), new_length=cache.length)
    keys = [stored(prompt[0, b, :n], fp4) for b, n in enumerate((70, 12, 41))]          # per request [places, heads, dim], head by head after eviction
    vals = [stored(prompt[1, b, :n], fp4) for b, n in enumerate((70, 12, 41))]
    weights = torch.zeros(B, H, per * P, device=DEV)
    mine = [torch.zeros(H, n, dtype=torch.float64) for n in (70, 12, 41)]
    for step in range(3):
        logits = torch.randn(B, L, V, generator=g) * 2
        logits[:, :, step] += 6
        tree = G.cadd_build_tree(logits.to(DEV), K, B_max, R, cost_coef=torch.tensor([[1.0, 2.0, 0.01, 0.0005]] * B, dtype=torch.float64))
        q, k, v = (torch.randn(B, R, n, D, generator=g).bfloat16() for n in (HQ, H, H))
        att = G.cadd_tree_attention(q.to(DEV), k.to(DEV), v.to(DEV), cache, mask_bits=tree.mask_bits, n_nodes=tree.n_nodes, depth=tree.depth)
        y = torch.randn(B, R, V, generator=g)
        y[:, :, step] += 9                                                           # the target agrees with the boosted token
        verdict = G.cadd_verify_tree(y.to(DEV), L, tree.n_nodes, tree.token_ids, tree.parent_idx)
        base = cache.length.clone()
        G.cadd_cache_append(cache, k.to(DEV), v.to(DEV), path=verdict.accepted_nodes, path_len=verdict.accepted_len, new_length=cache.length)
        G.cadd_cache_weights(q.to(DEV), att.lse, cache, base, weights, path=verdict.accepted_nodes, path_len=verdict.accepted_len)
        accepted = verdict.accepted_len.tolist()
        assert max(accepted) >= 1
        p = Problem(batch=B, heads=H, group=GR, dim=D, page=P, fp4=False, lens=[x.shape[0] for x in keys], R=R,
                    live=[int(n) + 1 for n in tree.n_nodes], causal=False)
        p.q, p.k, p.v, p.K, p.V, p.depth = q, k, v, keys, vals, tree.depth.cpu()
        bits = tree.mask_bits.cpu().long()
        p.mask = ((bits[..., None] >> torch.arange(32)) & 1).bool().flatten(2)[:, :, :R]
        from cache_util import check_attention
        check_attention(p, att)
        rows = [[0] + verdict.accepted_nodes[b, :accepted[b]].tolist() for b in range(B)]
        keys = [torch.cat([keys[b], stored(k[b, rows[b]], fp4)]) for b in range(B)]
        vals = [torch.cat([vals[b], stored(v[b, rows[b]], fp4)]) for b in range(B)]
        p.K = keys
        w_in = torch.zeros(B, H, per * P, dtype=torch.float64)
        for b in range(B):
            w_in[b, :, :mine[b].shape[1]] = mine[b]
        want, tol = weights_wanted(p, [x.shape[1] for x in mine], rows, att.lse.cpu(), w_in)
        for b in range(B):
            n = keys[b].shape[0]
            assert int(cache.length[b]) == n
            assert bool(((weights[b, :, :n].cpu().double() - want[b]).abs() <= tol[b] + 2.0 ** -20 * want[b]).all())
        # eviction goes by the library's own running totals, which the check above has bounded
        w_now = weights.cpu()
        ev = G.cadd_cache_evict(cache, weights, tables[step + 1], budget, n_sinks=2, n_recent=8)
        p.lens = [x.shape[0] for x in keys]
        kept = [evict_wanted(p, b, w_now, budget, 2, 8) for b in range(B)]
        for b in range(B):
            for h in range(H):
                assert ev.kept[b, h, :len(kept[b][h])].tolist() == kept[b][h]
        keys = [torch.stack([keys[b][kept[b][h], h] for h in range(H)], 1) for b in range(B)]
        vals = [torch.stack([vals[b][kept[b][h], h] for h in range(H)], 1) for b in range(B)]
        mine = [torch.stack([w_now[b, h, kept[b][h]].double() for h in range(H)]) for b in range(B)]
        cache, weights = make(tables[step + 1], ev.new_length), ev.weights
        got_k, _ = read_all(cache, budget)
        for b in range(B):
            assert torch.equal(got_k[b, :keys[b].shape[0]], keys[b])


@pytest.mark.parametrize("fp4", [False, True])
def test_a_captured_round_follows_its_inputs(fp4):
    """Attention, commit in place, weights and eviction captured into one graph: replayed with other lengths, paths and rows it gives
    what the calls give one by one, bit for bit."""
    B, H, GR, D, P, R, L, budget = 3, 2, 4, 64, 16, 12, 4, 48
    g = torch.Generator().manual_seed(11)
    per, new_per = 8, 3
    n_pages = B * (per + new_per)
    table = torch.arange(B * per, dtype=torch.int32, device=DEV).reshape(B, per)
    new_table = torch.arange(B * per, n_pages, dtype=torch.int32, device=DEV).reshape(B, new_per)

    def buffers():
        if fp4:
            pools = [torch.zeros(n_pages, H, P, n, dtype=torch.uint8, device=DEV) for n in (D // 2, D // 2, D // 16, D // 16)]
        else:
            pools = [torch.zeros(n_pages, H, P, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [None, None]
        d = dict(pools=pools, length=i32([0] * B), base=i32([0] * B), path=torch.zeros(B, L, dtype=torch.int32, device=DEV), path_len=i32([0] * B),
                 q=torch.zeros(B, R, H * GR, D, dtype=torch.bfloat16, device=DEV), k=torch.zeros(B, R, H, D, dtype=torch.bfloat16, device=DEV),
                 v=torch.zeros(B, R, H, D, dtype=torch.bfloat16, device=DEV), w=torch.zeros(B, H, per * P, device=DEV),
                 att=G.Attention(out=torch.zeros(B, R, H * GR, D, dtype=torch.bfloat16, device=DEV), lse=torch.zeros(B, R, H * GR, device=DEV), status=i32([0] * B)),
                 ev=G.Evicted(new_length=i32([0] * B), kept=torch.zeros(B, H, budget, dtype=torch.int32, device=DEV),
                              weights=torch.zeros(B, H, new_per * P, device=DEV), status=i32([0] * B)))
        d["cache"] = G.KvCache(k=pools[0], v=pools[1], k_scale=pools[2], v_scale=pools[3], block_table=table, length=d["length"])
        d["ws"] = torch.zeros(G.cadd_tree_attention_workspace_bytes(B, R, H * GR, d["cache"]), dtype=torch.uint8, device=DEV)
        return d

    def step(d):
        G.cadd_tree_attention(d["q"], d["k"], d["v"], d["cache"], out=d["att"], workspace=d["ws"])
        d["base"].copy_(d["length"])
        G.cadd_cache_append(d["cache"], d["k"], d["v"], path=d["path"], path_len=d["path_len"], new_length=d["length"])
        G.cadd_cache_weights(d["q"], d["att"].lse, d["cache"], d["base"], d["w"], path=d["path"], path_len=d["path_len"])
        G.cadd_cache_evict(d["cache"], d["w"], new_table, budget, n_sinks=2, n_recent=5, out=d["ev"])

    def put(d, x):
        for name in ("length", "path", "path_len", "q", "k", "v", "w"):
            d[name].copy_(x[name])
        G.cadd_cache_append(d["cache"], x["prompt"][0], x["prompt"][1], n_rows=x["n"], new_length=d["length"])

    a, b = buffers(), buffers()
    step(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for lens, path_lens in (([100, 1, 47], [4, 0, 2]), ([0, 60, 124], [1, 3, 3]), ([33, 32, 31], [0, 4, 1])):
        x = dict(length=i32([0] * B), path=torch.randint(1, R, (B, L), generator=g).int().to(DEV), path_len=i32(path_lens), n=i32(lens),
                 q=torch.randn(B, R, H * GR, D, generator=g).bfloat16().to(DEV), k=torch.randn(B, R, H, D, generator=g).bfloat16().to(DEV),
                 v=torch.randn(B, R, H, D, generator=g).bfloat16().to(DEV), w=torch.rand(B, H, per * P, generator=g).to(DEV),
                 prompt=torch.randn(2, B, max(lens), H, D, generator=g).bfloat16().to(DEV))
        put(a, x)
        put(b, x)
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        assert a["length"].tolist() == [n + m + 1 for n, m in zip(lens, path_lens)]
        for i in range(4 if fp4 else 2):
            assert torch.equal(a["pools"][i], b["pools"][i])
        for t, u in ((a["att"].out, b["att"].out), (a["att"].lse, b["att"].lse), (a["w"], b["w"]), (a["length"], b["length"]), (a["base"], b["base"]),
                     (a["ev"].new_length, b["ev"].new_length), (a["ev"].kept, b["ev"].kept), (a["ev"].weights, b["ev"].weights), (a["ev"].status, b["ev"].status)):
            assert torch.equal(t, u)


def test_rows_of_a_pool_of_more_than_four_gigabytes():
    """Four-bit pools whose last pages are used: every call's row offsets need 64 bits.  Small pools with the same contents say what is right."""
    H, P, D, B, R = 8, 64, 128, 2, 3
    n_pages = (1 << 32) // (H * P * D // 2) + 40
    sizes = (D // 2, D // 2, D // 16, D // 16)
    prompt = torch.randn(2, B, 150, H, D, generator=torch.Generator().manual_seed(3)).bfloat16().to(DEV)
    q = torch.randn(B, R, 2 * H, D, device=DEV).bfloat16()
    got = []
    for pages in (12, n_pages):
        pools = [torch.empty(pages, H, P, n, dtype=torch.uint8, device=DEV) for n in sizes]
        table = torch.arange(pages - 6, pages, dtype=torch.int32, device=DEV).reshape(B, 3)
        new = torch.arange(pages - 10, pages - 6, dtype=torch.int32, device=DEV).reshape(B, 2)
        c = G.KvCache(k=pools[0], v=pools[1], k_scale=pools[2], v_scale=pools[3], block_table=table, length=i32([0, 0]))
        G.cadd_cache_append(c, prompt[0], prompt[1], n_rows=i32([150, 97]), new_length=c.length)
        own = prompt[:, :, :R].contiguous()
        outs = [G.cadd_tree_attention(q, own[0], own[1], c, flags=f) for f in (0, G.ATTENTION_TILED_PATH)]
        w = torch.zeros(B, H, 3 * P, device=DEV)
        G.cadd_cache_weights(q, outs[0].lse, c, i32([147, 94]), w, n_rows=i32([3, 3]))
        ev = G.cadd_cache_evict(c, w, new, 100, n_sinks=1)
        after = G.KvCache(k=pools[0], v=pools[1], k_scale=pools[2], v_scale=pools[3], block_table=new, length=ev.new_length)
        got.append([*G.cadd_cache_read(c, 160), *G.cadd_cache_read(after, 100), outs[0].out, outs[0].lse, outs[1].out, outs[1].lse, w, ev.kept])
        assert ev.status.tolist() == [0, 0]
    for t, u in zip(*got):
        assert torch.equal(t, u)
    assert torch.equal(got[1][0][0, :150].cpu(), stored(prompt[0, 0].cpu(), True).bfloat16())


# ---- what is stored, byte by byte; queries and shapes out of the ordinary ----

@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("exps", [(0, 0), (4, -3), (-16, 16)])
def test_append_stores_the_bytes_of_the_definition(dim, exps):
    """Zero has one code, 0, under a zero scale and under any other."""
    p = problem(fp4=True, dim=dim, lens=[0, 0], R=48, live=[48, 48], k_exp=exps[0], v_exp=exps[1], page=8)
    for b in range(2):
        for x in (p.k, p.v):
            x[b, :10] = awkward_rows(10, 2, dim, p.g)
            x[b, 10] = -x[b, 10].abs() * 2.0 ** -40                        # blocks of tiny negative numbers
            x[b, 11] = -0.0
            x[b, 12] = torch.where(torch.arange(dim) % 16 == 3, 1.0, -2.0 ** -9).bfloat16()
            x[b, 13] = -x[b, 13].abs()
    c = p.cache(G)
    G.cadd_cache_append(c, p.k.to(DEV), p.v.to(DEV))
    for src, pool, scale, exp in ((p.k, c.k, c.k_scale, exps[0]), (p.v, c.v, c.v_scale, exps[1])):
        codes, scales = encode(src.double(), exp)
        for b in range(2):
            for i in range(48):
                page, slot = int(p.block_table[b, i // 8]), i % 8
                assert torch.equal(scale[page, :, slot].cpu(), scales[b, i]), (b, i)
                assert torch.equal(pool[page, :, slot].cpu(), codes[b, i]), (b, i)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("power", [12, 20, 30, 33, 60, 100, -100])
@pytest.mark.parametrize("path_lens", [[4, 0], [60, 3]])
def test_weights_of_queries_with_an_element_far_above_the_others(dim, power, path_lens):
    """Keys are zero at that element: the scores are the other elements', which have to keep their bits."""
    base = [300, 70]
    p, path, path_lens, base, rows, lse, w, *_ = weights_case(fp4=True, dim=dim, group=4, R=70, base=base, path_lens=path_lens)
    for b in range(2):
        k = p.K[b].clone()
        k[:, :, 5] = 0.0
        codes, scales = encode(k)
        p.put(0, b, 0, codes)
        p.put(2, b, 0, scales)
        p.K[b] = decode(codes, scales)
        p.q[b, rows[b][::2], :, 5] = 1.5 * 2.0 ** power
        for i, r in enumerate(rows[b]):
            for h in range(p.heads * p.group):
                lse[b, r, h] = torch.logsumexp(p.K[b][:base[b] + i + 1, h // p.group] @ p.q[b, r, h].double() * p.scale, 0)
    check_weights((p, path, path_lens, base, rows, lse, w, 0, 0))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("page,window", [(16, 0), (64, 0), (64, 5000)])
def test_weights_of_warps_that_go_through_many_steps(fp4, page, window):
    """32 heads' caches of up to 16000 places: a CTA has 512 keys and more, a warp four steps and more, totals and pages fetched ahead."""
    case = weights_case(fp4=fp4, heads=8, group=2, page=page, R=9, base=[16000, 9000, 12345, 100], path_lens=[3, 8, 0, 5], window=window, sinks=40 if window else 0)
    check_weights(case)
    check_weights(case, in_place=True)
