"""Plain 64-bit forms of the cache and tree-attention operators, and small random problems for them.

Everything here works on CPU tensors in float64, place by place from the definitions; nothing of the library is used."""
import math
from dataclasses import dataclass, field

import torch

E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def e4m3_table():
    """All non-negative e4m3 numbers, indexed by their byte (0x7f is NaN)."""
    v = [(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)]
    v[127] = math.nan
    return torch.tensor(v, dtype=torch.float64)


E4M3 = e4m3_table()


def nearest_even(x, grid):
    """Index of the entry of an ascending grid nearest to each x (>= 0); half way goes to the even index."""
    hi = torch.searchsorted(grid, x).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = (grid[hi] - x).abs(), (x - grid[lo]).abs()
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def encode(x, exp=0):
    """float64 [..., D] -> codes uint8 [..., D/2], scales uint8 [..., D/16]."""
    b = (torch.nan_to_num(x, nan=0.0, posinf=1e30, neginf=-1e30) * 2.0 ** exp).unflatten(-1, (-1, 16))
    s = nearest_even((b.abs().amax(-1) / 6).clamp(max=448.0), E4M3[:127])
    sv = E4M3[s].unsqueeze(-1)
    y = torch.where(sv > 0, b / torch.where(sv > 0, sv, torch.ones_like(sv)), torch.zeros_like(b))
    code = nearest_even(y.abs().clamp(max=6.0), E2M1[:8])
    code = (code + 8 * ((y < 0) & (code > 0))).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), s.to(torch.uint8)


def decode(codes, scales, exp=0):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    return E2M1[c] * (E4M3[scales.long()] * 2.0 ** -exp).repeat_interleave(16, -1)


@dataclass
class Problem:
    """A cache with its contents (float64, as the cache stands for them) and a batch of rows on top."""
    batch: int
    heads: int
    group: int
    dim: int
    page: int
    fp4: bool
    lens: list
    R: int
    live: list
    causal: bool
    window: int = 0
    sinks: int = 0
    k_exp: int = 0
    v_exp: int = 0
    token_major: bool = False           # pools laid out [n_pages, page, heads, ...] instead of [n_pages, heads, page, ...]
    extra_places: int = 0               # room in the tables behind the longest length
    scale: float = None
    seed: int = 0
    K: list = field(default_factory=list)
    V: list = field(default_factory=list)

    def __post_init__(self):
        g = self.g = torch.Generator().manual_seed(self.seed)
        self.scale = self.dim ** -0.5 if self.scale is None else self.scale
        P, H, D = self.page, self.heads, self.dim
        self.max_pages = max(1, (max(self.lens) + self.extra_places + P - 1) // P)
        n_pages = self.batch * self.max_pages + 3
        order = torch.randperm(n_pages, generator=g)
        self.block_table = order[:self.batch * self.max_pages].reshape(self.batch, self.max_pages).int().contiguous()
        self.spare = order[self.batch * self.max_pages:]
        self.n_pages = n_pages
        # unused slots hold NaN (bf16) or bytes that are no scale the library writes
        if self.fp4:
            self.pools = [torch.full((n_pages, H, P, D // 2), 0xff, dtype=torch.uint8), torch.full((n_pages, H, P, D // 2), 0xff, dtype=torch.uint8),
                          torch.full((n_pages, H, P, D // 16), 0xff, dtype=torch.uint8), torch.full((n_pages, H, P, D // 16), 0xff, dtype=torch.uint8)]
        else:
            self.pools = [torch.full((n_pages, H, P, D), math.nan, dtype=torch.bfloat16) for _ in range(2)]
        for b, n in enumerate(self.lens):
            for which, store in ((0, self.K), (1, self.V)):
                x = torch.randn(n, H, D, generator=g, dtype=torch.float64) * (1 + which)
                if self.fp4:
                    exp = (self.k_exp, self.v_exp)[which]
                    codes, scales = encode(x * 2.0 ** -exp, exp)
                    self.put(which, b, 0, codes)
                    self.put(which + 2, b, 0, scales)
                    x = decode(codes, scales, exp)
                else:
                    self.put(which, b, 0, x.bfloat16())
                    x = x.bfloat16().double()
                store.append(x)
        B, R, HQ = self.batch, self.R, self.heads * self.group
        self.q = (2 * torch.randn(B, R, HQ, D, generator=g)).bfloat16()
        self.k = torch.randn(B, R, H, D, generator=g).bfloat16()
        self.v = torch.randn(B, R, H, D, generator=g).bfloat16()
        self.depth = torch.zeros(B, R, dtype=torch.int32)
        self.mask = torch.zeros(B, R, R, dtype=torch.bool)
        for b in range(B):
            for j in range(self.live[b]):
                if self.causal:
                    self.mask[b, j, :j + 1] = True
                    self.depth[b, j] = j
                elif j:
                    p = int(torch.randint(max(0, j - 6), j, (1,), generator=g))
                    self.mask[b, j] = self.mask[b, p]
                    self.depth[b, j] = self.depth[b, p] + 1
                self.mask[b, j, j] = True

    def put(self, which, b, start, rows):
        """rows [n, heads, ...] into pool `which` at places start.. of request b."""
        for i in range(rows.shape[0]):
            pos = start + i
            self.pools[which][int(self.block_table[b, pos // self.page]), :, pos % self.page] = rows[i]

    def get(self, which, b, pos, table=None):
        table = self.block_table if table is None else table
        return self.pools[which][int(table[b, pos // self.page]), :, pos % self.page]

    def mask_bits(self):
        W = (self.R + 31) // 32
        m = torch.zeros(self.batch, self.R, W * 32, dtype=torch.int64)
        m[:, :, :self.R] = self.mask
        bits = (m.view(self.batch, self.R, W, 32) << torch.arange(32)).sum(-1)
        return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()

    # ---- on the device ----
    def cache(self, G, dev="cuda"):
        pools = [p.transpose(1, 2).contiguous().transpose(1, 2) if self.token_major else p for p in self.pools]
        pools = [p.transpose(1, 2).to(dev).transpose(1, 2) if self.token_major else p.to(dev) for p in pools]
        return G.KvCache(k=pools[0], v=pools[1], block_table=self.block_table.to(dev), length=torch.tensor(self.lens, dtype=torch.int32, device=dev),
                         k_scale=pools[2] if self.fp4 else None, v_scale=pools[3] if self.fp4 else None, k_exp=self.k_exp, v_exp=self.v_exp)

    def run(self, G, cache=None, dev="cuda", **kw):
        cache = self.cache(G, dev) if cache is None else cache
        n_nodes = torch.tensor([n - 1 for n in self.live], dtype=torch.int32, device=dev)
        if not self.causal:
            kw.setdefault("mask_bits", self.mask_bits().to(dev))
            kw.setdefault("depth", self.depth.to(dev))
        return G.cadd_tree_attention(self.q.to(dev), self.k.to(dev), self.v.to(dev), cache, n_nodes=n_nodes, scale=self.scale,
                                     window=self.window, n_sinks=self.sinks, **kw)

    # ---- in 64 bits ----
    def keys(self, b):
        n = self.live[b]
        return torch.cat([self.K[b], self.k[b, :n].double()]), torch.cat([self.V[b], self.v[b, :n].double()])

    def sees(self, b):
        """[live, len + live]"""
        n, r = self.lens[b], self.live[b]
        place = torch.cat([torch.arange(n), n + self.depth[b, :r]])
        mine = n + self.depth[b, :r]
        see = torch.ones(r, n + r, dtype=torch.bool)
        see[:, n:] = self.mask[b, :r, :r]
        if self.window:
            see &= (mine[:, None] - place[None] < self.window) | (place[None] < self.sinks)
        return see

    def attention(self, b):
        """out [live, heads_q, D], lse [live, heads_q] and, for the tolerances, sum_p w_p |v_p| and the largest sum_d |q_d k_d|."""
        k, v = self.keys(b)
        see = self.sees(b)
        r, HQ, D = self.live[b], self.heads * self.group, self.dim
        out, amass = torch.zeros(r, HQ, D, dtype=torch.float64), torch.zeros(r, HQ, D, dtype=torch.float64)
        lse, size = torch.full((r, HQ), -math.inf, dtype=torch.float64), torch.zeros(r, HQ, dtype=torch.float64)
        for h in range(HQ):
            q = self.q[b, :r, h].double()
            kh, vh = k[:, h // self.group], v[:, h // self.group]
            for i in range(r):
                at = see[i].nonzero().flatten()
                if len(at) == 0:
                    continue
                s = kh[at] @ q[i] * self.scale
                lse[i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[i, h])
                out[i, h] = w @ vh[at]
                amass[i, h] = w @ vh[at].abs()
                size[i, h] = (kh[at].abs() @ q[i].abs()).max()
        return out, lse, amass, size


def attention_tolerance(p, out, lse, amass, size, n_keys):
    """Largest admissible errors of out and lse.

    A score is a sum of dim products of bf16 numbers, exact each, added in fp32: off by at most dim 2^-24 sum|q k| scale, plus
    roundings of the scaled score, of its difference to the running maximum and inside exp2 (2^-22 relative each at |s - m| of
    order one, 2^-24 |s| each): ds = scale size (dim + 4) 2^-24 + 2^-20.  Weights are off by ds relative and rounded to bf16, 2^-8;
    sums of n keys in fp32 by n 2^-24 at most; numerator and denominator both carry the fp32 part (2 x).  The result is
    rounded to bf16, 2^-8 of itself."""
    ds = p.scale * size * (p.dim + 4) * 2.0 ** -24 + 2.0 ** -20 + n_keys * 2.0 ** -24
    rel = (2.0 ** -8 + 2 * ds).unsqueeze(-1)
    tol_out = rel * (1 + 2.0 ** -7) * amass + 2.0 ** -8 * out.abs()
    return tol_out + 1e-30, ds + lse.abs().nan_to_num(posinf=0.0) * 2.0 ** -23 + 1e-7


def check_attention(p, got, before_out=None, before_lse=None):
    out, lse = got.out.cpu().double(), got.lse.cpu().double()
    for b in range(p.batch):
        r = p.live[b]
        want, wlse, amass, size = p.attention(b)
        tol, tol_lse = attention_tolerance(p, want, wlse, amass, size, p.lens[b] + r)
        err = (out[b, :r] - want).abs()
        assert bool((err <= tol).all()), (b, float((err / tol).max()))
        none = wlse == -math.inf
        assert torch.equal(lse[b, :r] == -math.inf, none)
        err = (lse[b, :r] - wlse)[~none].abs()
        assert bool((err <= tol_lse[~none]).all()), (b, float(err.max()))
        rest = out[b, r:]
        assert torch.equal(rest, before_out[b, r:].double() if before_out is not None else torch.zeros_like(rest))
