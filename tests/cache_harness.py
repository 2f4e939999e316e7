"""Paged caches for the tests: built from plain rows, with the operators' definitions in 64 bits.

Stale slots, the pages of nobody and the rows past a sequence's end hold NaN, so that
anything read from them shows.
"""

from __future__ import annotations

import math

import torch

from paper_2608_02134_gb300 import gmc

F64 = torch.float64


class Case:
    """B sequences of `lens` tokens of which `news` are new (default: one each)."""

    def __init__(self, lens, H, Hkv, d, dtype="bf16", page=16, news=None, seed=0, extra_pages=2,
                 layout="heads", width=None, spread=1.0):
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.lens, self.news = list(lens), list(news if news is not None else [1] * len(lens))
        self.B, self.H, self.Hkv, self.d, self.page = len(lens), H, Hkv, d, page
        g = self.gen = torch.Generator().manual_seed(1234 + seed)
        per = max(1, -(-max(self.lens) // page)) if width is None else width
        n = self.B * per + extra_pages
        self.table = torch.randperm(n, generator=g)[:self.B * per].reshape(self.B, per).int()
        rnd = lambda *s: torch.randn(*s, generator=g).to(self.dt)  # noqa: E731
        self.K = [rnd(m, Hkv, d) for m in self.lens]
        self.V = [rnd(m, Hkv, d) for m in self.lens]
        self.q = (spread * torch.randn(sum(self.news), H, d, generator=g)).to(self.dt)
        shape = (n, Hkv, page, d) if layout == "heads" else (n, page, Hkv, d)
        self.pool_k = torch.full(shape, math.nan, dtype=self.dt)
        self.pool_v = torch.full(shape, math.nan, dtype=self.dt)
        self.layout = layout
        for b in range(self.B):
            self.put(b, range(self.lens[b]))

    def views(self):
        """[page, Hkv, slot, d] views of the pools."""
        if self.layout == "heads":
            return self.pool_k, self.pool_v
        return self.pool_k.permute(0, 2, 1, 3), self.pool_v.permute(0, 2, 1, 3)

    def put(self, b, places):
        k, v = self.views()
        for j in places:
            p = int(self.table[b, j // self.page])
            k[p, :, j % self.page] = self.K[b][j]
            v[p, :, j % self.page] = self.V[b][j]

    def blank(self, b, j):
        """The slot of one token back to NaN (a token that the call itself appends)."""
        k, v = self.views()
        p = int(self.table[b, j // self.page])
        k[p, :, j % self.page] = math.nan
        v[p, :, j % self.page] = math.nan

    def cache(self, max_len=None, **kw):
        self.dk, self.dv = self.pool_k.cuda(), self.pool_v.cuda()
        k, v = (self.dk, self.dv) if self.layout == "heads" else \
            (self.dk.permute(0, 2, 1, 3), self.dv.permute(0, 2, 1, 3))
        self.dlens = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        return gmc.KVCache(k, v, self.table.cuda(), self.dlens,
                           max_len=max(self.lens) if max_len is None else max_len,
                           status=self.status, **kw)

    def offsets(self):
        at = [0]
        for t in self.news:
            at.append(at[-1] + t)
        return torch.tensor(at, dtype=torch.int32).cuda()


def seen(n, i, window, sinks):
    j = torch.arange(n)
    ok = j <= i
    if window:
        ok &= (i - j < window) | (j < sinks)
    return ok


def attention(K, V, q, i, window=0, sinks=0, scale=None):
    """One query row [H, d] at place i: (out [H, d], lse [H], weights [H, n], bound [H, d]),
    bound the sum of p |v| that rounding errors are measured against, and the largest
    sum of |q k| scale of the row."""
    n, Hkv, d = K.shape
    H = q.shape[0]
    G = H // Hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse = torch.zeros(H, d, dtype=F64), torch.full((H,), -math.inf, dtype=F64)
    w, bound = torch.zeros(H, n, dtype=F64), torch.zeros(H, d, dtype=F64)
    size = 0.0
    at = torch.nonzero(seen(n, i, window, sinks)).flatten()
    if at.numel():
        for h in range(H):
            k, v = K[at, h // G].to(F64), V[at, h // G].to(F64)
            x = k @ q[h].to(F64) * scale
            size = max(size, float((k.abs() @ q[h].to(F64).abs()).max()) * scale)
            lse[h] = torch.logsumexp(x, 0)
            p = (x - lse[h]).exp()
            w[h, at] = p
            out[h], bound[h] = p @ v, p @ v.abs()
    return out, lse, w, bound, size


def tolerance(dtype, d, size, roundings=1):
    """Relative to sum p |v|.  bf16: 2^-8 for each rounding (the output's; with two, the
    weights' as well).  fp32: a logit of `size` = sum |q k| scale is off by some sqrt(d)
    roundings of it, and so is every weight."""
    f32 = 2.0 ** -24 * (8.0 * math.sqrt(d) * size + 64.0)
    return f32 + (roundings * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)


def lse_tolerance(d, size):
    return 2.0 ** -24 * (8.0 * math.sqrt(d) * size + 64.0)
