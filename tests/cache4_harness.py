"""Caches held in 4 bits for the tests: the packing's definition in 64 bits, and paged pools
whose stale slots stand for NaN."""

from __future__ import annotations

import math

import torch

from paper_2608_02134_gb300 import gmc
from tests.cache_harness import Case

F64 = torch.float64
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
# every scale byte's value, in order; NaN from 0xf9 on
SCALES = [(b & 7) * 2.0 ** -17 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 15)
          for b in range(0xe1)]


def nearest(x, table):
    """The place of the nearest value of an ascending table, ties to the even place."""
    t = torch.tensor(table, dtype=F64)
    hi = torch.searchsorted(t, x.contiguous()).clamp(1, len(table) - 1)
    lo = hi - 1
    a, b = x - t[lo], t[hi] - x  # exact: few bits each
    return torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def pack(x):
    """Codes [..., d / 2] and scales [..., d / 16] (uint8) of rows [..., d] of bf16 values."""
    x = x.to(F64).unflatten(-1, (-1, 16))
    top = x.abs().amax(-1)  # NaN where any is
    fine = torch.isfinite(top)
    s = nearest(torch.where(fine, top, torch.zeros_like(top)).clamp(max=6 * 8192.0) / 6, SCALES)
    s = torch.where((top > 0) & (s == 0), 1, s)
    value = torch.tensor(SCALES, dtype=F64)[s]
    y = x.abs() / torch.where(value > 0, value, torch.ones_like(value))[..., None]
    code = nearest(torch.where(fine[..., None], y, torch.zeros_like(y)).clamp(max=6.0), LEVELS)
    code = torch.where((x < 0) & fine[..., None], code + 8, code).flatten(-2)
    s = torch.where(fine, s, 0xf9)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), s.to(torch.uint8)


def unpack(codes, scales):
    """The values, fp64 [..., d]."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=F64)[code].unflatten(-1, (-1, 16))
    table = torch.tensor(SCALES + [math.nan] * (256 - len(SCALES)), dtype=F64)
    return (v * table[scales.long()][..., None]).flatten(-2)


class Case4(Case):
    """A Case whose pools hold 4 bits; K and V are the values that they stand for."""

    def __init__(self, lens, H, Hkv, d, page=16, news=None, seed=0, extra_pages=2, width=None,
                 spread=1.0, pad=0):
        self.pad = pad
        super().__init__(lens, H, Hkv, d, "bf16", page, news, seed, extra_pages, "heads", width,
                         spread)
        n = self.table.numel() + extra_pages
        part = gmc.cache4_part_size(page, d)
        self.pool_k = torch.full((n, Hkv, part + pad), 0xf9, dtype=torch.uint8)
        self.pool_v = torch.full((n, Hkv, part + pad), 0xf9, dtype=torch.uint8)
        self.raw_K, self.raw_V = self.K, self.V
        self.K = [unpack(*pack(x)).to(torch.bfloat16) for x in self.K]
        self.V = [unpack(*pack(x)).to(torch.bfloat16) for x in self.V]
        for b in range(self.B):
            self.fill(b, range(self.lens[b]))

    def put(self, b, places):  # of bf16 pools: not these
        pass

    def halves(self, pool):
        """Views of codes [page, Hkv, slot, d / 2] and scales [page, Hkv, slot, d / 16]."""
        n = self.page * self.d // 2
        return (pool[..., :n].unflatten(-1, (self.page, self.d // 2)),
                pool[..., n:n + n // 8].unflatten(-1, (self.page, self.d // 16)))

    def fill(self, b, places):
        for raw, pool in ((self.raw_K[b], self.pool_k), (self.raw_V[b], self.pool_v)):
            codes, scales = self.halves(pool)
            c, s = pack(raw)
            for j in places:
                p = int(self.table[b, j // self.page])
                codes[p, :, j % self.page], scales[p, :, j % self.page] = c[j], s[j]

    def blank(self, b, j):
        for pool in (self.pool_k, self.pool_v):
            for x in self.halves(pool):
                x[int(self.table[b, j // self.page]), :, j % self.page] = 0xf9

    def cache(self, max_len=None, **kw):
        self.dk, self.dv = self.pool_k.cuda(), self.pool_v.cuda()
        self.dlens = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        return gmc.KVCache4(self.dk, self.dv, self.table.cuda(), self.dlens, page_size=self.page,
                            d=self.d, max_len=max(self.lens) if max_len is None else max_len,
                            status=self.status, **kw)

    def rows(self, pool, b, places):
        """(codes, scales) of the places of a sequence in a pool (on the host)."""
        codes, scales = self.halves(pool)
        p = self.table[b].long()
        j = torch.tensor(list(places))
        return codes[p[j // self.page], :, j % self.page], scales[p[j // self.page], :, j % self.page]


def same_rows(got, want, what):
    """Codes and scales alike; the two zeros are one."""
    zero = lambda c: torch.where(torch.stack([c & 15, c >> 4], -1) == 8, 0,  # noqa: E731
                                 torch.stack([c & 15, c >> 4], -1))
    assert torch.equal(got[1], want[1]), what + ": scales"
    assert torch.equal(zero(got[0]), zero(want[0])), what + ": codes"


def tolerance(c, size):
    """Relative to sum p |v|: logits' sums, a weight rounded to half (2^-11), the output (2^-8)."""
    return 2.0 ** -24 * (8.0 * math.sqrt(c.d) * size + 64.0) + 2.0 ** -8 + 2.0 ** -11
