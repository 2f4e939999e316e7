"""fp32 attention on floats whose three bf16 parts leave out the most: the bound of what is
left out."""

import math

import numpy as np
import pytest
import torch


def _parts(x):
    """A float as three that have the upper 16 bits only, cut."""
    def up(v):
        return (v.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    a = up(x)
    b = up(x - a)
    c = (x - a) - b
    assert np.array_equal(up(c), c)
    return [p.astype(np.float64) for p in (a, b, c)]


def _left_out(x, y):
    p, q = _parts(x), _parts(y)
    return (p[1] * q[2] + p[2] * q[1] + p[2] * q[2]) / (x.astype(np.float64) * y)


def test_what_the_six_products_leave_out():
    # q1 < 2^-7 and q2 < 2^-15 of q's power of two, k's alike: q1 k2 + q2 k1 + q2 k2 is less
    # than (2^-21 + 2^-30) |q| |k|, of the product's sign, and the worst floats come near it
    g = np.random.default_rng(5)
    x, y = (g.standard_normal(200000).astype(np.float32) for _ in range(2))
    worst = np.array([0x3f80ffff], dtype=np.uint32).view(np.float32)
    e = _left_out(x, y)
    assert e.min() >= 0 and e.max() < 2.0 ** -21 + 2.0 ** -30
    assert 2.0 ** -25 < e.mean() < 2.0 ** -24
    assert 2.0 ** -21.1 < _left_out(worst, worst)[0] < 2.0 ** -21


@pytest.mark.gpu
@pytest.mark.parametrize("d,n,t", [(128, 300, 9), (64, 700, 3)])
def test_the_worst_mantissas(d, n, t):
    from paper_2608_02134_gb300 import gmc
    from tests import cache_harness as C
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = C.Case([n], 4, 2, d, "f32", 16, [t])
    w = float(np.array([0x3f80ffff], dtype=np.uint32).view(np.float32)[0])
    share = torch.rand(n, 1, 1, generator=c.gen)  # logits from minus to plus the largest
    c.K[0] = torch.where(torch.rand(n, 2, d, generator=c.gen) < share, w, -w)
    c.q = torch.full((t, 4, d), 2 * w)
    c.put(0, range(n))
    q = c.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(t, 4, device="cuda")
    gmc.attend(c.cache(), q, out, t, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for x in range(t):
        want, z, _, bound, size = C.attention(c.K[0], c.V[0], c.q[x], n - t + x)
        assert size > 0.9 * 2 * math.sqrt(d)
        # a logit: parts left out 2^-21 (4 units of 2^-23), sums in tensor memory cut a unit a
        # step, 8 steps of the largest parts and 8 of the small ones; scaling, exponential and
        # base 32 units.  An error of a logit is one of every weight, twice
        logit = 2.0 ** -23 * ((16 + 4) * size + 32)
        assert bool(((out[x].double().cpu() - want).abs() <= 2 * logit * bound).all()), x
        assert bool(((lse[x].double().cpu() - z).abs() <= logit + 2.0 ** -23 * z.abs()).all()), x
