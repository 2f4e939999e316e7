"""fp32 attention whose products are taken from three bf16 parts of every float: sizes far from
one, infinities that are seen, and logits that grow along the keys."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _harness():
    from tests import cache_harness as C
    return C


def _run(c):
    from paper_2608_02134_gb300 import gmc
    q = c.q.cuda()
    out = torch.full_like(q, math.nan)
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    offsets = c.offsets() if len(set(c.news)) > 1 else None
    gmc.attend(c.cache(), q, out, max(c.news), q_offsets=offsets, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    return out.double().cpu(), lse.double().cpu()


def _tolerance(size):
    """Relative to sum p |v|.  Parts that are left out: 3 x 2^-24 of a product's sum.  Sums in
    tensor memory cut 2^-23 of the running sum a step: d / 16 = 8 steps of the largest parts
    for a logit (of `size` = sum |q k| scale at most), 4 for a turn's output, and as much
    again for the small parts; scaling, the exponential and a weight's base 2^-22 each.  An
    error of a logit is one of every weight, twice (its own and the sum's)."""
    return 2.0 ** -23 * (2 * (16 + 2) * size + 32)


def _check(c, out, lse):
    C = _harness()
    at = 0
    for b, (n, t) in enumerate(zip(c.lens, c.news)):
        for x in range(t):
            want, z, _, bound, size = C.attention(c.K[b], c.V[b], c.q[at + x], n - t + x)
            tol = _tolerance(size)
            assert bool(((out[at + x] - want).abs() <= tol * bound).all()), (b, x)
            assert bool(((lse[at + x] - z).abs() <= tol * (1 + z.abs())).all()), (b, x)
        at += t


@pytest.mark.parametrize("d", [64, 128, 100])
def test_sizes_far_from_one(d):
    c = _harness().Case([200, 70], 4, 2, d, "f32", 16, [70, 3])
    c.q *= 2.0 ** -40
    for b in range(2):
        c.K[b] *= 2.0 ** 40
        c.V[b] *= 2.0 ** 100
        c.put(b, range(c.lens[b]))
    _check(c, *_run(c))


def test_values_near_the_largest_float():
    # the upper part of a float is cut, not rounded, or it would pass the largest bf16
    # the one key has the weight 1, and the three parts of a value add up to it exactly
    c = _harness().Case([1], 2, 1, 128, "f32", 16, [1])
    big = torch.finfo(torch.float32).max
    c.V[0] = big * (1.0 - 2.0 ** -20 * torch.arange(128)).reshape(1, 1, 128).float()
    c.V[0][:, :, ::2] *= -1.0
    c.put(0, [0])
    out, _ = _run(c)
    assert torch.equal(out[0], c.V[0].double().expand(1, 2, 128)[0])


def test_logits_that_grow_along_the_keys():
    # every turn's maximum is some powers of two above the last one's
    c = _harness().Case([1000], 4, 2, 128, "f32", 16, [9])
    c.K[0] *= torch.linspace(0.05, 4.0, 1000)[:, None, None]
    c.put(0, range(1000))
    _check(c, *_run(c))


def test_keys_of_minus_infinity_take_no_weight():
    c = _harness().Case([300], 2, 2, 64, "f32", 16, [40])
    c.q[:, :, 3] = c.q[:, :, 3].abs() + 0.5
    for j in (7, 150, 280):
        c.K[0][j, :, 3] = -math.inf
    c.put(0, range(300))
    out, lse = _run(c)
    for j in (7, 150, 280):  # the definition without them
        c.K[0][j] = 0.0
        c.K[0][j, :, 3] = -1e6
    C = _harness()
    for x in range(40):
        want, z, _, bound, size = C.attention(c.K[0], c.V[0], c.q[x], 260 + x)
        tol = 2.0 ** -24 * (8.0 * 8.0 * 60.0 + 64.0)  # computed row by row in fp32
        assert bool(((out[x] - want).abs() <= tol * bound).all()), x
        assert bool(((lse[x] - z).abs() <= tol * (1 + z.abs())).all()), x


def test_the_same_bits_every_time():
    c = _harness().Case([700, 333, 64], 28, 4, 128, "f32", 32, [100, 1, 64])
    first = _run(c)
    for _ in range(3):
        again = _run(c)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
