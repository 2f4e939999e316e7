"""Attention over 4 bits where one key outweighs all others: small weights are not lost.

A weight is rounded to half after its reference, within 2^8 of the largest so far, is put to 2^7:
it is off by at most half a step, 2^-11 of itself, or 2^-25 / 2^7 = 2^-32 of the reference where
it is that small.  So an output row is off by tolerance() and 2^-32 sum |v| / (sum of weights),
where the sum of weights is at least the reference's own.
"""

import math

import pytest
import torch

from tests.test_gpu_cache4 import _attend, _close, _decode, _gmc, _h, _lib  # noqa: F401

pytestmark = pytest.mark.gpu


def _case(lens, H, Hkv, d, page, bits, at=0, news=None, width=None):
    """Key `at` of every sequence outweighs the others by about 2^bits; its value is 0, theirs
    are 0.5 to 2.5: all of the output comes from the small weights."""
    C = _h()
    c = C.Case4(lens, H, Hkv, d, page, news, width=width)
    c.q[:] = bits * math.log(2.0) / (1.5 * math.sqrt(d))
    for b in range(c.B):
        k, v = c.raw_K[b], c.raw_V[b]
        k.copy_((k.float() * 2.0 ** -6).bfloat16())
        v.copy_((v.float().abs().clamp(max=2.0) + 0.5).bfloat16())
        k[at:at + 1] = 1.5  # exact in 4 bits
        v[at:at + 1] = 0.0
        c.K[b], c.V[b] = (C.unpack(*C.pack(x)).to(torch.bfloat16) for x in (k, v))
        c.fill(b, range(lens[b]))
    return c


def _check(c, b, n, row, out, lse, what):
    from tests import cache_harness as A
    ref, z, _, bound, size = A.attention(c.K[b], c.V[b], c.q[row], n - 1)
    tol = _h().tolerance(c, size)
    small = 2.0 ** -32 * c.V[b][:n].double().abs().sum(0).repeat_interleave(c.H // c.Hkv, 0)
    _close(out, ref, bound + small / tol, tol, what)
    _close(lse, z, torch.ones_like(z), A.lse_tolerance(c.d, size) * 4, what + ", lse")


BITS = [(26.0, 0), (28.5, 0), (26.0, 5), (7.9, 70), (8.1, 70), (15.5, 70)]


@pytest.mark.parametrize("bits,at", BITS)
@pytest.mark.parametrize("room", [None, 6016], ids=["a block a pair", "stretches"])
@pytest.mark.parametrize("H,Hkv,d", [(7, 1, 128), (16, 1, 128), (4, 2, 64), (12, 1, 64),
                                     (8, 1, 256)])
def test_decode_keeps_small_weights(H, Hkv, d, room, bits, at):
    lens = [96, 75, 1500]
    c = _case(lens, H, Hkv, d, 32, bits, at, width=None if room is None else room // 32)
    out, lse, _, _ = _decode(c, 0, 0, True, False, max_len=room)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        _check(c, b, n, b, out[b], lse[b], f"sequence {b}")


@pytest.mark.parametrize("bits,at", BITS)
@pytest.mark.parametrize("lens,news", [([130, 200, 90], [9, 8, 9]), ([1900], [12])],
                         ids=["one part", "parts"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_from_the_codes_keeps_small_weights(d, lens, news, bits, at):
    c = _case(lens, 14, 2, d, 32, bits, at, news)
    size = _gmc().attend_workspace_size(c.cache(max_len=max(lens) + 1), 14, max(news))
    assert size < c.B * max(lens) * 2 * d * 4  # no room to unpack in
    assert (size > 256) == (len(lens) == 1)
    out, lse = _attend(c, 0, 0)
    torch.cuda.synchronize()
    row = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        for x in range(t):
            _check(c, b, n - t + x + 1, row, out[row], lse[row], f"sequence {b}, new token {x}")
            row += 1


def test_attend_of_256_channels_and_of_one_token_keep_small_weights():
    for d, news in ((256, [3, 2]), (128, [1, 1])):
        lens = [64, 90]
        c = _case(lens, 8, 2, d, 16, 26.0, 0, news)
        cache, q = c.cache(), c.q.cuda()
        out, lse = torch.empty_like(q), torch.empty(len(q), 8, device="cuda")
        offsets = c.offsets() if d == 256 else None
        _gmc().attend(cache, q, out, max(news), q_offsets=offsets, lse=lse)
        torch.cuda.synchronize()
        row = 0
        for b, (n, t) in enumerate(zip(lens, news)):
            for x in range(t):
                _check(c, b, n - t + x + 1, row, out[row], lse[row], f"d {d}, sequence {b}")
                row += 1


@pytest.mark.parametrize("power", [16, 20, 23, 26])
def test_enormous_logits_give_finite_rows(power):
    """A weight that is off by the rounding of a logit of 2^power is still no infinity: every
    output is an average of values."""
    C = _h()
    c = C.Case4([700, 1300, 90], 14, 2, 128, 32, [9, 8, 9])
    c.q = (c.q.float() * 2.0 ** power).bfloat16()
    out, lse = _attend(c, 0, 0)
    one = C.Case4([700, 1300, 90], 14, 2, 128, 32)
    one.q = (one.q.float() * 2.0 ** power).bfloat16()
    new, z, _, _ = _decode(one, 0, 0, True, False)
    torch.cuda.synchronize()
    for got, s, case in ((out[:-1], lse, c), (new, z, one)):
        top = max(float(x.double().abs().max()) for x in case.V)
        assert bool((got.double().abs() <= top * (1 + 2.0 ** -7)).all())
        assert bool(torch.isfinite(s).all())
