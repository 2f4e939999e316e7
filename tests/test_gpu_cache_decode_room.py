"""Decoding of short sequences in a cache with room for long ones (stretches of the whole
batch, joined) and of batches that fill the GPU (a CTA a sequence and key head)."""

import pytest
import torch

from tests import test_gpu_cache as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _check(c, window, sinks, max_len):
    from tests import cache_harness as C
    S = max_len + 3
    scores = torch.rand(c.B, c.Hkv, S, generator=c.gen)
    out, lse, so = base._decode(c, window, sinks, scores, max_len=max_len)
    assert int(c.status.item()) == 0
    for b, n in enumerate(c.lens):
        ref, z, w, bound, size = C.attention(c.K[b], c.V[b], c.q[b], n - 1, window, sinks)
        base._close(out[b], ref, bound, C.tolerance(c.dt, c.d, size), f"sequence {b}")
        base._close(lse[b], z, torch.ones_like(z), 4 * C.lse_tolerance(c.d, size), "lse")
        want = scores[b].double().clone()
        want[:, n - 1] = 0.0
        gain = w.reshape(c.Hkv, c.H // c.Hkv, n).sum(1)
        want[:, :n] += gain
        base._close(so[b, :, :n], want[:, :n], gain + want[:, :n],
                    4 * C.lse_tolerance(c.d, size), f"scores of {b}")
        assert bool((so[b, :, n:] == -5.0).all())


@pytest.mark.parametrize("lens,H,Hkv,d,dtype,page,window,sinks", base.DECODE)
def test_short_sequences_with_room(lens, H, Hkv, d, dtype, page, window, sinks):
    from tests import cache_harness as C
    width = -(-max(2600, max(lens)) // page)
    c = C.Case(lens, H, Hkv, d, dtype, page, spread=2.0, width=width)
    _check(c, window, sinks, width * page)


FULL = [  # lens, H, Hkv, d, dtype, page, window, sinks
    ([300, 17, 1, 640, 128, 129, 16, 500, 77, 2] * 2, 28, 4, 128, "bf16", 16, 0, 0),
    ([300, 17, 1, 640, 128, 129, 16, 500, 77, 2], 16, 8, 64, "bf16", 48, 100, 3),
    ([300, 17, 1, 200, 128] * 4, 4, 4, 128, "f32", 16, 0, 0),
    ([300, 17, 1, 200, 128] * 3, 6, 6, 256, "bf16", 7, 0, 0),
    ([180, 17, 1, 100, 128] * 3, 12, 6, 256, "f32", 32, 50, 1),
    ([600, 3, 90, 16] * 5, 40, 4, 36, "f32", 5, 0, 0),
]


@pytest.mark.parametrize("lens,H,Hkv,d,dtype,page,window,sinks", FULL)
def test_batches_that_fill_the_gpu(lens, H, Hkv, d, dtype, page, window, sinks):
    from tests import cache_harness as C
    c = C.Case(lens, H, Hkv, d, dtype, page, spread=2.0)
    _check(c, window, sinks, max(lens))


def test_an_empty_sequence_among_others():
    from tests import cache_harness as C
    c = C.Case([64, 5] * 10, 28, 4, 128, "bf16", 16)
    c.lens[7] = 0
    scores = torch.rand(20, 4, 64, generator=c.gen)
    out, lse, so = base._decode(c, scores=scores, append=False, max_len=64)
    assert torch.equal(out[7], torch.zeros_like(out[7]))
    assert bool((lse[7] == -float("inf")).all())
    assert bool((so[7] == -5.0).all())
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse[:7]).all())
