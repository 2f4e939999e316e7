"""Running scores over 4 bits: what a window hides keeps its score, whatever the seen keys hold."""

import pytest
import torch

from tests.test_gpu_cache4 import _decode, _gmc, _h, _lib  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("room", [None, 6016], ids=["a block a pair", "stretches"])
@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("window,sinks", [(100, 4), (50, 0), (33, 40), (1, 1)])
@pytest.mark.parametrize("H,Hkv,d", [(8, 2, 128), (3, 1, 64), (18, 1, 256)])
def test_nan_in_a_seen_key_leaves_unseen_scores(H, Hkv, d, window, sinks, append, room):
    C, gmc = _h(), _gmc()
    width = None if room is None else room // 16
    c = C.Case4([500, 333], H, Hkv, d, 16, width=width)
    n, bad = 500, 499 - (append or window > 1)
    if append and window == 1:
        c.raw_K[0][-1] = float("nan")
    else:
        c.blank(0, bad)
    unseen = slice(sinks, n - window)
    out, _, before, new = _decode(c, window, sinks, append, True, max_len=room)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and bool(torch.isnan(out[0]).all())
    assert bool(torch.isfinite(out[1]).all())
    assert torch.equal(new[0, :, unseen].cpu(), before[0, :, unseen])
    assert bool(torch.isnan(new[0, :, n - window:n]).all())
    assert bool(torch.isfinite(new[1, :, :333]).all()) and bool((new[0, :, n:] == 9.0).all())
    # in place
    cache, scores = c.cache(max_len=room or 503), before.cuda()
    k, v = (torch.stack([x[-1] for x in r]).cuda() for r in (c.raw_K, c.raw_V))
    gmc.decode(cache, c.q.cuda(), out, k if append else None, v if append else None, window, sinks,
               scores=scores, out_scores=scores)
    torch.cuda.synchronize()
    assert torch.equal(scores[0, :, unseen].cpu(), before[0, :, unseen])
    assert bool(torch.isnan(scores[0, :, n - window:n]).all())
