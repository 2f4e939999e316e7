"""Attention over pages of 4 bits that do not hold whole runs of 16 keys, read from the codes."""

import pytest
import torch

from tests.test_gpu_cache4 import _attend, _close, _gmc, _h, _lib  # noqa: F401

pytestmark = pytest.mark.gpu

# lens, news, H, Hkv: one part of the key axis, and several
ONE = ([130, 20, 77], [9, 4, 5], 14, 2)
SEVERAL = ([700], [11], 8, 2)


@pytest.mark.parametrize("lens,news,H,Hkv", [ONE, SEVERAL], ids=["one part", "parts"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 20), (64, 3)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 4, 7, 8, 12, 15, 24, 40])
def test_attend_over_pages_of_any_size(page, d, window, sinks, lens, news, H, Hkv):
    from tests import cache_harness as A
    C = _h()
    # behind every part codes and scales of another size, none of them NaN
    c = C.Case4(lens, H, Hkv, d, page, news, spread=2.0, pad=16 * (d // 2 + d // 16 + 4))
    for pool in (c.pool_k, c.pool_v):
        pool[..., page * d * 9 // 16:] = 0x50
    cap = min(max(lens) + 1, c.table.shape[1] * page)
    size = _gmc().attend_workspace_size(c.cache(max_len=cap), H, max(news))
    assert (size > 256) == (len(lens) == 1)        # parts
    assert size < c.B * cap * Hkv * d * 4          # no room to unpack in
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and bool((out[-1] == 7.0).all())
    at = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        small = 2.0 ** -25 * c.V[b].double().abs().sum(0).repeat_interleave(H // Hkv, 0)
        for x in range(t):
            ref, z, _, bound, s = A.attention(c.K[b], c.V[b], c.q[at + x], n - t + x, window,
                                              sinks)
            tol = C.tolerance(c, s)
            _close(out[at + x], ref, bound + small / tol, tol, f"sequence {b}, new token {x}")
            _close(lse[at + x], z, torch.ones_like(z), A.lse_tolerance(d, s) * 4, "lse")
        at += t
