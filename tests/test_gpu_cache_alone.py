"""Rows computed one by one where a value that some of them do not see is not finite, with the
key axis split over CTAs."""

import math

import pytest
import torch

from tests.test_gpu_cache import _close, _gmc, _harness

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("d,page", [(128, 16), (64, 64), (96, 256)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_bf16_rows_of_a_split_key_axis(value, d, page):
    gmc, C = _gmc(), _harness()
    n, t, bad = 2000, 40, 1979  # seen by the last 21 of the new tokens alone
    c = C.Case([n], 4, 2, d, "bf16", page, [t], spread=2.0)
    c.V[0][bad, :, 5] = value
    c.put(0, [bad])
    cache = c.cache()
    # more than the 256 bytes of a call in one part
    assert gmc.attend_workspace_size(cache, 4, t) > 256
    q = c.q.cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full((t, 4), 7.0, device="cuda")
    gmc.attend(cache, q, out, t, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    clean = c.V[0].clone()
    clean[bad, :, 5] = 0.0
    for x in range(t):
        i = n - t + x
        ref, z, _, bound, size = C.attention(c.K[0], clean, c.q[x], i)
        tol = C.tolerance(c.dt, d, size, roundings=2)
        _close(lse[x], z, torch.ones_like(z), 4 * C.lse_tolerance(d, size), f"lse of {x}")
        if i < bad:
            _close(out[x], ref, bound, tol, f"new token {x}")
        else:
            assert not bool(torch.isfinite(out[x, :, 5].float()).any())
            others = [y for y in range(d) if y != 5]
            _close(out[x][:, others], ref[:, others], bound[:, others], tol, f"new token {x}")
