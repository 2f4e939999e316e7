"""Calls whose sequences all have no new rows: nothing to do, with tensors of no elements."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_at_all(dtype):
    from paper_2608_02134_gb300 import gmc
    from tests import cache_harness as C
    c = C.Case([20, 7], 4, 2, 64, dtype, 16)
    cache = c.cache()
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    rows, q = (torch.empty(0, h, 64, dtype=c.dt, device="cuda") for h in (2, 4))
    gmc.cache_append(cache, rows, rows, 5, offsets=none)
    gmc.cache_append(cache, rows, None, 5, offsets=none)
    gmc.attend(cache, q, torch.empty_like(q), 5, q_offsets=none,
               lse=torch.empty(0, 4, device="cuda"))
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for dev, host in ((c.dk, c.pool_k), (c.dv, c.pool_v)):
        assert torch.equal(dev.cpu().view(torch.uint8), host.view(torch.uint8))
