"""CPU tests: calls without rows take NULL for what has no elements, others do not."""

import pytest

from tests.test_cache_args import FAKE, _append, _attend, _attn, _cache, gmc  # noqa: F401


def test_no_rows_need_no_pointers(gmc):  # noqa: F811
    c, a = _cache(gmc), _attn(gmc)
    assert _append(gmc, c, rows=0, off=FAKE, k=None, v=None) == gmc.GMC_OK
    assert _attend(gmc, c, a, rows=0, off=FAKE, q=None, out=None, ws=None, n=0) == gmc.GMC_OK


@pytest.mark.parametrize("change", [dict(rows=1, off=FAKE), dict(rows=6, T=3)])
def test_rows_do(gmc, change):  # noqa: F811
    c, a = _cache(gmc), _attn(gmc)
    assert _append(gmc, c, k=None, **change) == gmc.GMC_ERR_ARG
    assert _attend(gmc, c, a, q=None, **change) == gmc.GMC_ERR_ARG
    assert _attend(gmc, c, a, out=None, **change) == gmc.GMC_ERR_ARG


def test_the_other_checks_stay(gmc):  # noqa: F811
    # without rows, a bad cache, head count or row count is refused all the same
    a = _attn(gmc)
    assert _append(gmc, _cache(gmc, d=0), rows=0, off=FAKE) == gmc.GMC_ERR_ARG
    assert _attend(gmc, _cache(gmc), _attn(gmc, H=30), rows=0, off=FAKE) == gmc.GMC_ERR_ARG
    assert _attend(gmc, _cache(gmc), a, rows=0) == gmc.GMC_ERR_ARG  # B * T rows without offsets


@pytest.mark.parametrize("T", [2 ** 30 + 1, 2 ** 31 - 1])
def test_more_rows_a_sequence_than_places_are_counted_in(gmc, T):  # noqa: F811
    # the tiles of so many rows do not fit 32 bits
    c, a = _cache(gmc), _attn(gmc)
    assert _append(gmc, c, T=T, off=FAKE) == gmc.GMC_ERR_UNSUPPORTED
    assert _attend(gmc, c, a, T=T, off=FAKE) == gmc.GMC_ERR_UNSUPPORTED
    assert gmc.lib().gmc_attend_workspace_size(c, 28, T) == 0
    assert gmc.lib().gmc_attend_workspace_size(c, 28, 2 ** 30) > 0
