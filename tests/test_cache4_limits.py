"""CPU tests of the largest rows that the rotated append takes (nothing launches)."""

import pytest

from tests.test_cache4_args import _cache4, _rope, _turned, gmc  # noqa: F401
from tests.test_cache_args import FAKE, _cache


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("Hkv,G,fits", [(4096, 128, True), (8192, 64, True), (4097, 128, False),
                                        (65535, 128, False), (65535, 9, False)])
def test_a_row_of_queries_has_at_most_2_26_values(gmc, kind, Hkv, G, fits):  # noqa: F811
    part = 16 * 72
    c = _cache4(gmc, B=1, Hkv=Hkv, num_pages=1, max_pages=1, page_stride=Hkv * part) \
        if kind == "fp4" else _cache(gmc, B=1, Hkv=Hkv, num_pages=1, max_pages=1)
    want = gmc.GMC_OK if fits else gmc.GMC_ERR_UNSUPPORTED
    # no rows: the arguments are checked, nothing is launched
    assert _turned(gmc, c, _rope(gmc, H=Hkv * G), rows=0, off=FAKE) == want
    assert _turned(gmc, c, _rope(gmc, H=0), rows=0, off=FAKE, q=None, out=None) == gmc.GMC_OK
