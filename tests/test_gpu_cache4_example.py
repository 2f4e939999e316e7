"""The example that runs the cache's operators behind a compression, over 4 bits with positions."""

import pytest
import torch

from tests.test_gpu_cache_example import _example

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def test_every_decoded_token_hands_out_its_whole_weight():
    # as over bf16: every step adds the weight 1 of each of the 7 query heads of a key head
    r = _example().main(steps=20, verbose=False, four_bits=True)
    assert r["evictions"] == 0 and r["length"] == 321 + 24 + 20
    total = r["scores"].double().sum(-1)
    assert bool(((total - 20 * 7).abs() < 20 * 7 * 2.0 ** -16).all())
    assert bool((r["scores"][..., r["length"]:] == 0).all())


def test_decoding_goes_on_after_evictions():
    r = _example().main(prompts=1, steps=140, verbose=False, four_bits=True)
    assert r["evictions"] == 2 and r["length"] == 300 + (140 - 39 - 84)
    assert bool((r["scores"][..., :r["length"]] >= 0).all())
    assert bool((r["scores"][..., r["length"]:] == 0).all())
