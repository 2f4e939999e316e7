"""The example that runs the cache's operators behind a compression."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _example():
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location(
        "decode_after_compression", os.path.join(root, "examples", "decode_after_compression.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_every_decoded_token_hands_out_its_whole_weight():
    # without an eviction, every step adds the weight 1 of each of the 7 query heads of a
    # key head to its keys' scores; 20 fp32 softmaxes are off by some 2^-20 together
    r = _example().main(steps=20, verbose=False)
    assert r["evictions"] == 0 and r["length"] == 321 + 24 + 20
    total = r["scores"].double().sum(-1)
    assert bool(((total - 20 * 7).abs() < 20 * 7 * 2.0 ** -16).all())
    assert bool((r["scores"][..., r["length"]:] == 0).all())


def test_decoding_goes_on_after_evictions():
    r = _example().main(prompts=1, steps=140, verbose=False)
    assert r["evictions"] == 2 and r["length"] == 300 + (140 - 39 - 84)
    assert bool((r["scores"][..., :r["length"]] >= 0).all())
    assert bool((r["scores"][..., r["length"]:] == 0).all())
