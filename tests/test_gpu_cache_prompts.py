"""bf16 attention of prompts that fill the GPU on a cache that may grow long: a CTA alternates
between two tiles of queries, and the key axis is not split."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _harness():
    from tests import cache_harness as C
    return C


def _run(c, window=0, sinks=0):
    from paper_2608_02134_gb300 import gmc
    rows = sum(c.news)
    out = torch.full((rows, c.H, c.d), math.nan, dtype=c.dt, device="cuda")
    lse = torch.full((rows, c.H), math.nan, device="cuda")
    offsets = c.offsets() if len(set(c.news)) > 1 else None
    # as many key heads and sequences as fill the GPU, room for 2,400 tokens and more: no
    # split of the keys and two tiles a CTA
    gmc.attend(c.cache(max_len=c.table.shape[1] * c.page), c.q.cuda(), out, max(c.news),
               q_offsets=offsets, window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    return out.double().cpu(), lse.double().cpu()


def _check(c, out, lse, window=0, sinks=0, rows=None):
    """Every row of the given new tokens (all of them by default), all heads at once."""
    C = _harness()
    at = 0
    for b, (n, t) in enumerate(zip(c.lens, c.news)):
        for x in range(t):
            if rows is not None and (b, x) not in rows:
                continue
            want, z, _, bound, size = C.attention(c.K[b], c.V[b], c.q[at + x], n - t + x, window,
                                                  sinks)
            tol = C.tolerance(c.dt, c.d, size, roundings=2)
            assert bool(((out[at + x] - want).abs() <= tol * bound + 1e-30).all()), (b, x)
            seen = torch.isfinite(z)
            assert bool(((lse[at + x] - z).abs()[seen] <= 4 * C.lse_tolerance(c.d, size)).all())
            assert bool((lse[at + x][~seen] == -math.inf).all())
        at += t


PROMPTS = [  # lens, news, H, Hkv, d, page, window, sinks
    ([140], [140], 152, 152, 128, 16, 0, 0),
    ([300, 41], [130, 41], 160, 80, 128, 64, 0, 0),
    ([129, 257, 1], [1, 257, 1], 60, 60, 128, 8, 0, 0),
    ([300, 90], [75, 74], 112, 16, 128, 32, 0, 0),
    ([700], [73], 154, 22, 128, 128, 100, 5),
    ([520, 513], [400, 20], 80, 40, 96, 256, 150, 0),
    ([260, 260], [100, 129], 80, 80, 72, 16, 33, 1),
]


@pytest.mark.parametrize("lens,news,H,Hkv,d,page,window,sinks", PROMPTS)
def test_prompts_match_the_definition(lens, news, H, Hkv, d, page, window, sinks):
    c = _harness().Case(lens, H, Hkv, d, "bf16", page, news, spread=2.0, width=-(-2560 // page))
    out, lse = _run(c, window, sinks)
    t = sum(news)
    pick = None
    if t * H > 8000:  # rows at the edges of tiles and turns, and some between
        pick = {(b, x) for b, k in enumerate(news) for x in range(k)
                if x in (0, 1, k - 1, 17, 18, 35, 36, 53, 54, 71, 72) or x % 64 in (0, 63)
                or x % 23 == 5}
    _check(c, out, lse, window, sinks, pick)
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("page,column", [(16, 5), (128, 70)])
def test_prompts_keep_values_that_are_not_seen_from_a_row(page, column):
    # a column of either half of the values
    C = _harness()
    c = C.Case([300], 152, 152, 128, "bf16", page, [200], width=-(-2560 // page))
    bad = {150: math.nan, 220: math.inf, 299: -math.inf}
    for j, x in bad.items():
        c.V[0][j, :, column] = x
        c.put(0, [j])
    window, sinks = 40, 3
    out, lse = _run(c, window, sinks)
    clean = [x for x in range(200)
             if not any(bool(C.seen(300, 100 + x, window, sinks)[j]) for j in bad)]
    _check(c, out, lse, window, sinks, {(0, x) for x in clean[::9] + clean[-1:]})
    for x in clean:
        assert bool(torch.isfinite(out[x]).all()), x
    for x in (55, 125):
        assert not bool(torch.isfinite(out[x, :, column]).any())
        assert bool(torch.isfinite(out[x, :, column ^ 64]).all())


def test_prompts_give_the_same_bits_every_time():
    c = _harness().Case([1000, 333], 112, 16, 128, "bf16", 64, [600, 333], width=40)
    first = _run(c)
    for _ in range(4):
        again = _run(c)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
