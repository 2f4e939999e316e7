"""Windows: pages that no query sees are not looked up, and a window as wide as integers go is
none."""

import pytest
import torch

from tests.test_gpu_cache import _attend, _check_attend, _close, _decode, _gmc, _harness

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _release_unseen_pages(c, window, sinks, to):
    """The table's entries of pages that none of the call's queries sees, set to `to`; how many."""
    C, released = _harness(), 0
    for b, (n, t) in enumerate(zip(c.lens, c.news)):
        any_row = torch.zeros(n, dtype=torch.bool)
        for i in range(max(0, n - t), n):
            any_row |= C.seen(n, i, window, sinks)
        for p in range(c.table.shape[1]):
            if not bool(any_row[p * c.page:(p + 1) * c.page].any()):
                c.table[b, p] = to(c)
                released += 1
    return released


RELEASED = {"minus one": lambda c: -1, "past the pool": lambda c: c.pool_k.shape[0],
            "another's": lambda c: _page_of_nobody(c)}


def _page_of_nobody(c):
    """A page that the table does not hold: all NaN."""
    held = set(c.table.flatten().tolist())
    return next(p for p in range(c.pool_k.shape[0]) if p not in held)


WINDOWS = [  # lens, news, H, Hkv, d, dtype, page, window, sinks
    ([700, 333], [40, 40], 4, 2, 128, "bf16", 16, 70, 3),
    ([700, 333], [40, 40], 4, 2, 128, "bf16", 16, 70, 0),
    ([900], [9], 28, 4, 128, "bf16", 8, 33, 20),
    ([900], [200], 4, 2, 64, "bf16", 48, 50, 50),
    ([900], [20], 4, 2, 64, "bf16", 128, 40, 1),
    ([900], [20], 4, 2, 64, "bf16", 256, 40, 1),
    ([900], [20], 4, 2, 64, "bf16", 136, 140, 137),
    ([700, 333], [40, 40], 4, 2, 128, "f32", 16, 70, 3),
    ([700], [40], 4, 2, 256, "f32", 16, 70, 3),
    ([700], [40], 4, 2, 128, "bf16", 20, 70, 3),
]


@pytest.mark.parametrize("released", list(RELEASED))
@pytest.mark.parametrize("lens,news,H,Hkv,d,dtype,page,window,sinks", WINDOWS)
def test_attend_does_not_look_up_pages_that_nobody_sees(lens, news, H, Hkv, d, dtype, page, window,
                                                        sinks, released):
    c = _harness().Case(lens, H, Hkv, d, dtype, page, news, spread=2.0)
    assert _release_unseen_pages(c, window, sinks, RELEASED[released]) > 0
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, window, sinks)


@pytest.mark.parametrize("H,Hkv,dtype,page,window,sinks", [
    (152, 152, "bf16", 16, 70, 3), (152, 152, "bf16", 64, 130, 0), (160, 160, "f32", 16, 70, 3)])
def test_prompts_that_fill_the_gpu_do_not_either(H, Hkv, dtype, page, window, sinks):
    c = _harness().Case([500], H, Hkv, 64, dtype, page, [40], width=-(-2560 // page))
    assert _release_unseen_pages(c, window, sinks, RELEASED["minus one"]) > 0
    out, lse = _attend(c, window, sinks, max_len=c.table.shape[1] * page)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, window, sinks)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 128), ("f32", 16)])
def test_decode_does_not_look_up_pages_that_nobody_sees(dtype, page):
    C = _harness()
    c = C.Case([700, 333], 8, 2, 128, dtype, page, spread=2.0)
    assert _release_unseen_pages(c, 50, 3, RELEASED["minus one"]) > 0
    out, lse, _ = _decode(c, 50, 3, append=False)
    assert int(c.status.item()) == 0
    for b, n in enumerate(c.lens):
        ref, z, _, bound, size = C.attention(c.K[b], c.V[b], c.q[b], n - 1, 50, 3)
        _close(out[b], ref, bound, C.tolerance(c.dt, 128, size), f"sequence {b}")
        _close(lse[b], z, torch.ones_like(z), 4 * C.lse_tolerance(128, size), "lse")


def test_a_page_that_is_seen_in_part_is_still_looked_at():
    # the first page that the window reaches into, and the last of the sinks
    gmc, C = _gmc(), _harness()
    for p in (0, 38):
        c = C.Case([700], 4, 2, 128, "bf16", 16, [8])
        c.table[0, p] = -1
        _attend(c, 70, 3)  # the first new token sees places 623 and on: page 38 holds the last one
        torch.cuda.synchronize()
        assert int(c.status.item()) == gmc.STATUS_CACHE


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 12, 2 ** 30])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 64), ("f32", 256)])
def test_attend_with_a_window_as_wide_as_integers_go(dtype, d, window):
    # the first queries of the first sequence lie before it
    c = _harness().Case([10, 300], 4, 2, d, dtype, 16, [20, 20])
    out, lse = _attend(c, window, 2)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_window_of_all_places_is_none(dtype):
    c = _harness().Case([300, 40], 4, 2, 128, dtype, 16, [60, 40])
    want = _attend(c)
    got = _attend(c, 300, 2)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
